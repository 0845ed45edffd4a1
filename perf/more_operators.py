"""Workloads of the attention around the cache pages, for measurement against their plain forms.

Five kinds, in the order in which a model's pass over a prompt or a block meets them:

  rotate  norms of queries and keys for each head and the rotation by position, in the rows of a fused projection
  prompt  causal attention over whole prompts of different lengths, packed one behind the other, with grouped heads
  append  keys and values of new rows into the cache's pages, in 4 bits with a scale and an offset per token and head
  attend  attention of a block's rows over the pages; where asked for, the weight that every cached token was given
  evict   shortening caches to a budget by that weight, pages given back

Where ``own`` is false everything is computed with elementary torch operations; where it is true, with the package's calls.

A page of one layer's keys or values is [kv_heads, page_tokens / 8] units of eight tokens: 8 D / 2 bytes of codes, then eight pairs of
bf16 numbers (scale, offset); a value is scale * code + offset.  Code e of eight neighbours is in the four bits from bit
4 (e / 2) + 16 (e mod 2) on of a 32-bit word.  A unit of keys holds its words by token; a unit of values holds word 8 h + g of token
2 t + o at place ((4 g + t) 2 + o) D/64 + h.
"""
import torch

own = False

DEV = "cuda"
UNIT = 8            # tokens of a unit


def listed():
    return [
        # one sequence's verification block far into its text: k = 8 drafted tokens and the bonus row
        {"name": "rotate_block", "kind": "rotate", "rows": 9, "heads": 32, "kv_heads": 8, "d": 128, "rotary": 128, "interleaved": False, "norm": True, "far": 120000},
        # the rows of a batch of prompts, pairs side by side
        {"name": "rotate_prompt", "kind": "rotate", "rows": 8195, "heads": 32, "kv_heads": 8, "d": 128, "rotary": 128, "interleaved": True, "norm": True, "far": 8192},
        # a drafter's short prompts of different lengths, as many key heads as query heads
        {"name": "prompt_short", "kind": "prompt", "lens": "61,130,7,384", "heads": 16, "kv_heads": 16, "d": 64},
        # the target's prompts: one long, others of a batch behind it
        {"name": "prompt_long", "kind": "prompt", "lens": "8192,1111,2500,389", "heads": 32, "kv_heads": 8, "d": 128},
        # the block of every sequence of a batch
        {"name": "append_block", "kind": "append", "B": 64, "most": 9, "len": 2000, "kv_heads": 8, "d": 128, "page_tokens": 16},
        # prompts of a batch into empty caches
        {"name": "append_prompt", "kind": "append", "B": 12, "most": 1500, "len": 0, "kv_heads": 8, "d": 128, "page_tokens": 64},
        # a token of one sequence
        {"name": "attend_one", "kind": "attend", "B": 1, "most": 1, "len": 4000, "heads": 32, "kv_heads": 8, "d": 128, "page_tokens": 16, "weigh": False},
        # the verification blocks of a batch: k = 8 and the bonus row
        {"name": "attend_block", "kind": "attend", "B": 64, "most": 9, "len": 8192, "heads": 32, "kv_heads": 8, "d": 128, "page_tokens": 16, "weigh": False},
        # single tokens over long texts of very different lengths
        {"name": "attend_long", "kind": "attend", "B": 16, "most": 1, "len": 65536, "heads": 32, "kv_heads": 8, "d": 128, "page_tokens": 64, "weigh": False},
        # a drafter with narrow heads whose cache is kept short by weight: blocks of five
        {"name": "attend_weights", "kind": "attend", "B": 33, "most": 5, "len": 3001, "heads": 20, "kv_heads": 4, "d": 64, "page_tokens": 48, "weigh": True},
        # one sequence's cache cut from just over its budget, all 32 layers
        {"name": "evict_one", "kind": "evict", "B": 1, "len": 4300, "budget": 4096, "first": 4, "recent": 256, "planes": 64, "kv_heads": 8, "d": 128, "page_tokens": 16},
        # a batch's caches after their prompts, cut to half
        {"name": "evict_batch", "kind": "evict", "B": 32, "len": 2048, "budget": 1024, "first": 4, "recent": 128, "planes": 64, "kv_heads": 4, "d": 128, "page_tokens": 32},
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["rotate", "prompt", "prompt", "append", "attend", "attend", "attend", "evict"])
    d = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 8, 8])
    if kind == "rotate":
        heads = kv * rng.choice([1, 2, 4, 5, 8])
        rows = min(_log(rng, 1, 16384), 8195 * 40 * 128 // ((heads + kv) * d))
        return {"kind": kind, "rows": rows, "heads": heads, "kv_heads": kv, "d": d, "rotary": rng.choice([d, d, d // 2]), "interleaved": rng.random() < 0.4,
                "norm": rng.random() < 0.7, "far": _log(rng, 100, 1000000)}
    if kind == "prompt":
        kv = rng.choice([2, 4, 8])
        heads = kv * rng.choice([1, 2, 3, 4])
        n = rng.randint(1, 8)
        lens = [_log(rng, 1, min(8192, 16384 // n)) for _ in range(n)]
        return {"kind": kind, "lens": ",".join(map(str, lens)), "heads": heads, "kv_heads": kv, "d": d}
    P = rng.choice([8, 16, 32, 48, 64])
    if kind == "append":
        B = _log(rng, 1, 128)
        most = _log(rng, 1, max(2, 18000 // B))
        return {"kind": kind, "B": B, "most": most, "len": rng.choice([0, _log(rng, 10, 2000)]), "kv_heads": kv, "d": d, "page_tokens": P}
    if kind == "attend":
        B, most = _log(rng, 1, 128), rng.randint(1, 12)
        room = 16 * 65536 * 8 * 128 // (B * kv * d * (1 if most == 1 else 4))
        return {"kind": kind, "B": B, "most": most, "len": _log(rng, 20, min(65536, room)), "heads": kv * rng.choice([1, 2, 4, 4, 5, 8]), "kv_heads": kv, "d": d,
                "page_tokens": P, "weigh": rng.random() < 0.3}
    B, length, kv = _log(rng, 1, 64), _log(rng, 300, 8192), rng.choice([2, 4, 8])
    planes = 2 * max(1, min(32, 32 * 2048 * 64 * 4 * 128 // (2 * B * length * kv * d)))
    return {"kind": kind, "B": B, "len": length, "budget": int(length * rng.uniform(0.3, 1.0)), "first": rng.choice([0, 4, 17]), "recent": rng.choice([0, 32, 64]),
            "planes": planes, "kv_heads": kv, "d": d, "page_tokens": P}


# ------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _ints(g, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=g, device=DEV, dtype=torch.int32)


def _normal(g, shape):
    return torch.randn(shape, generator=g, device=DEV)


def _page_bytes(kv_heads, d, page_tokens):
    return kv_heads * (page_tokens // UNIT) * (UNIT * d // 2 + UNIT * 4)


def _starts(counts):
    """[B] counts -> [B + 1] int32 row numbers at which each sequence's rows begin."""
    return torch.cat([torch.zeros(1, dtype=torch.int32, device=DEV), counts.cumsum(0).to(torch.int32)])


def _tables(g, s, length, most_tokens):
    """Page tables of sequences of `length` [B] tokens, their pages scattered over a pool with some to spare."""
    P, B = s["page_tokens"], length.numel()
    most = (most_tokens + P - 1) // P
    n_pages = B * most + 5
    held = (length + P - 1) // P
    ids = torch.randperm(n_pages, generator=g, device=DEV)[: B * most].to(torch.int32).view(B, most)
    there = torch.arange(most, device=DEV) < held.view(-1, 1)
    s["n_pages"], s["max_pages"] = n_pages, most
    s["table"] = torch.where(there, ids, torch.full_like(ids, -1)).contiguous()
    s["refs"] = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    s["refs"][s["table"][there].long()] = 1
    s["len"] = length.to(torch.int32)
    s["free_bits"] = _free_bits(s["refs"])


def _free_bits(refs):
    n = refs.numel()
    free = torch.zeros((n + 31) // 32 * 32, dtype=torch.int64, device=refs.device)
    free[:n] = (refs == 0).long()
    w = (free.view(-1, 32) << torch.arange(32, device=refs.device)).sum(-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)


def _pool(g, planes, n_pages, s):
    """Pages full of codes, with scales and offsets as keys and values of unit size have them."""
    size = _page_bytes(s["kv_heads"], s["d"], s["page_tokens"])
    pool = torch.randint(-2 ** 31, 2 ** 31, (planes, n_pages, size // 4), generator=g, device=DEV, dtype=torch.int64).to(torch.int32).view(torch.uint8)
    n = planes * n_pages * (size // (UNIT * s["d"] // 2 + UNIT * 4))
    scale = (torch.rand((n, UNIT), generator=g, device=DEV) * 0.2 + 0.25).to(torch.bfloat16)
    offset = (scale.float() * (-7.5 + _normal(g, (n, UNIT)))).to(torch.bfloat16)
    params = torch.stack([scale, offset], -1).reshape(n, 2 * UNIT).view(torch.uint8)
    pool.view(n, -1)[:, UNIT * s["d"] // 2:] = params
    return pool


def _counts(case):
    """Rows of a batch's sequences, from half of the most to the most (the seed says whose are which)."""
    B, most = case["B"], case["most"]
    return [most - b * 7 % (most - most // 2 + (most > 1)) for b in range(B)]


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case)
    kind = case["kind"]
    if kind in ("rotate", "prompt"):
        if kind == "prompt":
            s["spans"] = [int(n) for n in case["lens"].split(",")]
            s["rows_at"] = _starts(torch.tensor(s["spans"], device=DEV))
            s["rows"] = sum(s["spans"])
        H, K, d, n = case["heads"], case["kv_heads"], case["d"], s["rows"]
        # the rows of one fused projection: queries, keys, values
        s["qkv"] = _normal(g, (n, H + 2 * K, d)).to(torch.bfloat16)
        s["q"], s["k"], s["v"] = s["qkv"].split([H, K, K], 1)
        if kind == "rotate":
            s["positions"] = _ints(g, 0, case["far"], (n,))
            r = case["rotary"] // 2
            s["frequencies"] = (500000.0 ** -(torch.arange(r, device=DEV).double() / r)).float()
            s["q_weight"] = (1 + 0.2 * _normal(g, (d,))).to(torch.bfloat16) if case["norm"] else None
            s["k_weight"] = (1 + 0.2 * _normal(g, (d,))).to(torch.bfloat16) if case["norm"] else None
            s["q_out"] = torch.empty((n, H, d), dtype=torch.bfloat16, device=DEV)
            s["k_out"] = torch.empty((n, K, d), dtype=torch.bfloat16, device=DEV)
        else:
            s["q"] *= 2
            s["out"] = torch.empty((n, H, d), dtype=torch.bfloat16, device=DEV)
            s["lse"] = torch.empty((n, H), dtype=torch.float32, device=DEV)
        return s
    if kind == "evict":
        B, T = case["B"], case["len"]
        length = T - _ints(g, 0, max(1, T // 20), (B,))
        _tables(g, s, length, T)
        s["pool"] = _pool(g, case["planes"], s["n_pages"], s)
        s["budget"] = torch.full((B,), max(case["budget"], case["first"] + case["recent"] + 1), dtype=torch.int32, device=DEV)
        # few tokens have most of the weight
        s["weights"] = torch.rand((B, s["max_pages"] * case["page_tokens"]), generator=g, device=DEV).clamp(min=1e-6).pow(-0.7)
        s["before"] = {k: s[k].clone() for k in ("table", "len", "refs", "free_bits", "weights")}
        return s
    B, most = case["B"], case["most"]
    counts = torch.tensor(_counts(case), dtype=torch.int32, device=DEV)[torch.randperm(B, generator=g, device=DEV)]
    s["base"] = (torch.rand(B, generator=g, device=DEV) * case["len"] * 0.5 + case["len"] * 0.5).to(torch.int32)
    if kind == "attend" and case["most"] == 1 and B > 1:        # lengths far apart
        s["base"] = (case["len"] * 100.0 ** -torch.rand(B, generator=g, device=DEV)).to(torch.int32)
    s["rows_at"] = _starts(counts)
    s["rows"] = sum(_counts(case))
    _tables(g, s, s["base"] + counts, case["len"] + most)
    s["pool"] = _pool(g, 2, s["n_pages"], s)
    K, d, n = case["kv_heads"], case["d"], s["rows"]
    if kind == "append":
        s["qkv"] = _normal(g, (n, 6 * K, d)).to(torch.bfloat16)
        _, s["k"], s["v"] = s["qkv"].split([4 * K, K, K], 1)
        s["k_held"] = torch.empty((n, K, d), dtype=torch.bfloat16, device=DEV)
        s["v_held"] = torch.empty((n, K, d), dtype=torch.bfloat16, device=DEV)
    else:
        H = case["heads"]
        s["q"] = (_normal(g, (n, H, d)) * 2).to(torch.bfloat16)
        s["out"] = torch.empty((n, H, d), dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.empty((n, H), dtype=torch.float32, device=DEV)
        if case["weigh"]:
            s["weights"] = torch.rand((B, s["max_pages"] * case["page_tokens"]), generator=g, device=DEV)
    return s


# ------------------------------------------------------------------ plain forms
def _plain_rotate_one(x, weight, s):
    r = s["rotary"]
    y = x.float()
    if weight is not None:
        y = y / (y.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * weight.float()
    angle = s["positions"].double().view(-1, 1, 1) * s["frequencies"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    rot, rest = y[..., :r], y[..., r:]
    a, b = (rot[..., 0::2], rot[..., 1::2]) if s["interleaved"] else (rot[..., : r // 2], rot[..., r // 2:])
    a, b = a * cos - b * sin, a * sin + b * cos
    rot = torch.stack([a, b], -1).flatten(-2) if s["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([rot, rest], -1).to(x.dtype)


def _plain_rotate(s):
    return {"q": _plain_rotate_one(s["q"], s["q_weight"], s), "k": _plain_rotate_one(s["k"], s["k_weight"], s)}


def _plain_softmax(z, seen):
    z = z.masked_fill(~seen, float("-inf"))
    top = z.amax(-1, keepdim=True)
    p = (z - top).exp()
    total = p.sum(-1, keepdim=True)
    return p / total, (top + total.log()).squeeze(-1)


def _plain_prompt(s):
    H, K, d = s["heads"], s["kv_heads"], s["d"]
    out, lse, at = [], [], 0
    for n in s["spans"]:
        q, k, v = (s[x][at:at + n].float() for x in "qkv")
        at += n
        z = torch.einsum("ikgd,jkd->kgij", q.view(n, K, H // K, d), k) * d ** -0.5
        p, l = _plain_softmax(z, torch.ones((n, n), dtype=torch.bool, device=DEV).tril())
        out.append(torch.einsum("kgij,jkd->ikgd", p, v).reshape(n, H, d))
        lse.append(l.permute(2, 0, 1).reshape(n, H))
    return {"out": torch.cat(out).to(s["q"].dtype), "lse": torch.cat(lse)}


def _places(s):
    """For every row: its sequence, its slot in that sequence's cache."""
    row = torch.arange(s["rows"], device=DEV)
    seq = torch.searchsorted(s["rows_at"][1:].long(), row, right=True)
    return seq, s["base"].long()[seq] + row - s["rows_at"].long()[seq]


def _unit_views(plane, s):
    """One plane of a pool: its words [pages, kv_heads, units, 8, D/8] by token, and its pairs [pages, kv_heads, units, 8, 2], as views."""
    return plane.view(plane.shape[0], s["kv_heads"], s["page_tokens"] // UNIT, -1).split([UNIT * s["d"] // 2, UNIT * 4], -1)


def _word_order(s, values):
    """Where word w of token r of a unit lies: [8, D/8]."""
    n = s["d"] // 8
    if not values:
        return torch.arange(UNIT * n, device=DEV).view(UNIT, n)
    at = torch.arange(UNIT * n, device=DEV).view(8, 4, 2, n // 8)           # g, t, o, h
    return at.permute(1, 2, 3, 0).reshape(UNIT, n)


NIBBLE = [0, 4, 1, 5, 2, 6, 3, 7]           # the four bits, counted from bit 0, that hold code e of eight


def _plain_read(plane, pages, values, s):
    """The values that `pages` [...] of a plane stand for: [..., page_tokens, kv_heads, D]."""
    codes, params = _unit_views(plane[pages.flatten()], s)
    words = codes.contiguous().view(torch.int32)[..., _word_order(s, values)]
    shifts = torch.tensor([4 * p for p in NIBBLE], dtype=torch.int32, device=DEV)
    code = ((words.unsqueeze(-1) >> shifts) & 15).flatten(-2).float()
    pair = params.contiguous().view(torch.bfloat16).float().unflatten(-1, (UNIT, 2))
    x = pair[..., :1] * code + pair[..., 1:]
    return x.flatten(2, 3).transpose(1, 2).reshape(*pages.shape, s["page_tokens"], s["kv_heads"], s["d"])


def _plain_append_one(plane, x, held, values, s):
    x = x.float()
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    down = low.to(torch.bfloat16)
    down = torch.where(down.float() > low, torch.nextafter(down, torch.full_like(down, float("-inf"))), down)
    step = (high - down.float()) / torch.full_like(high, 15.0)
    up = step.to(torch.bfloat16)
    up = torch.where(up.float() < step, torch.nextafter(up, torch.full_like(up, float("inf"))), up)
    up = torch.where(up == 0, torch.ones_like(up), up)
    code = ((x - down.float()) / up.float()).round().clamp(0, 15).to(torch.int64)
    word = (code.unflatten(-1, (-1, 8)) << torch.tensor([4 * p for p in NIBBLE], device=DEV)).sum(-1)
    word = torch.where(word >= 2 ** 31, word - 2 ** 32, word).to(torch.int32)
    seq, slot = _places(s)
    P, n = s["page_tokens"], s["d"] // 8
    page = s["table"][seq, slot // P].long().view(-1, 1, 1)
    head = torch.arange(s["kv_heads"], device=DEV).view(1, -1, 1)
    at = slot % P
    # in 32-bit words: units of 8 D/8 + 8
    unit = ((page * s["kv_heads"] + head) * (P // UNIT) + (at // UNIT).view(-1, 1, 1)) * (UNIT * n + UNIT)
    flat = plane.view(torch.int32).view(-1)
    flat[unit + _word_order(s, values)[at % UNIT].unsqueeze(1)] = word
    flat[(unit + UNIT * n + (at % UNIT).view(-1, 1, 1)).squeeze(-1)] = torch.cat([up, down], -1).view(torch.int32).squeeze(-1)
    held.copy_(up.float() * code.float() + down.float())


def _plain_append(s):
    _plain_append_one(s["pool"][0], s["k"], s["k_held"], False, s)
    _plain_append_one(s["pool"][1], s["v"], s["v_held"], True, s)
    return {"pool": s["pool"], "k_held": s["k_held"], "v_held": s["v_held"]}


def _plain_attend(s):
    B, H, K, d, n = s["B"], s["heads"], s["kv_heads"], s["d"], s["most"]
    pages = s["table"].clamp(min=0).long()
    k = _plain_read(s["pool"][0], pages, False, s).flatten(1, 2)
    v = _plain_read(s["pool"][1], pages, True, s).flatten(1, 2)
    seq, slot = _places(s)
    i = torch.arange(s["rows"], device=DEV) - s["rows_at"].long()[seq]
    q = torch.zeros((B, n, K, H // K, d), device=DEV)
    q[seq, i] = s["q"].float().view(-1, K, H // K, d)
    z = torch.einsum("bikgd,bjkd->bkgij", q, k) * d ** -0.5
    at = torch.arange(k.shape[1], device=DEV)
    there = torch.zeros((B, n), dtype=torch.bool, device=DEV)
    there[seq, i] = True
    # rows that a sequence does not have see its first token only and are left out below
    seen = at <= torch.where(there, s["base"].view(-1, 1) + torch.arange(n, device=DEV), 0).unsqueeze(-1)
    p, lse = _plain_softmax(z, seen.view(B, 1, 1, n, -1))
    s["out"].copy_(torch.einsum("bkgij,bjkd->bikgd", p, v).reshape(B, n, H, d)[seq, i])
    s["lse"].copy_(lse.permute(0, 3, 1, 2).reshape(B, n, H)[seq, i])
    r = {"out": s["out"], "lse": s["lse"]}
    if s["weigh"]:
        more = (p * there.view(B, 1, 1, n, 1)).sum((1, 2, 3))
        s["weights"].copy_(torch.where(at < s["len"].view(-1, 1), s["weights"] * 0.9 + more, s["weights"]))
        r["weights"] = s["weights"]
    return r


def _plain_evict(s):
    for name, x in s["before"].items():         # the caches, as the prompts left them
        s[name].copy_(x)
    B, P, T = s["B"], s["page_tokens"], s["weights"].shape[1]
    length, budget = s["len"].long().view(-1, 1), s["budget"].long().view(-1, 1)
    at = torch.arange(T, device=DEV).view(1, -1)
    must = (at < s["first"]) | (at >= length - s["recent"])
    rank = torch.where(must, float("inf"), s["weights"]).masked_fill(at >= length, float("-inf"))
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices
    keep = torch.zeros((B, T), dtype=torch.bool, device=DEV).scatter_(1, order, at < budget) & (at < length)
    keep |= (length <= budget) & (at < length)
    kept = keep.sum(1, keepdim=True)
    seq, old = keep.nonzero(as_tuple=True)                  # by sequence, then by slot
    new = (keep.cumsum(1) - 1)[seq, old]
    s["weights"][seq, new] = s["before"]["weights"][seq, old]
    # tokens as they lie in a page: words of codes and the pair, for every plane and head
    n, K = s["d"] // 8, s["kv_heads"]
    flat = s["pool"].view(torch.int32).view(s["planes"] // 2, 2, -1)

    def where(slot, values):
        page = s["before"]["table"][seq, slot // P].long().view(-1, 1, 1)
        place = slot % P
        unit = ((page * K + torch.arange(K, device=DEV).view(1, -1, 1)) * (P // UNIT) + (place // UNIT).view(-1, 1, 1)) * (UNIT * n + UNIT)
        order = torch.cat([_word_order(s, values), UNIT * n + torch.arange(UNIT, device=DEV).view(-1, 1)], 1)
        return unit + order[place % UNIT].unsqueeze(1)

    moved = new < old
    seq, old, new = seq[moved], old[moved], new[moved]
    flat[:, 0, where(new, False)] = flat[:, 0, where(old, False)]
    flat[:, 1, where(new, True)] = flat[:, 1, where(old, True)]
    cols = torch.arange(s["max_pages"], device=DEV)
    drop = (cols >= (kept + P - 1) // P) & (cols < (length + P - 1) // P)
    s["refs"].index_add_(0, torch.where(drop, s["table"], 0).flatten().long(), -drop.flatten().to(torch.int32))
    s["table"].masked_fill_(drop, -1)
    s["len"].copy_(kept.view(-1))
    s["free_bits"].copy_(_free_bits(s["refs"]))
    return _evicted(s)


def _evicted(s):
    return {k: s[k] for k in ("table", "len", "refs", "free_bits", "weights", "pool")}


PLAIN = {"rotate": _plain_rotate, "prompt": _plain_prompt, "append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}


# ------------------------------------------------------------------ the package's calls
def _own_rotate(s):
    from paper_2510_26527_b200 import binding
    q, k = binding.polyspec_rotate_heads(s["q"], s["k"], s["positions"], s["frequencies"], s["q_weight"], s["k_weight"], interleaved=s["interleaved"],
                                         q_out=s["q_out"], k_out=s["k_out"])
    return {"q": q, "k": k}


def _own_prompt(s):
    from paper_2510_26527_b200 import binding
    out, lse, _ = binding.polyspec_prompt_attention(s["q"], s["k"], s["v"], s["rows_at"], out=s["out"], lse=s["lse"])
    return {"out": out, "lse": lse}


def _own_pages(s):
    """The package, and the page tables' handle, which a program makes once."""
    from paper_2510_26527_b200 import binding
    if "pages" not in s:
        s["pages"] = binding.CachePages(s["table"], s["len"], s["refs"], s["free_bits"], s["page_tokens"])
    return binding, s["pages"]


def _own_append(s):
    binding, pages = _own_pages(s)
    binding.polyspec_cache_append(pages, s["k"], s["v"], s["pool"], s["rows_at"], s["base"], k_held=s["k_held"], v_held=s["v_held"])
    return {"pool": s["pool"], "k_held": s["k_held"], "v_held": s["v_held"]}


def _own_attend(s):
    binding, pages = _own_pages(s)
    binding.polyspec_cache_attention(pages, s["q"], s["pool"], s["kv_heads"], s["rows_at"], s["base"], out=s["out"], lse=s["lse"])
    r = {"out": s["out"], "lse": s["lse"]}
    if s["weigh"]:
        binding.polyspec_cache_weigh(pages, s["q"], s["pool"], s["kv_heads"], s["rows_at"], s["base"], s["lse"], s["weights"], keep=0.9)
        r["weights"] = s["weights"]
    return r


def _own_evict(s):
    binding, pages = _own_pages(s)
    for name, x in s["before"].items():         # the caches, as the prompts left them
        s[name].copy_(x)
    binding.polyspec_cache_evict(pages, s["budget"], s["weights"], s["pool"], s["kv_heads"], s["d"], first=s["first"], recent=s["recent"])
    return _evicted(s)


OWN = {"rotate": _own_rotate, "prompt": _own_prompt, "append": _own_append, "attend": _own_attend, "evict": _own_evict}


def run(state):
    return (OWN if own else PLAIN)[state["kind"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind, K, d = case["kind"], case["kv_heads"], case["d"]
    token = K * (d + 8)                 # bytes of a token's keys and values in a layer's pages
    if kind == "rotate":
        size = case["rows"] * (case["heads"] + K) * d
        return {"bytes": 4 * size + case["rows"] * 4, "flops": 8 * size}
    if kind == "prompt":
        lens = [int(n) for n in case["lens"].split(",")]
        pairs = sum(n * (n + 1) // 2 for n in lens)
        return {"bytes": sum(lens) * (4 * case["heads"] * d + 4 * K * d + 4 * case["heads"]), "flops": 4 * pairs * case["heads"] * d}
    B = case["B"]
    if kind == "evict":
        kept = min(case["budget"], case["len"])
        # the first token to go is among the first few; all kept tokens behind it move
        moved = B * max(0, kept - case["first"]) if kept < case["len"] * 0.975 else B * kept // 2
        return {"bytes": moved * token // 2 * case["planes"] * 2 + B * case["len"] * 8, "flops": 0}
    rows = sum(_counts(case))
    if kind == "append":
        return {"bytes": rows * (token + 8 * K * d), "flops": 12 * rows * K * d}
    mean = case["len"] * (0.75 if case["most"] > 1 or B == 1 else 0.215) + 1
    size = 2 * rows * case["heads"] * d * 2 + rows * case["heads"] * 4
    if case["weigh"]:
        size += int(B * mean * 8)
    return {"bytes": int(B * mean * token) + size, "flops": int(4 * rows * mean * case["heads"] * d * (1.5 if case["weigh"] else 1))}


# ------------------------------------------------------------------ 64-bit references, from the definitions
def _exact_rotate(x, weight, s):
    y = x.double()
    if weight is not None:
        y = y * torch.rsqrt((y * y).sum(-1, keepdim=True) / y.shape[-1] + 1e-6) * weight.double()
    r = s["rotary"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["positions"].double()[:, None, None] * s["frequencies"].double())
    z = y[..., :r]
    if s["interleaved"]:
        y[..., :r] = torch.view_as_real(torch.view_as_complex(z.reshape(*z.shape[:-1], r // 2, 2)) * turn).flatten(-2)
    else:
        z = torch.complex(z[..., : r // 2], z[..., r // 2:]) * turn
        y[..., :r] = torch.cat([z.real, z.imag], -1)
    return y


def _exact_values(bytes_, d, values):
    """Units [..., 4 D + 32] bytes -> [..., 8, D] values, byte by byte."""
    body, tail = bytes_[..., : 4 * d], bytes_[..., 4 * d:]
    word = torch.arange(UNIT * d // 8, device=DEV)
    if values:
        h, o, t, g = word % (d // 64), word // (d // 64) % 2, word // (d // 32) % 4, word // (d // 8)
        token, part = 2 * t + o, 8 * h + g
    else:
        token, part = word // (d // 8), word % (d // 8)
    x = torch.empty((*body.shape[:-1], UNIT, d), dtype=torch.float64, device=DEV)
    for b, pair in enumerate(((0, 2), (4, 6), (1, 3), (5, 7))):            # the codes of a word's byte b
        byte = body[..., b::4]
        x[..., token, 8 * part + pair[0]] = (byte % 16).double()
        x[..., token, 8 * part + pair[1]] = (byte // 16).double()
    both = tail.contiguous().view(torch.bfloat16).double()
    return x * both[..., 0::2, None] + both[..., 1::2, None]


def exact(case, seed):
    kind = case["kind"]
    if kind == "evict":
        return None         # selected and moved data: nothing is computed
    s = prepare(case, seed)
    if kind == "rotate":
        return {"q": _exact_rotate(s["q"], s["q_weight"], s), "k": _exact_rotate(s["k"], s["k_weight"], s)}
    K, d = case["kv_heads"], case["d"]
    if kind == "append":        # the pages' bytes are whole numbers; a held value is the level next to the row's
        r = {"pool": None}
        for name in ("k", "v"):
            x = s[name].double()
            lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)

            def grid(y, towards):       # the bf16 number next to y on one side; powers of two from their bits
                e = torch.floor(torch.log2(y.abs().clamp(min=1e-30))).long() - 7
                return towards(y * ((1023 - e) << 52).view(torch.float64)) * ((1023 + e) << 52).view(torch.float64)
            lo = grid(lo, torch.floor)
            step = grid(((hi - lo).float() / torch.full_like(lo, 15.0).float()).double(), torch.ceil)
            r[name + "_held"] = lo + step * torch.round((x - lo) / step)
        return r
    H = case["heads"]
    out = torch.zeros((s["rows"], H, d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((s["rows"], H), dtype=torch.float64, device=DEV)
    if kind == "prompt":
        at = 0
        for n in s["spans"]:
            for h in range(H):
                q, k, v = s["q"][at:at + n, h].double(), s["k"][at:at + n, h // (H // K)].double(), s["v"][at:at + n, h // (H // K)].double()
                z = (q @ k.t() / d ** 0.5).masked_fill_(torch.triu(torch.ones((n, n), dtype=torch.bool, device=DEV), 1), float("-inf"))
                lse[at:at + n, h] = torch.logsumexp(z, -1)
                out[at:at + n, h] = torch.exp(z - lse[at:at + n, h].view(-1, 1)) @ v
            at += n
        return {"out": out, "lse": lse}
    weights = s["weights"].double() if case["weigh"] else None
    P = case["page_tokens"]
    for b in range(case["B"]):
        n = int(s["len"][b])
        ids = s["table"][b, : (n + P - 1) // P].long()
        lo, hi = int(s["rows_at"][b]), int(s["rows_at"][b + 1])
        first = int(s["base"][b])
        if case["weigh"]:
            weights[b, :n] *= 0.9
        for h in range(K):
            k, v = (_exact_values(s["pool"][p, ids].view(ids.numel(), K, P // UNIT, -1)[:, h], d, p == 1).reshape(-1, d)[:n] for p in (0, 1))
            for i in range(lo, hi):
                m = first + i - lo + 1
                heads = slice(h * (H // K), (h + 1) * (H // K))
                z = s["q"][i, heads].double() @ k[:m].t() / d ** 0.5
                lse[i, heads] = torch.logsumexp(z, -1)
                p = torch.exp(z - lse[i, heads].view(-1, 1))
                out[i, heads] = p @ v[:m]
                if case["weigh"]:
                    weights[b, :m] += p.sum(0)
    r = {"out": out, "lse": lse}
    if case["weigh"]:
        r["weights"] = weights
    return r
