"""Workloads of the operators that stand around the verification step, for measurement against their plain forms.

Three kinds, in the order in which a decode cycle of a staged chain meets them:

  head    the LM head of a 4-bit (group-scaled) verifier: hidden states -> logits of every block position
  logits  a request's sampling controls on the logits rows of a block: penalties for repeated tokens, biases, masks
  pages   the page tables of the models' caches around a verified block: reserve, roll back, fork, compact

Where ``own`` is false everything is computed with elementary torch operations; where it is true, with the package's calls.
"""
import torch

own = False

DEV = "cuda"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one decode step of a single sequence through a 4-bit LM head (vocabulary and width of the fused configuration)
        {"name": "head_one_token", "kind": "head", "rows": 1, "V": 32000, "d": 4096, "group": 128, "zeros": True, "out": "f32"},
        # one sequence's verification block: k = 8 drafted tokens and the bonus row
        {"name": "head_block", "kind": "head", "rows": 9, "V": 32000, "d": 4096, "group": 128, "zeros": True, "out": "f32"},
        # a slice of a vocabulary that divides by nothing, small groups, symmetric codes, two short blocks of a batch
        {"name": "head_odd", "kind": "head", "rows": 37, "V": 12807, "d": 2080, "group": 32, "zeros": False, "out": "bf16"},
        # the fused configuration's batch: 32 sequences x 9 rows
        {"name": "head_batch", "kind": "head", "rows": 288, "V": 32000, "d": 4096, "group": 128, "zeros": True, "out": "f32"},
        # the widest vocabulary of the configurations over a wide model, one sequence's short block (k = 4)
        {"name": "head_wide", "kind": "head", "rows": 5, "V": 152064, "d": 8192, "group": 64, "zeros": True, "out": "bf16"},
        # one sequence with penalties and a few biases
        {"name": "controls_single", "kind": "controls", "B": 1, "rows": 9, "V": 32000, "dt": "f32", "history": 700, "bias": 16, "mask": False},
        # the three-model configuration's batch with long texts
        {"name": "controls_batch", "kind": "controls", "B": 64, "rows": 7, "V": 128256, "dt": "bf16", "history": 4096, "bias": 32, "mask": False},
        # the four-model configuration's batch, everything at once: penalties, biases, grammar masks
        {"name": "controls_full", "kind": "controls", "B": 256, "rows": 5, "V": 152064, "dt": "bf16", "history": 1024, "bias": 64, "mask": True},
        # structured output: grammar masks alone, laid over the logits where they stand
        {"name": "grammar_in_place", "kind": "grammar", "B": 64, "rows": 7, "V": 128256, "dt": "bf16"},
        # one cycle's bookkeeping: room for a block of every sequence, then back to what was accepted
        {"name": "pages_cycle", "kind": "cycle", "B": 64, "max_pages": 640, "n_pages": 41500, "page_tokens": 16, "block": 9},
        # parallel sampling: eight continuations of each of sixteen prompts, their last pages copied before the first write
        {"name": "pages_fork", "kind": "fork", "parents": 16, "children": 8, "tokens": 1000, "page_tokens": 16, "n_pages": 2048, "planes": 64,
         "page_bytes": 16384, "block": 9},
        # a pool left full of holes by finished sequences, moved together
        {"name": "pages_compact", "kind": "compact", "B": 48, "max_pages": 64, "n_pages": 4000, "page_tokens": 32, "planes": 48, "page_bytes": 8192},
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["head", "head", "controls", "grammar", "cycle", "fork", "compact"])
    if kind == "head":
        group = rng.choice([32, 64, 128, 128])
        d = max(1, _log(rng, 256, 8192) // group) * group
        rows = _log(rng, 1, 300)
        V = min(_log(rng, 1000, 152064), 288 * 32000 * 4096 // (rows * d))
        return {"kind": kind, "rows": rows, "V": V, "d": d, "group": group, "zeros": rng.random() < 0.7, "out": rng.choice(["f32", "bf16"])}
    if kind in ("controls", "grammar"):
        V = _log(rng, 125, 19008) * 8
        rows = rng.randint(1, 12)
        B = max(1, min(_log(rng, 1, 256), 256 * 5 * 152064 // (rows * V)))
        case = {"kind": kind, "B": B, "rows": rows, "V": V, "dt": rng.choice(["f32", "bf16"])}
        if case["dt"] == "f32":
            case["B"] = max(1, B // 2)
        if kind == "controls":
            case.update(history=_log(rng, 1, 8192), bias=rng.choice([0, 3, 40, 300]), mask=rng.random() < 0.5)
        return case
    if kind == "cycle":
        B, pages = _log(rng, 1, 512), _log(rng, 4, 640)
        return {"kind": kind, "B": B, "max_pages": pages, "n_pages": B * pages + rng.randint(0, 1000), "page_tokens": rng.choice([8, 16, 32, 48, 64]),
                "block": rng.randint(1, 33)}
    if kind == "fork":
        parents, children, P = rng.randint(1, 16), rng.randint(1, 8), rng.choice([8, 16, 32])
        tokens, block = _log(rng, 20, 1000), rng.randint(1, 12)
        used = parents * (tokens // P + 1) + parents * children * (2 + block // P)
        return {"kind": kind, "parents": parents, "children": children, "tokens": tokens, "page_tokens": P, "n_pages": used + rng.randint(0, 99),
                "planes": rng.randint(2, 64), "page_bytes": 512 * rng.randint(1, 32), "block": block}
    B, pages = rng.randint(2, 48), _log(rng, 4, 64)
    return {"kind": kind, "B": B, "max_pages": pages, "n_pages": B * pages + rng.randint(0, 900), "page_tokens": rng.choice([16, 32, 64]),
            "planes": rng.randint(2, 48), "page_bytes": 512 * rng.randint(1, 16)}


# ------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _ints(g, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=g, device=DEV, dtype=torch.int32)


def _uniform(g, lo, hi, shape):
    return torch.rand(shape, generator=g, device=DEV) * (hi - lo) + lo


def _tokens(g, V, shape):
    """Token ids with the skew of text: a few of them often, most rarely."""
    return (torch.rand(shape, generator=g, device=DEV).pow(4) * V).to(torch.int32).clamp_(max=V - 1)


def _grammar(g, B, rows, V):
    """Allowed-token bits: every other row tight (some forty tokens allowed), the others loose (one in sixteen forbidden)."""
    W = (V + 31) // 32
    bits = torch.zeros((B, rows, W), dtype=torch.int32, device=DEV)
    for _ in range(4):
        bits |= torch.randint(-2 ** 31, 2 ** 31, (B, rows, W), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    tight = torch.zeros((B, rows, W * 32), dtype=torch.int64, device=DEV)
    tight.scatter_(2, _ints(g, 0, V, (B, rows, 40)).long(), 1)
    sparse = _words(tight.view(B, rows, W, 32))
    some = (torch.arange(B * rows, device=DEV).view(B, rows, 1) + int(_ints(g, 0, 2, (1,)))) % 2 == 0
    return torch.where(some, sparse, bits).contiguous()


def _words(bits):
    """[..., 32] zeros and ones -> [...] int32, bit i from entry i."""
    w = (bits.long() << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)


def _page_state(table, length, refs, page_tokens):
    return {"table": table, "len": length, "refs": refs, "free_bits": _free_bits(refs), "page_tokens": page_tokens}


def _free_bits(refs):
    n = refs.numel()
    free = torch.zeros((n + 31) // 32 * 32, dtype=torch.int64, device=refs.device)
    free[:n] = (refs == 0).long()
    return _words(free.view(-1, 32))


def _filled(g, held, max_pages, n_pages):
    """A table of sequences holding `held` [B] pages each, ids scattered over the pool, and the references they make."""
    B = held.numel()
    ids = torch.randperm(n_pages, generator=g, device=DEV)[: B * max_pages].to(torch.int32).view(B, max_pages)
    there = torch.arange(max_pages, device=DEV) < held.view(-1, 1)
    table = torch.where(there, ids, torch.full_like(ids, -1)).contiguous()
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[table[there].long()] = 1
    return table, refs


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case)
    kind = case["kind"]
    if kind == "head":
        rows, V, d, group = case["rows"], case["V"], case["d"], case["group"]
        s["hidden"] = torch.randn((rows, d), generator=g, device=DEV).to(torch.bfloat16)
        s["qweight"] = torch.randint(-2 ** 31, 2 ** 31, (V, d // 8), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
        s["scales"] = _uniform(g, 0.002, 0.02, (V, d // group)).to(torch.bfloat16)
        s["zero_points"] = _ints(g, 5, 11, (V, d // group)).to(torch.uint8) if case["zeros"] else None
        s["logits"] = torch.empty((rows, V), dtype=DT[case["out"]], device=DEV)
    elif kind in ("controls", "grammar"):
        B, rows, V = case["B"], case["rows"], case["V"]
        s["logits"] = (torch.randn((B, rows, V), generator=g, device=DEV) * 3).to(DT[case["dt"]])
        s["bits"] = _grammar(g, B, rows, V) if case.get("mask", True) else None
        if kind == "controls":
            H, n = case["history"], case["bias"]
            s["draft_tokens"] = _tokens(g, V, (B, max(1, rows - 1)))
            s["tokens"] = _tokens(g, V, (B, H))
            s["history_len"] = _ints(g, H // 2, H + 1, (B,))
            s["prompt_len"] = (s["history_len"].float() * torch.rand(B, generator=g, device=DEV)).to(torch.int32)
            s["repetition"] = _uniform(g, 1.0, 1.3, (B,))
            s["frequency"] = _uniform(g, 0.0, 0.5, (B,))
            s["presence"] = _uniform(g, 0.0, 1.0, (B,))
            s["bias_tokens"] = _tokens(g, V, (B, n)) if n else None
            s["bias_values"] = _uniform(g, -6.0, 6.0, (B, n)) if n else None
            s["out"] = torch.empty_like(s["logits"])
    elif kind == "cycle":
        B, P, most = case["B"], case["page_tokens"], case["max_pages"]
        room = most * P - case["block"]
        length = (_uniform(g, 0.5, 1.0, (B,)) * max(room, 0)).to(torch.int32)
        table, refs = _filled(g, (length + P - 1) // P, most, case["n_pages"])
        s.update(_page_state(table, length, refs, P))
        s["committed"] = length.clone()
        s["accepted"] = _ints(g, 0, case["block"] + 1, (B,))
    elif kind == "fork":
        P, n, c = case["page_tokens"], case["parents"], case["children"]
        length = torch.zeros(n * (1 + c), dtype=torch.int32, device=DEV)
        length[:n] = (_uniform(g, 0.5, 1.0, (n,)) * case["tokens"]).to(torch.int32)
        most = (case["tokens"] + case["block"]) // P + 2
        held = (length[:n] + P - 1) // P
        table, refs = _filled(g, held, case["tokens"] // P + 1, case["n_pages"])
        whole = torch.full((n * (1 + c), most), -1, dtype=torch.int32, device=DEV)
        whole[:n, : table.shape[1]] = table
        s.update(_page_state(whole, length, refs, P))
        s["src"] = torch.arange(n, device=DEV, dtype=torch.int32).repeat_interleave(c)
        s["dst"] = torch.arange(n, n * (1 + c), device=DEV, dtype=torch.int32)
        s["back_to"] = length.clone()
        base = torch.full((n * (1 + c),), -case["block"], dtype=torch.int32, device=DEV)
        base[n:] = length[:n].repeat_interleave(c)
        s["base"] = base
    elif kind == "compact":
        B, P, most = case["B"], case["page_tokens"], case["max_pages"]
        held = _ints(g, 0, most + 1, (B,))
        length = (held * P - _ints(g, 0, P, (B,))).clamp_(min=0)
        table, refs = _filled(g, (length + P - 1) // P, most, case["n_pages"])
        s.update(_page_state(table, length, refs, P))
        s["before"] = {k: s[k].clone() for k in ("table", "refs", "free_bits")}
    if "planes" in case:
        n = case["planes"] * case["n_pages"] * case["page_bytes"] // 2
        s["pool"] = torch.randn(n, generator=g, device=DEV, dtype=torch.bfloat16).view(case["planes"], case["n_pages"], case["page_bytes"] // 2)
    return s


# ------------------------------------------------------------------ plain forms
def _plain_head(s):
    q, group = s["qweight"], s["group"]
    V, d = s["V"], s["d"]
    # weight 8 i + e of a row is the nibble at bit 4 (e / 2) + 16 (e mod 2) of its word i
    shifts = torch.tensor([4 * (e // 2) + 16 * (e % 2) for e in range(8)], dtype=torch.int32, device=q.device)
    codes = ((q.unsqueeze(-1) >> shifts) & 15).view(V, d // group, group).float()
    zero = 8.0 if s["zero_points"] is None else s["zero_points"].float().unsqueeze(-1)
    weight = ((codes - zero) * s["scales"].float().unsqueeze(-1)).view(V, d)
    return {"logits": (s["hidden"].float() @ weight.t()).to(s["logits"].dtype)}


def _allowed(bits, V):
    flags = (bits.unsqueeze(-1) >> torch.arange(32, device=bits.device, dtype=torch.int32)) & 1
    return flags.flatten(-2)[..., :V].bool()


def _plain_controls(s):
    B, rows, V = s["B"], s["rows"], s["V"]
    at = torch.arange(s["tokens"].shape[1], device=DEV)
    live = at < s["history_len"].view(B, 1)
    said = live & (at >= s["prompt_len"].view(B, 1))
    tokens = s["tokens"].long()
    seen = torch.zeros((B, V), device=DEV).scatter_add_(1, tokens, live.float()).unsqueeze(1)
    count = torch.zeros((B, V), device=DEV).scatter_add_(1, tokens, said.float())
    # row j has the drafted tokens before it in its context
    count = count.unsqueeze(1).expand(B, rows, V).contiguous()
    draft = s["draft_tokens"].long()
    before = (torch.arange(draft.shape[1], device=DEV) < torch.arange(rows, device=DEV).view(rows, 1)).float()
    count.scatter_add_(2, draft.unsqueeze(1).expand(B, rows, -1), before.expand(B, rows, -1).contiguous())
    z = s["logits"].float()
    r = s["repetition"].view(B, 1, 1)
    z = torch.where((seen > 0) | (count > 0), torch.where(z > 0, z / r, z * r), z)
    z = z - s["frequency"].view(B, 1, 1) * count - s["presence"].view(B, 1, 1) * (count > 0).float()
    if s["bias_tokens"] is not None:
        z = z + torch.zeros((B, V), device=DEV).scatter_add_(1, s["bias_tokens"].long(), s["bias_values"]).unsqueeze(1)
    if s["bits"] is not None:
        z = z.masked_fill(~_allowed(s["bits"], V), float("-inf"))
    return {"logits": z.to(s["logits"].dtype)}


def _plain_grammar(s):
    return {"logits": s["logits"].masked_fill(~_allowed(s["bits"], s["V"]), float("-inf"))}


def _pages_of(tokens, P):
    return (tokens + P - 1) // P


def _plain_rollback(p, to, P):
    """Sequences fall back to `to` tokens (never up); pages wholly behind the new end are given back."""
    table, length, refs = p
    cols = torch.arange(table.shape[1], device=DEV)
    back = (to >= 0) & (to < length)
    drop = back.view(-1, 1) & (cols >= _pages_of(to, P).view(-1, 1)) & (cols < _pages_of(length, P).view(-1, 1))
    refs = refs.index_add(0, torch.where(drop, table, 0).flatten().long(), -drop.flatten().to(torch.int32))
    return torch.where(drop, -1, table), torch.where(back, to, length), refs


def _plain_reserve(p, want, P):
    """Sequences grow to `want` tokens: free pages by ascending number, in the order of the sequences; a shared last page is
    replaced by a copy first.  Returns the state and the copies, (from, to) with -1 where there is none."""
    table, length, refs = p
    most, n_pages = table.shape[1], refs.numel()
    grow = (want > length) & (want <= most * P)
    held, wanted = _pages_of(length, P), _pages_of(want, P)
    last = (length // P).clamp(max=most - 1).long().view(-1, 1)
    last_page = table.gather(1, last).view(-1)
    copy = grow & (length % P != 0) & (refs[last_page.clamp(min=0).long()] > 1)
    n = torch.where(grow, wanted - held + copy.int(), 0)
    end = n.cumsum(0)
    order = torch.sort((refs > 0).to(torch.int8), stable=True).indices.to(torch.int32)        # free pages first, ascending
    ok = grow & ((n == 0) | (end <= (refs == 0).sum()))
    first = end - n
    copy = copy & ok
    cols = torch.arange(most, device=DEV).view(1, -1)
    new = ok.view(-1, 1) & (cols >= held.view(-1, 1)) & (cols < wanted.view(-1, 1))
    rank = (first + copy.int() - held).view(-1, 1) + cols
    table = torch.where(new, order[rank.clamp(0, n_pages - 1).long()], table)
    fresh = order[first.clamp(0, n_pages - 1).long()]
    table = torch.where(copy.view(-1, 1) & (cols == last), fresh.view(-1, 1), table)
    refs = refs.index_add(0, torch.where(new, table, 0).flatten().long(), new.flatten().to(torch.int32))
    refs = refs.index_add(0, torch.where(copy, fresh, 0).long(), copy.to(torch.int32))
    refs = refs.index_add(0, torch.where(copy, last_page, 0).long(), -copy.to(torch.int32))
    return (table, torch.where(ok, want, length), refs), torch.where(copy, last_page, -1), torch.where(copy, fresh, -1)


def _plain_cycle(s):
    P = s["page_tokens"]
    p = (s["table"], s["len"], s["refs"])
    p, _, _ = _plain_reserve(p, s["committed"] + s["block"], P)
    p = _plain_rollback(p, s["committed"] + s["accepted"], P)
    return {"table": p[0], "len": p[1], "refs": p[2], "free_bits": _free_bits(p[2])}


def _plain_fork(s):
    P = s["page_tokens"]
    table, length, refs = _plain_rollback((s["table"], s["len"], s["refs"]), s["back_to"], P)
    src, dst = s["src"].long(), s["dst"].long()
    table, length = table.clone(), length.clone()
    table[dst], length[dst] = table[src], length[src]
    refs = refs.index_add(0, table[src].clamp(min=0).flatten().long(), (table[src] >= 0).flatten().to(torch.int32))
    (table, length, refs), old, new = _plain_reserve((table, length, refs), s["base"] + s["block"], P)
    there = old >= 0
    s["pool"][:, new[there].long()] = s["pool"][:, old[there].long()]
    return {"table": table, "len": length, "refs": refs, "free_bits": _free_bits(refs), "pool": s["pool"]}


def _plain_compact(s):
    table, refs = s["before"]["table"], s["before"]["refs"]
    live = refs > 0
    ids = torch.arange(refs.numel(), device=DEV)
    n_live = live.sum()
    movers, holes = ids[live & (ids >= n_live)], ids[~live & (ids < n_live)]
    to = ids.clone()
    to[movers] = holes
    s["pool"][:, holes] = s["pool"][:, movers]
    moved = torch.zeros_like(refs)
    moved[to[live]] = refs[live]
    table = torch.where(table >= 0, to[table.clamp(min=0).long()].to(torch.int32), table)
    return {"table": table, "len": s["len"], "refs": moved, "free_bits": _free_bits(moved), "pool": s["pool"]}


PLAIN = {"head": _plain_head, "controls": _plain_controls, "grammar": _plain_grammar, "cycle": _plain_cycle, "fork": _plain_fork,
         "compact": _plain_compact}


# ------------------------------------------------------------------ the package's calls
def _own_head(s):
    from paper_2510_26527_b200 import binding
    out, _ = binding.polyspec_lm_head_quantized(s["hidden"], s["qweight"], s["scales"], s["zero_points"], out=s["logits"])
    return {"logits": out}


def _own_controls(s):
    from paper_2510_26527_b200 import binding
    out, _ = binding.polyspec_process_logits(
        s["logits"], draft_tokens=s["draft_tokens"], history=s["tokens"], history_len=s["history_len"], prompt_len=s["prompt_len"],
        repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"], bias_tokens=s["bias_tokens"], bias_values=s["bias_values"],
        mask=s["bits"], out=s["out"])
    return {"logits": out}


def _own_grammar(s):
    from paper_2510_26527_b200 import binding
    out, _ = binding.polyspec_process_logits(s["logits"], mask=s["bits"], out=s["logits"])
    return {"logits": out}


def _own_pages(s):
    from paper_2510_26527_b200 import binding
    return binding, binding.CachePages(s["table"], s["len"], s["refs"], s["free_bits"], s["page_tokens"])


def _page_outputs(s):
    return {k: s[k] for k in ("table", "len", "refs", "free_bits", "pool") if k in s}


def _own_cycle(s):
    binding, pages = _own_pages(s)
    binding.polyspec_cache_reserve(pages, s["committed"], plus=s["block"])
    binding.polyspec_cache_rollback(pages, s["committed"], s["accepted"])
    return _page_outputs(s)


def _own_fork(s):
    binding, pages = _own_pages(s)
    binding.polyspec_cache_rollback(pages, s["back_to"])
    binding.polyspec_cache_fork(pages, s["src"], s["dst"])
    binding.polyspec_cache_reserve(pages, s["base"], plus=s["block"], pools=[s["pool"]])
    return _page_outputs(s)


def _own_compact(s):
    binding, pages = _own_pages(s)
    for k, v in s["before"].items():        # the holes, as the finished sequences left them
        s[k].copy_(v)
    binding.polyspec_cache_compact(pages, pools=[s["pool"]])
    return _page_outputs(s)


OWN = {"head": _own_head, "controls": _own_controls, "grammar": _own_grammar, "cycle": _own_cycle, "fork": _own_fork, "compact": _own_compact}


def run(state):
    return (OWN if own else PLAIN)[state["kind"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind == "head":
        rows, V, d, n = case["rows"], case["V"], case["d"], case["V"] * (case["d"] // case["group"])
        size = 2 if case["out"] == "bf16" else 4
        return {"bytes": V * d // 2 + n * (3 if case["zeros"] else 2) + rows * d * 2 + rows * V * size, "flops": 2 * rows * V * d}
    if kind in ("controls", "grammar"):
        B, rows, V = case["B"], case["rows"], case["V"]
        size = 2 if case["dt"] == "bf16" else 4
        masks = B * rows * ((V + 31) // 32) * 4
        if kind == "grammar":       # what is forbidden is written: about 17/32 of the entries
            return {"bytes": masks + int(B * rows * V * size * 17 / 32), "flops": 0}
        read = B * rows * V * size
        if case["mask"]:
            read = read * 17 // 32       # what the tight rows forbid need not be read (the loose rows' sectors all hold something allowed)
        return {"bytes": read + B * rows * V * size + B * (case["history"] * 3 + case["bias"] * 8 + 20) + (masks if case["mask"] else 0),
                "flops": 4 * B * rows * case["history"]}
    if kind == "cycle":
        return {"bytes": case["B"] * 32 + case["n_pages"] // 8, "flops": 0}
    if kind == "fork":
        n, P = case["parents"] * case["children"], case["page_tokens"]
        return {"bytes": int(2 * n * case["planes"] * case["page_bytes"] * (P - 1) / P) + n * 2 * 4 * (case["tokens"] // P + 1), "flops": 0}
    live = case["B"] * case["max_pages"] / 2
    moved = live * (1 - live / case["n_pages"])
    return {"bytes": int(2 * moved * case["planes"] * case["page_bytes"] + 8 * live + 8 * case["n_pages"]), "flops": 0}


# ------------------------------------------------------------------ 64-bit references, from the definitions
def exact(case, seed):
    if case["kind"] not in ("head", "controls", "grammar"):
        return None         # page numbers and moved data: nothing is computed
    s = prepare(case, seed)
    if case["kind"] == "head":
        V, d, group = case["V"], case["d"], case["group"]
        h = s["hidden"].double()
        out = torch.empty((case["rows"], V), dtype=torch.float64, device=DEV)
        step = max(1, (1 << 27) // d)
        place = torch.tensor([0, 4, 1, 5, 2, 6, 3, 7], device=DEV)       # the nibble (counted from bit 0) that holds weight e of eight
        for v in range(0, V, step):
            byte = s["qweight"][v:v + step].contiguous().view(torch.uint8)
            nib = torch.stack([byte % 16, byte // 16], -1).reshape(byte.shape[0], d // 8, 8)[..., place].reshape(-1, d).double()
            zero = s["zero_points"][v:v + step].double().repeat_interleave(group, 1) if case["zeros"] else 8.0
            out[:, v:v + step] = h @ ((nib - zero) * s["scales"][v:v + step].double().repeat_interleave(group, 1)).t()
        return {"logits": out}
    z = s["logits"].double()
    B, rows, V = z.shape
    if case["kind"] == "controls":
        for b in range(B):
            n, m = int(s["history_len"][b]), int(s["prompt_len"][b])
            r, f, p = (float(s[k][b]) for k in ("repetition", "frequency", "presence"))
            text = s["tokens"][b, :n].long()
            for j in range(rows):
                output = torch.cat([text[m:], s["draft_tokens"][b, :j].long()])
                ids, times = torch.unique(output, return_counts=True)
                row = z[b, j]
                some = torch.unique(torch.cat([text[:m], ids]))
                was = row[some]
                row[some] = torch.where(was > 0, was / r, was * r)
                row[ids] -= f * times.double() + p
                if case["bias"]:
                    row.index_put_((s["bias_tokens"][b].long(),), s["bias_values"][b].double(), accumulate=True)
    if s["bits"] is not None:
        byte = s["bits"].contiguous().view(torch.uint8).view(B, rows, -1)
        for i in range(8):
            part = z[..., i::8]
            part[((byte >> i) % 2 == 0)[..., : part.shape[-1]]] = float("-inf")
    return {"logits": z}
