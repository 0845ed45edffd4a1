"""The attention around the cache pages in plain 64-bit arithmetic, written from the formulas: nothing here is the product's code.

A Cache holds page tables, and codes, scales and offsets as plain arrays by (sequence, slot, head); `pool` lays them out as pages, with
NaN and random codes wherever no token lies.  Each computed result comes with a bound on the error that its arithmetic may have:
U16, UB, U32 are half a step of fp16, bf16 and fp32 relative to a value."""
import numpy as np
import torch

U16, UB, U32 = 2.0 ** -11, 2.0 ** -8, 2.0 ** -24
APPROX = 2.0 ** -21          # relative error of an approximated exponential, logarithm (absolute) or reciprocal, with room


def bf16(x):
    return torch.as_tensor(np.asarray(x, np.float32)).to(torch.bfloat16).float().numpy()


def bits(x):
    """fp32 numbers that are bf16 numbers -> their 16 bits."""
    return (np.ascontiguousarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint32)


def words(codes):
    """[..., d] codes -> [..., d / 8] words."""
    c = codes.reshape(*codes.shape[:-1], codes.shape[-1] // 8, 8).astype(np.uint32)
    out = np.zeros(c.shape[:-1], np.uint32)
    for e in range(8):
        out |= c[..., e] << np.uint32(4 * (e // 2) + 16 * (e % 2))
    return out


def word_places(d, values):
    n = d // 8
    at = np.zeros((8, n), int)
    for r in range(8):
        for w in range(n):
            g, h, t, o = w % 8, w // 8, r // 2, r % 2
            at[r, w] = ((4 * g + t) * 2 + o) * (d // 64) + h if values else r * n + w
    return at


def quantise(x):
    """[..., d] fp32 numbers that are bf16 numbers -> codes, scale, offset, held values (fp32 arithmetic, as the operator's definition has it)."""
    x = np.asarray(x, np.float32)
    lo, hi = x.min(-1), x.max(-1)
    with np.errstate(all="ignore"):
        step = ((hi - lo) / np.float32(15)).astype(np.float32)
        up = ((step.view(np.uint32) + np.uint32(0xffff)) & np.uint32(0xffff0000)).view(np.float32)
        up = np.where(up == 0, np.float32(1), np.maximum(up, np.float32(2.0 ** -126)))
        code = np.rint(((x - lo[..., None]) / up[..., None]).astype(np.float32))
        broken = ~np.isfinite(x).all(-1) | ~np.isfinite(hi - lo)
        code = np.where(broken[..., None], 0, np.minimum(code, 15)).astype(np.int64)
        up, lo = np.where(broken, np.float32(np.nan), up), np.where(broken, np.float32(np.nan), lo)
        held = bf16((up[..., None] * code.astype(np.float32)).astype(np.float32) + lo[..., None])
    return code, up, lo + np.float32(0), held


class Cache:
    def __init__(self, lens, kv_heads, d, page_tokens, seed=0, spare=3, max_tokens=None, scale=(0.2, 0.5), far=1.0):
        rng = np.random.default_rng(seed)
        self.rng, self.kv, self.d, self.P, self.lens = rng, kv_heads, d, page_tokens, list(lens)
        B = len(lens)
        most = max([1] + [-(-n // page_tokens) for n in lens])
        if max_tokens:
            most = max(most, -(-max_tokens // page_tokens))
        self.max_pages, self.cap = most, most * page_tokens
        held = [-(-n // page_tokens) for n in lens]
        self.n_pages = sum(held) + spare
        ids = rng.permutation(self.n_pages).astype(np.int32)
        self.table = np.full((B, most), -1, np.int32)
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = ids[at:at + n]
            at += n
        self.refs = np.zeros(self.n_pages, np.int32)
        self.refs[ids[:at]] = 1
        # [keys, values][sequence][slot, head]
        self.codes = [[rng.integers(0, 16, (n, kv_heads, d)) for n in lens] for _ in range(2)]
        self.scale = [[bf16(rng.uniform(*scale, (n, kv_heads))) for n in lens] for _ in range(2)]
        self.offset = [[bf16(s * (-7.5 + far * rng.standard_normal(s.shape))) for s in self.scale[p]] for p in range(2)]

    def value(self, plane, b):
        return self.scale[plane][b].astype(np.float64)[..., None] * self.codes[plane][b] + self.offset[plane][b].astype(np.float64)[..., None]

    def page_bytes(self):
        return self.kv * (self.P // 8) * (4 * self.d + 32)

    def empty_pool(self, planes=2):
        unit = self.d + 8
        x = self.rng.integers(0, 2 ** 32, (planes, self.n_pages, self.kv, self.P // 8, unit), dtype=np.uint32)
        x[..., self.d:] = np.uint32(0x7fc07fc0)
        return x

    def put(self, pool, plane, b, slots, codes, scale, offset, values=None):
        """Writes tokens [n, kv, d] of sequence b into a plane of a pool of words."""
        at = word_places(self.d, plane % 2 == 1 if values is None else values)
        w = words(codes)
        for i, slot in enumerate(slots):
            page, unit, r = self.table[b, slot // self.P], slot % self.P // 8, slot % 8
            pool[plane, page, :, unit][:, at[r]] = w[i]
            pool[plane, page, :, unit, self.d + r] = bits(scale[i]) | bits(offset[i]) << np.uint32(16)

    def pool(self, planes=2):
        x = self.empty_pool(planes)
        for p in range(planes):
            for b, n in enumerate(self.lens):
                self.put(x, p, b, range(n), self.codes[p % 2][b], self.scale[p % 2][b], self.offset[p % 2][b])
        return x

    def free_bits(self):
        free = np.zeros(-(-self.n_pages // 32) * 32, np.int64)
        free[: self.n_pages] = self.refs == 0
        return (free.reshape(-1, 32) << np.arange(32)).sum(1).astype(np.uint32).view(np.int32)

    def to(self, device):
        from paper_2510_26527_b200 import binding
        t = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(device)
        return binding.CachePages(t(self.table), t(np.asarray(self.lens, np.int32)), t(self.refs), t(self.free_bits()), self.P)

    def words_on(self, pool, device):
        return torch.from_numpy(pool.view(np.int32).reshape(pool.shape[0], self.n_pages, -1).copy()).to(device)


def attend(cache, q, rows_at, base, n_rows=None, scale=None):
    """q [rows, heads, d] fp32 (bf16 numbers).  Returns out, lse, bounds of both, and per sequence the weights [slots] with theirs."""
    rows, heads, d = q.shape
    group = heads // cache.kv
    scale = d ** -0.5 if scale is None else scale
    out, tol = np.full((rows, heads, d), np.nan), np.full((rows, heads, d), np.nan)
    lse, tol_lse = np.full((rows, heads), np.nan), np.full((rows, heads), np.nan)
    weights = [np.zeros(n) for n in cache.lens]
    tol_w = [np.zeros(n) for n in cache.lens]
    for b, n in enumerate(cache.lens):
        count = rows_at[b + 1] - rows_at[b] if n_rows is None else n_rows[b]
        K, V = cache.value(0, b), cache.value(1, b)
        for i in range(count):
            row, m = rows_at[b] + i, base[b] + i + 1
            if m > n or base[b] < 0:
                out[row], lse[row], tol[row], tol_lse[row] = 0, -np.inf, 0, 0
                continue
            for h in range(heads):
                k, v, x = K[:m, h // group], V[:m, h // group], q[row, h].astype(np.float64)
                s = scale * (k @ x)
                # sums of d products and a few roundings of scale, offset and maximum, in fp32
                size = abs(scale) * (cache.scale[0][b][:m, h // group] * (cache.codes[0][b][:m, h // group] @ np.abs(x))
                                     + np.abs(cache.offset[0][b][:m, h // group]) * np.abs(x).sum())
                e = (d + 8) * U32 * size + 4 * U32 * np.abs(s) + APPROX + 16 * U32
                top = s.max()
                p = np.exp(s - top)
                total = p.sum()
                p /= total
                out[row, h], lse[row, h] = p @ v, top + np.log(total)
                # rounded weights times codes; weights off by their scores' errors; sums; the last rounding
                coded = p[:, None] * cache.scale[1][b][:m, h // group][:, None] * cache.codes[1][b][:m, h // group]
                part = coded + p[:, None] * np.abs(cache.offset[1][b][:m, h // group])[:, None]
                few = p * e
                tol[row, h] = UB * np.abs(out[row, h]) + (U16 + 2.0 ** -31 * m) * coded.sum(0) + 2 * (e[:, None] * part).sum(0) \
                    + 2 * few.sum() * np.abs(out[row, h]) + (m + 64) * U32 * part.sum(0) + 2.0 ** -130
                tol_lse[row, h] = few.sum() + (m + 64) * U32 + 4 * U32 * abs(lse[row, h])
                weights[b][:m] += p
                tol_w[b][:m] += p * (2 * e + tol_lse[row, h] + (rows * heads + 8) * U32)
    return out, lse, tol, tol_lse, weights, tol_w


def prompt(q, k, v, rows_at, scale=None):
    """Causal attention of packed prompts in 64 bits, with bounds: scores of bf16 products summed in fp32, weights rounded to bf16 for their product."""
    rows, heads, d = q.shape
    kv = k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    out, tol = np.full((rows, heads, d), np.nan), np.full((rows, heads, d), np.nan)
    lse, tol_lse = np.full((rows, heads), np.nan), np.full((rows, heads), np.nan)
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    for b in range(len(rows_at) - 1):
        lo, hi = rows_at[b], rows_at[b + 1]
        if hi <= lo:
            continue
        n = hi - lo
        for h in range(heads):
            x, y, z = q[lo:hi, h], k[lo:hi, h // (heads // kv)], v[lo:hi, h // (heads // kv)]
            seen = np.tril(np.ones((n, n), bool))
            s = np.where(seen, scale * (x @ y.T), -np.inf)
            size = abs(scale) * (np.abs(x) @ np.abs(y).T)
            e = np.where(seen, (d + 8) * U32 * size + 4 * U32 * np.abs(np.where(seen, s, 0)) + APPROX + 16 * U32, 0)
            top = s.max(1, keepdims=True)
            p = np.exp(s - top)
            total = p.sum(1, keepdims=True)
            p /= total
            out[lo:hi, h], lse[lo:hi, h] = p @ z, (top + np.log(total))[:, 0]
            few = (p * e).sum(1)
            part = p @ np.abs(z)
            tol[lo:hi, h] = UB * np.abs(out[lo:hi, h]) + (UB + (n + 64) * U32 + 2.0 ** -31 * n) * part + 2 * ((p * e) @ np.abs(z)) + 2 * few[:, None] * part
            tol_lse[lo:hi, h] = few + (n + 64) * U32 + 4 * U32 * np.abs(lse[lo:hi, h])
    return out, lse, tol, tol_lse


def rotate(x, weight, positions, frequencies, interleaved, eps=1e-6):
    """[rows, heads, d] -> rotated in 64 bits, and the bound: fp32 norm, angle and products, one rounding to bf16."""
    d = x.shape[-1]
    y = x.astype(np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * weight.astype(np.float64)
    out, size = y.copy(), np.abs(y)
    r = 0 if frequencies is None else 2 * len(frequencies)
    if r:
        angle = positions.astype(np.float64)[:, None, None] * frequencies.astype(np.float64)
        c, s = np.cos(angle), np.sin(angle)
        i = np.arange(r // 2)
        ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        a, b = y[..., ia], y[..., ib]
        out[..., ia], out[..., ib] = a * c - b * s, a * s + b * c
        size[..., ia] = size[..., ib] = np.abs(a) + np.abs(b)
    return out, UB * np.abs(out) + (d + 32) * U32 * size + 2.0 ** -130


def evict_slots(weights, n, budget, first, recent):
    """The slots that stay, in order."""
    if budget < 0 or n <= budget:
        return None
    if budget < first + recent:
        return "bad"
    w = [(-np.inf if np.isnan(x) else x) for x in weights[:n].tolist()]
    nan = [np.isnan(x) for x in weights[:n].tolist()]
    middle = sorted(range(first, n - recent), key=lambda j: (nan[j], -w[j], j))[: budget - first - recent]
    return sorted(list(range(first)) + middle + list(range(n - recent, n)))
