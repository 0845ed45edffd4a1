"""Calls on 4-bit caches at the ends of what they take: scales of values far apart, heads of equal elements, rows that attend to nothing, ranges at the
end of fp32, tables of many tokens, shared pages, several calls at once.  Against 64-bit arithmetic."""
import numpy as np
import pytest
import torch

from paper_2510_26527_b200 import binding, buildlib
from tests import plain_attention as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BAD = binding.ERR_BAD_INPUT_ON_DEVICE


@pytest.fixture(scope="module", autouse=True)
def _lib():
    buildlib.build()
    binding.load_library()
    assert torch.cuda.is_available()


def _i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def _normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _close(got, want, tol):
    got = got.detach().cpu().double().numpy()
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want) - tol
    assert (same | (off <= 0)).all(), (float(np.nanmax(np.where(same, -1, off))), np.argwhere(~same & ~(off <= 0))[:4])


def _starts(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(int).tolist()


# ------------------------------------------------------------------ attention: scales of values
def _finest(c, q, at, base):
    """What the second product's weights, fp16 numbers of an absolute half step of 2^-25, may add to each output: 15 times that per token, where the
    largest weight times scale of a token with a code above 0 is held as 2^3 at least, or, where scales are too small for that, 1 as 2^121."""
    rows, heads, d = q.shape
    add = np.zeros((rows, heads, 1))
    for b in range(len(c.lens)):
        for row in range(at[b], at[b + 1]):
            m = base[b] + row - at[b] + 1
            for h in range(heads):
                g = h // (heads // c.kv)
                s = d ** -0.5 * (c.value(0, b)[:m, g] @ q[row, h].astype(np.float64))
                p = np.exp(s - s.max())
                p /= p.sum()
                real = c.codes[1][b][:m, g].any(-1)
                add[row, h] = m * (15 * 2.0 ** -28 * max([0.0, *(p * c.scale[1][b][:m, g])[real]]) + 2.0 ** -142)
    return add


SHAPES = [([1], 4, 4), ([1, 1], 16, 2), ([9], 8, 2), ([5, 3], 12, 3)]         # rows of a block, query heads, key heads: one group of 8 rows, or more


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("counts,heads,kv", SHAPES)
@pytest.mark.parametrize("lo,hi", [(-126, 96), (-126, -118), (-70, -50), (80, 96)])
def test_softmax_does_not_depend_on_the_scales_of_values(d, counts, heads, kv, lo, hi):
    lens = [150 + 40 * b for b in range(len(counts))]
    c = plain.Cache(lens, kv, d, 16, 400)
    for b, n in enumerate(lens):
        c.scale[1][b] = plain.bf16(np.exp2(c.rng.uniform(lo, hi, (n, kv))))
        c.offset[1][b] = plain.bf16(c.scale[1][b] * (-7.5 + c.rng.standard_normal((n, kv))))
    at, base = _starts(counts), [n - k for n, k in zip(lens, counts)]
    q = _normal(401, at[-1], heads, d)
    pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
    lse = torch.zeros((at[-1], heads), device=DEV)
    out, _, st = binding.polyspec_cache_attention(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse=lse)
    assert int(st) == 0
    qn = q.float().numpy()
    want, want_lse, tol, tol_lse, weights, tol_w = plain.attend(c, qn, at, base)
    _close(lse, want_lse, tol_lse)
    _close(out, want, tol + _finest(c, qn, at, base))
    w = torch.zeros((len(lens), c.cap), device=DEV)
    binding.polyspec_cache_weigh(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse, w)
    for b, n in enumerate(lens):
        _close(w[b, :n], weights[b], tol_w[b] + 4 * plain.U32 * (1 + weights[b]))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tiny", [-126, -100, -60])
@pytest.mark.parametrize("kind", ["equal scores", "offsets"])
def test_tokens_of_tiny_scales_keep_their_weight(d, tiny, kind):
    """Two tokens of equal scores, one with a tiny scale beside an ordinary one; or many with a tiny scale and an offset of any size."""
    n = 2 if kind == "equal scores" else 90
    c = plain.Cache([n], 2, d, 8, 410)
    c.scale[1][0][:1 if n == 2 else n] = 2.0 ** tiny
    c.offset[1][0][:] = plain.bf16(np.exp2(c.rng.uniform(-10, 60, (n, 2))) * c.rng.choice([-1, 1], (n, 2)))
    if n == 2:
        c.scale[1][0][1] = 16.0
        c.offset[1][0][:] = 0.0
        for x in (c.codes[0][0], c.scale[0][0], c.offset[0][0]):
            x[1] = x[0]
    q = _normal(411, 1, 4, d)
    lse = torch.zeros((1, 4), device=DEV)
    out, _, st = binding.polyspec_cache_attention(c.to(DEV), q.to(DEV), c.words_on(c.pool(), DEV), 2, _i32([0, 1]), _i32([n - 1]), lse=lse)
    assert int(st) == 0
    qn = q.float().numpy()
    want, want_lse, tol, tol_lse, _, _ = plain.attend(c, qn, [0, 1], [n - 1])
    _close(lse, want_lse, tol_lse)
    _close(out, want, tol + _finest(c, qn, [0, 1], [n - 1]))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("counts,heads,kv", [([1], 2, 2), ([9], 4, 1), ([3, 1], 8, 2)])
@pytest.mark.parametrize("at_slot,scale,value,size", [(0, 1.0, 0.0, 0.0006), (8000, 1.0, 0.0, 0.0006), (5000, 64.0, 0.0, 0.009), (0, 1.0, 0.25, 0.009)])
def test_a_head_of_equal_elements_takes_no_bits_from_the_others(d, counts, heads, kv, at_slot, scale, value, size):
    """A token whose values are all the same (all of its codes 0) has 0.99 of the weight, over thousands of small ones."""
    lens = [8192 - 100 * b for b in range(len(counts))]
    c = plain.Cache(lens, kv, d, 64, 420, scale=(0.01, 0.02))
    at, base = _starts(counts), [n - k for n, k in zip(lens, counts)]
    q = _normal(421, 1, kv, d).repeat_interleave(heads // kv, 1).repeat(at[-1], 1, 1)           # one direction for each key head's rows
    qn = q.float().numpy()
    for b, n in enumerate(lens):
        c.scale[1][b] = plain.bf16(c.rng.uniform(0.6 * size, size, (n, kv)))
        c.offset[1][b] = plain.bf16(c.scale[1][b] * (-7.5 + c.rng.standard_normal((n, kv))))
        slot = min(at_slot, base[b])
        for g in range(kv):
            x = qn[0, g * (heads // kv)].astype(np.float64)
            s = d ** -0.5 * (c.value(0, b)[:, g] @ x)
            target = np.log(99.0) + np.log(np.exp(s - s.max()).sum()) + s.max()
            c.codes[0][b][slot, g] = np.where(x > 0, 15, 0)
            c.scale[0][b][slot, g] = plain.bf16(target / (d ** -0.5 * 7.5 * np.abs(x).sum()))
            c.offset[0][b][slot, g] = plain.bf16(-7.5 * c.scale[0][b][slot, g])
            c.codes[1][b][slot, g], c.scale[1][b][slot, g], c.offset[1][b][slot, g] = 0, scale, value
    lse = torch.zeros((at[-1], heads), device=DEV)
    out, _, st = binding.polyspec_cache_attention(c.to(DEV), q.to(DEV), c.words_on(c.pool(), DEV), kv, _i32(at), _i32(base), lse=lse)
    assert int(st) == 0
    want, want_lse, tol, tol_lse, _, _ = plain.attend(c, qn, at, base)
    _close(lse, want_lse, tol_lse)
    _close(out, want, tol + _finest(c, qn, at, base))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("counts,heads,kv", [([1], 2, 2), ([9], 4, 1)])
@pytest.mark.parametrize("scale", [2.0 ** -126, 2.0 ** -45, 2.0 ** -23, 1.0])
def test_values_of_up_to_2_to_the_64th(d, counts, heads, kv, scale):
    """Offsets near 2^64 of either sign with any scale; half of the heads have codes of 0 throughout."""
    n = 3000
    c = plain.Cache([n], kv, d, 64, 425)
    c.scale[1][0][:] = scale
    c.offset[1][0][:] = plain.bf16(c.rng.uniform(-1, 1, (n, kv)) * 2.0 ** 64)
    c.codes[1][0][c.rng.random((n, kv)) < 0.5] = 0
    c.codes[1][0][:40] = 0
    at, base = _starts(counts), [n - counts[0]]
    q = _normal(426, at[-1], heads, d)
    lse = torch.zeros((at[-1], heads), device=DEV)
    out, _, st = binding.polyspec_cache_attention(c.to(DEV), q.to(DEV), c.words_on(c.pool(), DEV), kv, _i32(at), _i32(base), lse=lse)
    assert int(st) == 0
    qn = q.float().numpy()
    want, want_lse, tol, tol_lse, _, _ = plain.attend(c, qn, at, base)
    _close(lse, want_lse, tol_lse)
    _close(out, want, tol + _finest(c, qn, at, base))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("counts,heads,kv", [([1], 2, 2), ([9], 4, 1)])
@pytest.mark.parametrize("more", [10, 25, 45, 70])
@pytest.mark.parametrize("equal", [[0], [2000], list(range(300)), list(range(0, 2990, 3))], ids=["first", "middle", "many first", "every third"])
def test_a_head_of_equal_elements_of_any_weight(d, counts, heads, kv, more, equal):
    """Zero-valued tokens whose weights are 2^more of the others': these are all that the output is made of."""
    n = 3000
    c = plain.Cache([n], kv, d, 64, 427, scale=(0.01, 0.02))
    at, base = _starts(counts), [n - counts[0]]
    q = _normal(428, 1, kv, d).repeat_interleave(heads // kv, 1).repeat(at[-1], 1, 1)           # one direction for each key head's rows
    qn = q.float().numpy()
    for g in range(kv):
        x = qn[0, g * (heads // kv)].astype(np.float64)
        c.codes[0][0][equal, g] = np.where(x > 0, 15, 0)
        c.scale[0][0][equal, g] = plain.bf16(more * np.log(2.0) / (d ** -0.5 * 7.5 * np.abs(x).sum()))
        c.offset[0][0][equal, g] = plain.bf16(-7.5 * c.scale[0][0][equal, g])
        c.codes[1][0][equal, g], c.scale[1][0][equal, g], c.offset[1][0][equal, g] = 0, 1.0, 0.0
    lse = torch.zeros((at[-1], heads), device=DEV)
    out, _, st = binding.polyspec_cache_attention(c.to(DEV), q.to(DEV), c.words_on(c.pool(), DEV), kv, _i32(at), _i32(base), lse=lse)
    assert int(st) == 0
    want, want_lse, tol, tol_lse, _, _ = plain.attend(c, qn, at, base)
    _close(lse, want_lse, tol_lse)
    _close(out, want, tol + _finest(c, qn, at, base))


# ------------------------------------------------------------------ rows that attend to nothing
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("change", [{"n_rows": [3, 4, 3]}, {"n_rows": [3, -1, 3]}, {"n_rows": [3, 2, 3], "len": -1}, {"len": -1}, {"len": 1 << 20}, {"base": -4}, {"base": 2 ** 31 - 1}])
def test_every_row_of_a_sequence_whose_numbers_make_no_sense_gets_zeros(d, change):
    c = plain.Cache([20, 9, 33], 2, d, 8, 430)
    at, base, n_rows = [0, 3, 6, 9], [17, 6, 30], change.get("n_rows")
    q = _normal(431, 9, 4, d)
    want, want_lse, tol, tol_lse, weights, tol_w = plain.attend(c, q.float().numpy(), at, base)
    want[3:6], want_lse[3:6], tol[3:6], tol_lse[3:6] = 0, -np.inf, 0, 0
    if n_rows == [3, 2, 3]:                                 # the row that belongs to nobody stays
        want[5], want_lse[5] = 9, 9
    pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
    base[1] = change.get("base", base[1])
    pages.len[1] = change.get("len", 9)
    n_rows = None if n_rows is None else _i32(n_rows)
    out = torch.full((9, 4, d), 9.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((9, 4), 9.0, device=DEV)
    _, _, st = binding.polyspec_cache_attention(pages, q.to(DEV), on, 2, _i32(at), _i32(base), n_rows=n_rows, out=out, lse=lse)
    assert int(st) == BAD
    _close(out, want, tol)
    _close(lse, want_lse, tol_lse)
    w = torch.full((3, c.cap), 2.0, device=DEV)
    assert int(binding.polyspec_cache_weigh(pages, q.to(DEV), on, 2, _i32(at), _i32(base), lse, w, n_rows=n_rows)) == BAD
    for b in (0, 2):
        _close(w[b, :c.lens[b]], 2 + weights[b], tol_w[b] + 4 * plain.U32 * (2 + weights[b]))
    assert (w[1] == 2).all()
    x, before = _normal(432, 9, 2, d).to(DEV), on.clone()
    assert int(binding.polyspec_cache_append(pages, x, x, on, _i32(at), _i32(base), n_rows=n_rows)) == BAD
    held = torch.from_numpy(c.table[1][c.table[1] >= 0].astype(np.int64)).to(DEV)
    assert torch.equal(on[:, held], before[:, held])


@pytest.mark.parametrize("counts,heads,kv", [([1, 1], 2, 2), ([4, 2], 16, 2)])
def test_rows_none_of_whose_pages_can_be_read_get_zeros(counts, heads, kv):
    lens, d, P = [40, 300], 128, 8
    for unreadable in ([0], [1], [0, 1]):
        c = plain.Cache(lens, kv, d, P, 440)
        at, base = _starts(counts), [n - k for n, k in zip(lens, counts)]
        q = _normal(441, at[-1], heads, d)
        want, want_lse, tol, tol_lse, _, _ = plain.attend(c, q.float().numpy(), at, base)
        pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
        for b in unreadable:
            pages.table[b] = c.n_pages + 3
            rows = slice(at[b], at[b + 1])
            want[rows], want_lse[rows], tol[rows], tol_lse[rows] = 0, -np.inf, 0, 0
        out = torch.full((at[-1], heads, d), 9.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((at[-1], heads), 9.0, device=DEV)
        _, _, st = binding.polyspec_cache_attention(pages, q.to(DEV), on, kv, _i32(at), _i32(base), out=out, lse=lse)
        assert int(st) == BAD
        _close(out, want, tol)
        _close(lse, want_lse, tol_lse)


# ------------------------------------------------------------------ append, queries: ends of the number range
@pytest.mark.parametrize("d", [64, 128])
def test_append_of_ranges_up_to_the_end_of_fp32(d):
    """Ranges between 3.39e38 and the largest finite number have codes; beyond it every value is NaN."""
    n, kv = 24, 2
    c = plain.Cache([n], kv, d, 8, 450)
    x = _normal(451, n, kv, d).float() * 1e37
    top = torch.tensor(3.3895313892515355e38)
    x[:, :, 3] = top
    low = -torch.linspace(0.9e36, 2.1e36, n).view(n, 1)
    x = torch.maximum(x, low.unsqueeze(-1))
    x[:, :, 7] = low
    x = x.to(torch.bfloat16)
    code, scale, offset, back = plain.quantise(x.float().numpy())
    ranges = x.float().amax(-1) - x.float().amin(-1)
    assert (ranges.isfinite() & (ranges > 3.4e38)).any() and ranges.isinf().any()
    pool = c.empty_pool()
    pages, on = c.to(DEV), c.words_on(pool, DEV)
    held = torch.zeros((n, kv, d), dtype=torch.bfloat16, device=DEV)
    assert int(binding.polyspec_cache_append(pages, x.to(DEV), x.to(DEV), on, _i32([0, n]), _i32([0]), k_held=held)) == 0
    for p in range(2):
        c.put(pool, p, 0, range(n), code, scale, offset)
    assert (on.cpu().numpy().view(np.uint32).reshape(pool.shape) == pool).all()
    got = held.float().cpu().numpy()
    assert ((got == back) | (np.isnan(got) & np.isnan(back))).all()


@pytest.mark.parametrize("counts,heads,kv", [([1], 4, 4), ([9], 8, 2)])
@pytest.mark.parametrize("power", [60, 117, 118, 126])
def test_large_queries_with_a_small_scale(counts, heads, kv, power):
    n, d = 70, 128
    c = plain.Cache([n], kv, d, 16, 460)
    at, base = _starts(counts), [n - counts[0]]
    q = (_normal(461, at[-1], heads, d).float().clamp(-1.9, 1.9) * 2.0 ** power).to(torch.bfloat16)
    q[:, :, 0] = 2.0 ** power * 1.5
    scale = d ** -0.5 * 2.0 ** -power
    pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
    lse = torch.zeros((at[-1], heads), device=DEV)
    out, _, st = binding.polyspec_cache_attention(pages, q.to(DEV), on, kv, _i32(at), _i32(base), scale=scale, lse=lse)
    assert int(st) == 0
    want, want_lse, tol, tol_lse, weights, tol_w = plain.attend(c, q.float().numpy(), at, base, scale=scale)
    _close(out, want, tol)
    _close(lse, want_lse, tol_lse)
    w = torch.zeros((1, c.cap), device=DEV)
    binding.polyspec_cache_weigh(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse, w, scale=scale)
    _close(w[0, :n], weights[0], tol_w[0] + 4 * plain.U32 * (1 + weights[0]))


@pytest.mark.parametrize("counts,heads,kv", [([1], 4, 4), ([9], 8, 2)])
@pytest.mark.parametrize("scale", [-0.11, 0.0])
def test_scales_below_and_at_zero(counts, heads, kv, scale):
    n, d = 150, 64
    c = plain.Cache([n], kv, d, 16, 465)
    at, base = _starts(counts), [n - counts[0]]
    q = _normal(466, at[-1], heads, d)
    pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
    lse = torch.zeros((at[-1], heads), device=DEV)
    out, _, st = binding.polyspec_cache_attention(pages, q.to(DEV), on, kv, _i32(at), _i32(base), scale=scale, lse=lse)
    assert int(st) == 0
    want, want_lse, tol, tol_lse, weights, tol_w = plain.attend(c, q.float().numpy(), at, base, scale=scale)
    _close(out, want, tol)
    _close(lse, want_lse, tol_lse)
    w = torch.zeros((1, c.cap), device=DEV)
    binding.polyspec_cache_weigh(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse, w, scale=scale)
    _close(w[0, :n], weights[0], tol_w[0] + 4 * plain.U32 * (1 + weights[0]))


# ------------------------------------------------------------------ eviction
def test_evict_with_tables_of_more_tokens_than_shared_memory_holds():
    """Tables for 50048 tokens: a sequence of 50001, whose weights are read from memory, and a short one, whose weights fit."""
    lens, budget, kv, d, P = [50001, 700], [1500, 90], 1, 64, 64
    c = plain.Cache(lens, kv, d, P, 470, max_tokens=50048)
    w = np.random.default_rng(471).integers(0, 500, (2, c.cap)).astype(np.float32)
    w[:, ::9] = np.nan
    pages, pool = c.to(DEV), c.pool()
    on, won = c.words_on(pool, DEV), torch.from_numpy(w.copy()).to(DEV)
    kept_from = torch.full((2, c.cap), 5, dtype=torch.int32, device=DEV)
    assert int(binding.polyspec_cache_evict(pages, _i32(budget), won, on, kv, d, first=3, recent=40, kept_from=kept_from)) == 0
    assert pages.len.tolist() == budget
    want_from = np.full((2, c.cap), -1)
    for b in range(2):
        keep = plain.evict_slots(w[b], lens[b], budget[b], 3, 40)
        moved = [i for i, j in enumerate(keep) if i != j]
        old = [keep[i] for i in moved]
        for p in range(2):
            c.put(pool, p, b, moved, c.codes[p][b][old], c.scale[p][b][old], c.offset[p][b][old])
        w[b, : len(keep)] = w[b, keep]
        want_from[b, : len(keep)] = keep
        c.refs[c.table[b, -(-budget[b] // P):-(-lens[b] // P)]] -= 1
        c.table[b, -(-budget[b] // P):] = -1
    assert (kept_from.cpu().numpy() == want_from).all()
    assert (won.cpu().numpy().view(np.uint32) == w.view(np.uint32)).all()
    assert (pages.table.cpu().numpy() == c.table).all() and (pages.refs.cpu().numpy() == c.refs).all()
    assert (pages.free_bits.cpu().numpy() == c.free_bits()).all()
    assert (on.cpu().numpy().view(np.uint32).reshape(pool.shape) == pool).all()


def test_evict_where_nothing_moves_does_not_look_at_shared_pages():
    """The heaviest tokens are the first: sequences are cut behind them, a last page that is kept in part may be held by others."""
    lens, kv, d, P = [64, 64, 64], 2, 64, 8
    c = plain.Cache(lens, kv, d, P, 480)
    w = np.tile(np.arange(c.cap, dtype=np.float32)[::-1], (3, 1)).copy()
    budget = [44, 40, 44]
    w[2, 50] = 1000.0                                       # here one token moves, into the shared page
    for b in range(3):
        c.refs[c.table[b, 5]] = 2
    c.refs[c.table[0, 7]] = 3
    pages, pool = c.to(DEV), c.pool()
    on, won = c.words_on(pool, DEV), torch.from_numpy(w.copy()).to(DEV)
    kept_from = torch.full((3, c.cap), 5, dtype=torch.int32, device=DEV)
    assert int(binding.polyspec_cache_evict(pages, _i32(budget), won, on, kv, d, kept_from=kept_from)) == BAD
    assert pages.len.tolist() == [44, 40, 64]
    for b in range(2):
        c.refs[c.table[b, -(-budget[b] // P):]] -= 1
        c.table[b, -(-budget[b] // P):] = -1
        assert (kept_from[b].cpu().numpy() == [i if i < budget[b] else -1 for i in range(c.cap)]).all()
    assert (kept_from[2] == -1).all()
    assert (pages.table.cpu().numpy() == c.table).all() and (pages.refs.cpu().numpy() == c.refs).all()
    assert (won.cpu().numpy() == w).all()
    assert (on.cpu().numpy().view(np.uint32).reshape(pool.shape) == pool).all()


def test_evictions_side_by_side_with_attention():
    """Two caches shortened on two streams while a third and a fourth are attended to: each as if it were alone."""
    kv, d, P = 2, 128, 16
    lens = [900, 300, 1500, 40]
    budget = _i32([200, 300, 700, 39])

    def state(seed):
        c = plain.Cache(lens, kv, d, P, seed)
        w = torch.rand((len(lens), c.cap), generator=torch.Generator().manual_seed(seed)).to(DEV)
        return c.to(DEV), c.words_on(c.pool(4), DEV), w

    at, base = _i32(_starts([3] * 4)), _i32(n - 3 for n in lens)
    q = [_normal(490 + i, 12, 8, d).to(DEV) for i in range(2)]
    readers = [state(492 + i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(4)]
    evict = lambda s: binding.polyspec_cache_evict(s[0], budget, s[2], s[1], kv, d, first=2, recent=20)
    attend = lambda i: binding.polyspec_cache_attention(readers[i][0], q[i], readers[i][1][:2], kv, at, base)[0]
    alone, alone_out = [state(494 + i) for i in range(2)], [attend(i).clone() for i in range(2)]
    for s in alone:
        assert int(evict(s)) == 0
    for _ in range(5):
        cut, got = [state(494 + i) for i in range(2)], []
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                evict(cut[i])
            with torch.cuda.stream(streams[2 + i]):
                got.append(attend(i))
        torch.cuda.synchronize()
        for i in range(2):
            for name in ("table", "len", "refs", "free_bits"):
                assert torch.equal(getattr(cut[i][0], name), getattr(alone[i][0], name))
            assert torch.equal(cut[i][1], alone[i][1]) and torch.equal(cut[i][2], alone[i][2]) and torch.equal(got[i], alone_out[i])
