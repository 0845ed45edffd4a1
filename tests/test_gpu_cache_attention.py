"""Head rotation, prompt attention, 4-bit cache pages (append, attention, weights, eviction) against 64-bit arithmetic."""
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


def _starts(counts, gap=0):
    return np.concatenate([[gap], gap + np.cumsum(counts)]).astype(int).tolist()


# ------------------------------------------------------------------ rotation
@pytest.mark.parametrize("rows,heads,kv,d,rotary,interleaved,norm", [
    (1, 32, 8, 128, 128, False, True), (9, 32, 8, 128, 128, True, True), (130, 5, 5, 64, 64, False, True), (3, 3, 1, 256, 64, False, True),
    (7, 2, 1, 80, 48, True, False), (5, 1, 0, 16, 16, False, False), (65, 9, 3, 128, 0, False, True), (2050, 4, 2, 64, 32, True, True),
    (2, 40, 8, 96, 96, False, True), (4100, 12, 4, 128, 128, False, True),
])
def test_rotate(rows, heads, kv, d, rotary, interleaved, norm):
    q, k = _normal(1, rows, heads, d), _normal(2, rows, max(kv, 1), d)
    rng = np.random.default_rng(3)
    pos = rng.integers(0, 1 << 20, rows).astype(np.int32)
    pos[0] = 2 ** 31 - 1
    pos[-1] = -5
    freq = (10000.0 ** -(np.arange(rotary // 2) / max(1, rotary // 2))).astype(np.float32) if rotary else None
    wq, wk = (_normal(4, d), _normal(5, d)) if norm else (None, None)
    on = lambda x: None if x is None else torch.as_tensor(x).to(DEV)
    q[rows // 2] = 0
    got = binding.polyspec_rotate_heads(on(q), on(k) if kv else None, on(pos) if rotary else None, on(freq), on(wq), on(wk), interleaved=interleaved)
    for y, x, w in ((got[0], q, wq), (got[1], k, wk)):
        if y is not None:
            _close(y, *plain.rotate(x.float().numpy(), None if w is None else w.float().numpy(), pos, freq, interleaved))
    assert (got[1] is None) == (kv == 0)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_in_place_in_a_projection(interleaved):
    rows, heads, kv, d = 37, 6, 2, 64
    qkv = _normal(6, rows, heads + 2 * kv, d)
    pos, freq = np.arange(rows, dtype=np.int32) * 1000, (500000.0 ** -(np.arange(32) / 32)).astype(np.float32)
    w = _normal(7, d)
    on = qkv.to(DEV)
    q, k, v = on.split([heads, kv, kv], 1)
    binding.polyspec_rotate_heads(q, k, torch.from_numpy(pos).to(DEV), torch.from_numpy(freq).to(DEV), w.to(DEV), None, interleaved=interleaved, q_out=q, k_out=k)
    x = qkv.float().numpy()
    _close(on[:, :heads], *plain.rotate(x[:, :heads], w.float().numpy(), pos, freq, interleaved))
    _close(on[:, heads:heads + kv], *plain.rotate(x[:, heads:heads + kv], None, pos, freq, interleaved))
    assert torch.equal(on[:, heads + kv:].cpu(), qkv[:, heads + kv:])


def test_rotate_keeps_a_nan_in_its_head():
    q = _normal(8, 4, 3, 64)
    q[1, 2, 5] = float("nan")
    q[2, 0, 7] = float("inf")
    pos, freq = torch.zeros(4, dtype=torch.int32), torch.ones(32)
    got, _ = binding.polyspec_rotate_heads(q.to(DEV), None, pos.to(DEV), freq.to(DEV), _normal(9, 64).to(DEV))
    broken = torch.isnan(got).any(-1).cpu()
    assert broken[1, 2] and broken[2, 0] and int(broken.sum()) == 2


# ------------------------------------------------------------------ append
def _append_case(lens, counts, kv, d, P, seed, gap=0):
    """Rows that fill the last counts[b] slots of each sequence, and the pool before and after."""
    c = plain.Cache(lens, kv, d, P, seed)
    at = _starts(counts, gap)
    rows = at[-1] + gap
    x = [_normal(seed + 1 + p, max(1, rows), kv, d) for p in range(2)]
    pool = c.empty_pool()
    return c, at, rows, x, pool


@pytest.mark.parametrize("lens,counts,kv,d,P", [
    ([1], [1], 1, 64, 8), ([9, 40, 16], [9, 3, 0], 8, 128, 16), ([100, 7, 64, 33], [5, 7, 17, 1], 3, 64, 24), ([700], [700], 2, 128, 64),
    ([50] * 40, [9] * 40, 4, 128, 48), ([31, 5], [2, 1], 17, 64, 8),
])
def test_append(lens, counts, kv, d, P):
    c, at, rows, x, pool = _append_case(lens, counts, kv, d, P, 20)
    x[0][at[0], 0] = 3.5                                    # one value throughout: scale 1, code 0
    x[1][at[-1] - 1, kv - 1, d - 1] = float("nan")
    x[0][at[-1] - 1, 0, 0] = float("inf")
    pages, on = c.to(DEV), c.words_on(pool, DEV)
    weights = torch.full((len(lens), c.cap), 7.0, device=DEV)
    held = [torch.full((rows, kv, d), -1.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    base = [n - k for n, k in zip(lens, counts)]
    st = binding.polyspec_cache_append(pages, x[0].to(DEV), x[1].to(DEV), on, _i32(at), _i32(base), k_held=held[0], v_held=held[1], weights=weights)
    assert int(st) == 0
    want_w = np.full((len(lens), c.cap), 7.0)
    for p in range(2):
        code, scale, offset, back = plain.quantise(x[p].float().numpy())
        for b, n in enumerate(counts):
            c.put(pool, p, b, range(base[b], base[b] + n), code[at[b]:at[b] + n], scale[at[b]:at[b] + n], offset[at[b]:at[b] + n])
            want_w[b, base[b]:base[b] + n] = 0
        got = held[p].float().cpu().numpy()
        assert ((got == back) | (np.isnan(got) & np.isnan(back))).all()
    assert (on.cpu().numpy().view(np.uint32).reshape(pool.shape) == pool).all()
    assert (weights.cpu().numpy() == want_w).all()


def test_append_of_numbers_in_the_middle_between_codes_and_of_all_sizes():
    # whole numbers times powers of two: many quotients lie in the very middle, the smallest scales are the smallest normal number
    n, kv, d, P = 700, 3, 128, 16
    rng = np.random.default_rng(23)
    c = plain.Cache([n], kv, d, P, 24)
    x = [torch.from_numpy(np.ldexp(rng.integers(-(2 ** rng.integers(1, 8, (n, kv, 1))), 2 ** rng.integers(1, 8, (n, kv, 1)) + 1, (n, kv, d)).astype(np.float32),
                                   rng.integers(-126, 112, (n, kv, 1))).astype(np.float32)).to(torch.bfloat16) for _ in range(2)]
    pool = c.empty_pool()
    pages, on = c.to(DEV), c.words_on(pool, DEV)
    st = binding.polyspec_cache_append(pages, x[0].to(DEV), x[1].to(DEV), on, _i32([0, n]), _i32([0]))
    assert int(st) == 0
    for p in range(2):
        code, scale, offset, _ = plain.quantise(x[p].float().numpy())
        c.put(pool, p, 0, range(n), code, scale, offset)
    assert (on.cpu().numpy().view(np.uint32).reshape(pool.shape) == pool).all()


def test_append_takes_a_padded_batch_and_parts_of_a_projection():
    """n_rows below the rows given; base in two parts; rows before the first and behind the last sequence; strided rows."""
    lens, counts, kv, d, P = [30, 8, 21], [5, 5, 5], 2, 128, 16
    c, at, rows, _, pool = _append_case(lens, counts, kv, d, P, 30, gap=2)
    n_rows = [5, 0, 3]
    qkv = _normal(31, rows, 4 * kv, d)
    pages, on = c.to(DEV), c.words_on(pool, DEV)
    parts = qkv.to(DEV).split([2 * kv, kv, kv], 1)
    held = torch.full((rows, kv, d), -1.0, dtype=torch.bfloat16, device=DEV)
    base = [n - k for n, k in zip(lens, n_rows)]
    st = binding.polyspec_cache_append(pages, parts[1], parts[2], on, _i32(at), _i32(x - 2 for x in base), extra=_i32([2, 2, 2]), n_rows=_i32(n_rows), v_held=held)
    assert int(st) == 0
    for p in range(2):
        code, scale, offset, back = plain.quantise(qkv[:, (2 + p) * kv:(3 + p) * kv].float().numpy())
        for b, n in enumerate(n_rows):
            c.put(pool, p, b, range(base[b], base[b] + n), code[at[b]:at[b] + n], scale[at[b]:at[b] + n], offset[at[b]:at[b] + n])
    assert (on.cpu().numpy().view(np.uint32).reshape(pool.shape) == pool).all()
    written = np.zeros(rows, bool)
    for b, n in enumerate(n_rows):
        written[at[b]:at[b] + n] = True
    assert ((held.float().cpu().numpy() == -1).all((1, 2)) == ~written).all()


def test_append_leaves_what_was_not_granted_and_shared_pages():
    lens, counts, kv, d, P = [20, 16, 9], [6, 4, 3], 2, 64, 8
    c, at, rows, x, pool = _append_case(lens, counts, kv, d, P, 40)
    base = [18, 12, 6]                                      # four rows of the first are past its length
    c.refs[c.table[1, 1]] = 2                               # the second's last page is held by another
    pages, on = c.to(DEV), c.words_on(pool, DEV)
    st = binding.polyspec_cache_append(pages, x[0].to(DEV), x[1].to(DEV), on, _i32(at), _i32(base))
    assert int(st) == BAD
    for p in range(2):
        code, scale, offset, _ = plain.quantise(x[p].float().numpy())
        for b, n in ((0, 2), (2, 3)):
            c.put(pool, p, b, range(base[b], base[b] + n), code[at[b]:at[b] + n], scale[at[b]:at[b] + n], offset[at[b]:at[b] + n])
    assert (on.cpu().numpy().view(np.uint32).reshape(pool.shape) == pool).all()


@pytest.mark.parametrize("rows_at,base,n_rows", [
    ([0, 4, 2, 9], [0, 0, 0], None), ([-1, 3, 6, 9], [0, 0, 0], None), ([0, 3, 6, 20], [0, 0, 0], None), ([0, 3, 6, 9], [0, -4, 0], None),
    ([0, 3, 6, 9], [0, 0, 0], [3, 4, 3]), ([0, 3, 6, 9], [0, 0, 0], [3, -1, 3]), ([0, 3, 6, 9], [0, 2 ** 31 - 1, 0], None),
])
def test_numbers_that_make_no_sense_are_reported(rows_at, base, n_rows):
    c = plain.Cache([9, 9, 9], 2, 64, 8, 50)
    pages, pool = c.to(DEV), c.pool()
    on = c.words_on(pool, DEV)
    x = _normal(51, 9, 2, 64).to(DEV)
    n_rows = None if n_rows is None else _i32(n_rows)
    before = on.clone()
    assert int(binding.polyspec_cache_append(pages, x, x, on, _i32(rows_at), _i32(base), n_rows=n_rows)) == BAD
    on.copy_(before)
    out, lse, st = binding.polyspec_cache_attention(pages, x, on, 2, _i32(rows_at), _i32(base), n_rows=n_rows, lse=torch.zeros((9, 2), device=DEV))
    assert int(st) == BAD and not torch.isnan(out[:1]).any()
    w = torch.zeros((3, c.cap), device=DEV)
    assert int(binding.polyspec_cache_weigh(pages, x, on, 2, _i32(rows_at), _i32(base), lse, w, n_rows=n_rows)) == BAD


# ------------------------------------------------------------------ attention and weights
CASES = [  # lens (after the block), counts, heads, kv, d, P
    ([1], [1], 1, 1, 64, 8), ([1], [1], 1, 1, 128, 8), ([17], [1], 8, 2, 128, 16), ([8, 300, 16, 129], [1, 1, 1, 1], 32, 8, 128, 16),
    ([40, 7, 260, 131], [9, 7, 3, 1], 8, 2, 128, 24), ([40, 7, 260, 131], [9, 7, 3, 1], 12, 4, 64, 48), ([2000], [1], 4, 1, 128, 64),
    ([3000, 5], [2, 5], 5, 1, 64, 32), ([500, 0, 33, 64], [33, 0, 33, 1], 7, 7, 128, 8), ([90], [70], 16, 2, 64, 8), ([1300], [12], 8, 1, 128, 40),
    ([25] * 70, [2] * 70, 4, 2, 64, 16), ([7000, 1, 450], [1, 1, 1], 3, 3, 128, 16),
]


@pytest.mark.parametrize("lens,counts,heads,kv,d,P", CASES)
def test_attention_and_weights(lens, counts, heads, kv, d, P):
    c = plain.Cache(lens, kv, d, P, 60, max_tokens=max(lens) + 100)
    at = _starts(counts)
    q = _normal(61, at[-1], heads, d) * 2
    base = [n - k for n, k in zip(lens, counts)]
    pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
    lse = torch.zeros((at[-1], heads), device=DEV)
    out, _, st = binding.polyspec_cache_attention(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse=lse)
    want, want_lse, tol, tol_lse, weights, tol_w = plain.attend(c, q.float().numpy(), at, base)
    _close(out, want, tol)
    _close(lse, want_lse, tol_lse)
    assert int(st) == 0
    w = torch.full((len(lens), c.cap), 2.0, device=DEV)
    st = binding.polyspec_cache_weigh(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse, w, keep=0.5)
    assert int(st) == 0
    for b, n in enumerate(lens):
        _close(w[b, :n], 1.0 + weights[b], tol_w[b] + 4 * plain.U32 * (1 + weights[b]))
        assert (w[b, n:] == 2).all()
    # only the rows that were accepted count
    some = [k // 2 for k in counts]
    w.zero_()
    binding.polyspec_cache_weigh(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse, w, n_rows=_i32(some))
    _, _, _, _, weights, tol_w = plain.attend(c, q.float().numpy(), at, base, n_rows=some)
    for b, n in enumerate(lens):
        _close(w[b, :n], weights[b], tol_w[b] + 4 * plain.U32 * (1 + weights[b]))


def test_attention_of_a_padded_batch_and_strided_rows():
    lens, counts, heads, kv, d, P = [50, 20, 200], [6, 6, 6], 8, 2, 128, 16
    n_rows = [6, 0, 2]
    c = plain.Cache(lens, kv, d, P, 70)
    at = _starts(counts, 3)
    rows = at[-1] + 2
    qkv = (_normal(71, rows, heads + 2 * kv, d)).to(DEV)
    base = [n - k for n, k in zip(lens, n_rows)]
    pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
    out = torch.full((rows, heads, d), 9.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((rows, heads), 9.0, device=DEV)
    q = qkv[:, :heads]
    _, _, st = binding.polyspec_cache_attention(pages, q, on, kv, _i32(at), _i32(b - 1 for b in base), extra=_i32([1, 1, 1]), n_rows=_i32(n_rows), out=out,
                                                lse=lse, scale=0.3)
    assert int(st) == 0
    want, want_lse, tol, tol_lse, _, _ = plain.attend(c, q.float().cpu().numpy(), at, base, n_rows, scale=0.3)
    mine = ~np.isnan(want_lse[:, 0])
    _close(out[torch.from_numpy(mine)], want[mine], tol[mine])
    _close(lse[torch.from_numpy(mine)], want_lse[mine], tol_lse[mine])
    assert mine.sum() == 8 and (out[torch.from_numpy(~mine)] == 9).all() and (lse[torch.from_numpy(~mine)] == 9).all()


def test_attention_of_rows_that_were_not_granted_gives_zeros():
    lens, counts, heads, kv, d, P = [20, 3, 64], [4, 2, 3], 4, 2, 64, 8
    base = [18, 7, 61]
    c = plain.Cache(lens, kv, d, P, 80)
    at = _starts(counts)
    q = _normal(81, at[-1], heads, d)
    pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
    lse = torch.zeros((at[-1], heads), device=DEV)
    out, _, st = binding.polyspec_cache_attention(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse=lse)
    assert int(st) == BAD
    want, want_lse, tol, tol_lse, weights, tol_w = plain.attend(c, q.float().numpy(), at, base)
    _close(out, want, tol)
    _close(lse, want_lse, tol_lse)
    w = torch.zeros((3, c.cap), device=DEV)
    assert int(binding.polyspec_cache_weigh(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse, w)) == BAD
    for b, n in enumerate(lens):
        _close(w[b, :n], weights[b], tol_w[b])


@pytest.mark.parametrize("heads,kv,counts", [(4, 4, [1, 5]), (16, 2, [5, 5])])
def test_what_a_row_does_not_see_never_reaches_it(heads, kv, counts):
    """NaN scales and offsets in later rows of the block, NaN queries in other rows: only their own rows are broken."""
    lens, d, P = [45, 130], 128, 16
    c = plain.Cache(lens, kv, d, P, 90)
    at, base = _starts(counts), [n - k for n, k in zip(lens, counts)]
    q = _normal(91, at[-1], heads, d)
    q[at[1] + 1] = float("nan")
    for p in range(2):
        c.scale[p][1][base[1] + 3] = np.nan
        c.offset[p][1][base[1] + 3] = np.nan
    pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
    out, _, st = binding.polyspec_cache_attention(pages, q.to(DEV), on, kv, _i32(at), _i32(base))
    assert int(st) == 0
    broken = torch.isnan(out).all(-1).all(-1).tolist()
    assert torch.isnan(out).any(-1).any(-1).tolist() == broken == [i == at[1] + 1 or i >= at[1] + 3 for i in range(at[-1])]
    whole = plain.Cache(lens, kv, d, P, 90)
    want, _, tol, _, _, _ = plain.attend(whole, np.nan_to_num(q.float().numpy()), at, base)
    good = [i for i, x in enumerate(broken) if not x]
    _close(out[good], want[good], tol[good])


def test_attention_with_scores_far_apart_and_offsets_that_cancel():
    """One token far above all others, at any place; scales over five orders of magnitude; queries of zero."""
    lens, heads, kv, d, P = [400], 4, 1, 128, 16
    for peak in (0, 15, 16, 200, 399):
        c = plain.Cache(lens, kv, d, P, 100 + peak, scale=(0.01, 0.02))
        c.scale[1][0][:] = plain.bf16(10.0 ** c.rng.uniform(-4, 1, c.scale[1][0].shape))
        c.offset[1][0][:] = plain.bf16(c.scale[1][0] * -7.0)
        q = _normal(101, 1, heads, d)
        c.codes[0][0][peak, 0] = np.where(q[0, 0].float().numpy() > 0, 15, 0)
        c.scale[0][0][peak, 0] = 8.0
        c.offset[0][0][peak, 0] = -60.0
        q[0, 3] = 0
        pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
        lse = torch.zeros((1, heads), device=DEV)
        out, _, st = binding.polyspec_cache_attention(pages, q.to(DEV), on, kv, _i32([0, 1]), _i32([399]), lse=lse)
        want, want_lse, tol, tol_lse, _, _ = plain.attend(c, q.float().numpy(), [0, 1], [399])
        _close(out, want, tol)
        _close(lse, want_lse, tol_lse)


def test_attention_is_the_same_every_time_and_captured():
    lens, counts, heads, kv, d, P = [3000, 40, 700], [5, 5, 5], 8, 2, 128, 16
    c = plain.Cache(lens, kv, d, P, 110)
    at, base = _i32(_starts(counts)), _i32(n - k for n, k in zip(lens, counts))
    q = _normal(111, 15, heads, d).to(DEV)
    pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
    lse = torch.zeros((15, heads), device=DEV)
    first = binding.polyspec_cache_attention(pages, q, on, kv, at, base, lse=lse)[0].clone()
    first_lse = lse.clone()
    graphs = []
    for _ in range(2):                                      # two graphs, each with a workspace of its own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = binding.polyspec_cache_attention(pages, q, on, kv, at, base, lse=lse)[0]
        graphs.append((graph, out))
    for graph, out in graphs + graphs:
        out.zero_()
        lse.zero_()
        graph.replay()
        assert torch.equal(out, first) and torch.equal(lse, first_lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = binding.polyspec_cache_attention(pages, q, on, kv, at, base, stream=side)[0]
    side.synchronize()
    assert torch.equal(out, first)


def test_a_page_that_cannot_be_read_is_left_out_and_reported():
    lens, heads, kv, d, P = [100], 4, 2, 128, 16
    c = plain.Cache(lens, kv, d, P, 120)
    q = _normal(121, 1, heads, d)
    good = c.to(DEV)
    on = c.words_on(c.pool(), DEV)
    good.table[0, 2] = c.n_pages + 7
    good.table[0, 4] = -3
    out, _, st = binding.polyspec_cache_attention(good, q.to(DEV), on, kv, _i32([0, 1]), _i32([99]))
    assert int(st) == BAD
    keep = [j for j in range(100) if j // P not in (2, 4)]
    for p in range(2):
        c.codes[p][0], c.scale[p][0], c.offset[p][0] = c.codes[p][0][keep], c.scale[p][0][keep], c.offset[p][0][keep]
    c.lens = [len(keep)]
    want, _, tol, _, _, _ = plain.attend(c, q.float().numpy(), [0, 1], [len(keep) - 1])
    _close(out, want, tol)


# ------------------------------------------------------------------ eviction
@pytest.mark.parametrize("lens,budget,first,recent,kv,d,P,planes", [
    ([1], [0], 0, 0, 1, 64, 8, 2), ([30, 9, 100], [10, 9, 99], 2, 3, 2, 128, 8, 2), ([300, 4, 0, 77], [40, 2, 5, -1], 0, 0, 1, 64, 16, 4),
    ([700, 650], [300, 650], 4, 128, 4, 128, 48, 4), ([5000], [1], 0, 1, 1, 64, 64, 2), ([2100, 1500, 1024], [1024, 1024, 1024], 4, 64, 3, 64, 32, 2),
    ([260], [259], 0, 259, 8, 128, 16, 2), ([600], [300], 300, 0, 2, 64, 8, 2),
])
@pytest.mark.parametrize("kind", ["random", "ties", "odd"])
def test_evict(lens, budget, first, recent, kv, d, P, planes, kind):
    c = plain.Cache(lens, kv, d, P, 130, max_tokens=max(lens) + 40)
    rng = np.random.default_rng(131)
    B = len(lens)
    w = rng.random((B, c.cap)).astype(np.float32) ** 4
    if kind == "ties":
        w = rng.integers(0, 3, (B, c.cap)).astype(np.float32)
    if kind == "odd":
        w = rng.standard_normal((B, c.cap)).astype(np.float32)
        w[:, ::7], w[:, 1::11], w[:, 2::13], w[:, 3::17], w[:, 4::19] = np.nan, np.inf, -np.inf, 0.0, -0.0
    pages, pool = c.to(DEV), c.pool(planes)
    on, won = c.words_on(pool, DEV), torch.from_numpy(w.copy()).to(DEV)
    kept_from = torch.full((B, c.cap), 5, dtype=torch.int32, device=DEV)
    st = binding.polyspec_cache_evict(pages, _i32(budget), won, on, kv, d, first=first, recent=recent, kept_from=kept_from)
    bad = False
    want_from = np.full((B, c.cap), -1)
    new_len, new_table, refs = list(lens), c.table.copy(), c.refs.copy()
    for b in range(B):
        keep = plain.evict_slots(w[b], lens[b], budget[b], first, recent)
        bad |= keep == "bad"
        if keep is None or keep == "bad":
            continue
        moved = [i for i, j in enumerate(keep) if i != j]
        old = [keep[i] for i in moved]
        for p in range(planes):
            c.put(pool, p, b, moved, c.codes[p % 2][b][old], c.scale[p % 2][b][old], c.offset[p % 2][b][old])
        w[b, : len(keep)] = w[b, keep]
        want_from[b, : len(keep)] = keep
        new_len[b] = len(keep)
        for i in range(-(-len(keep) // P), -(-lens[b] // P)):
            refs[new_table[b, i]] -= 1
            new_table[b, i] = -1
    assert int(st) == (BAD if bad else 0)
    assert pages.len.tolist() == new_len
    assert (kept_from.cpu().numpy() == want_from).all()
    assert (won.cpu().numpy().view(np.uint32) == w.view(np.uint32)).all()
    assert (pages.table.cpu().numpy() == new_table).all() and (pages.refs.cpu().numpy() == refs).all()
    c.refs = refs
    assert (pages.free_bits.cpu().numpy() == c.free_bits()).all()
    assert (on.cpu().numpy().view(np.uint32).reshape(pool.shape) == pool).all()


def test_evict_leaves_sequences_whose_pages_others_hold():
    lens, kv, d, P = [64, 64, 64], 2, 64, 8
    c = plain.Cache(lens, kv, d, P, 140)
    w = np.tile(np.arange(c.cap, dtype=np.float32)[::-1], (3, 1)).copy()        # the first tokens are the heaviest
    c.refs[c.table[0, 3]] = 2                               # before the first slot that changes: none of its business
    c.refs[c.table[1, 5]] = 2
    w[:, 44:] += 1000                                       # slots 0 .. 35 and 44 .. 63 stay of a budget of 56
    pages, pool = c.to(DEV), c.pool()
    on = c.words_on(pool, DEV)
    st = binding.polyspec_cache_evict(pages, _i32([56, 56, 64]), torch.from_numpy(w).to(DEV), on, kv, d)
    assert int(st) == BAD
    assert pages.len.tolist() == [56, 64, 64]
    for p in range(2):
        old = list(range(44, 64))
        c.put(pool, p, 0, range(36, 56), c.codes[p][0][old], c.scale[p][0][old], c.offset[p][0][old])
    assert (on.cpu().numpy().view(np.uint32).reshape(pool.shape) == pool).all()


def test_evict_of_two_holders_of_a_page_at_once():
    # a page that changes in sequence 2 k lies behind what sequence 2 k + 1 keeps, and some of what that keeps comes from it: whichever is looked at
    # first, the page has two holders, 2 k stays as it was
    pairs, kv, d, P = 100, 2, 64, 8
    c = plain.Cache([64] * (2 * pairs), kv, d, P, 145)
    w = np.zeros((2 * pairs, c.cap), np.float32)
    for b in range(0, 2 * pairs, 2):
        c.refs[c.table[b, 5]] = 0
        c.table[b, 5] = c.table[b + 1, 7]
        c.refs[c.table[b, 5]] = 2
        for p in range(2):
            for x in (c.codes, c.scale, c.offset):
                x[p][b][40:48] = x[p][b + 1][56:64]
        w[b, :36], w[b, 44:64] = 1, 1                       # of a budget of 56; slots 36 .. change
        w[b + 1, :8], w[b + 1, 40:64] = 1, 1                # of a budget of 32; slots 8 .. change
    pages, pool = c.to(DEV), c.pool()
    on = c.words_on(pool, DEV)
    st = binding.polyspec_cache_evict(pages, _i32([56, 32] * pairs), torch.from_numpy(w).to(DEV), on, kv, d)
    assert int(st) == BAD
    assert pages.len.tolist() == [64, 32] * pairs
    for b in range(1, 2 * pairs, 2):
        for p in range(2):
            c.put(pool, p, b, range(8, 32), c.codes[p][b][40:64], c.scale[p][b][40:64], c.offset[p][b][40:64])
        c.refs[c.table[b, 4:8]] -= 1
        c.table[b, 4:8] = -1
    assert (pages.table.cpu().numpy() == c.table).all() and (pages.refs.cpu().numpy() == c.refs).all()
    assert (pages.free_bits.cpu().numpy() == c.free_bits()).all()
    assert (on.cpu().numpy().view(np.uint32).reshape(pool.shape) == pool).all()


# ------------------------------------------------------------------ prompts
@pytest.mark.parametrize("lens,heads,kv,d", [
    ([1], 1, 1, 64), ([1, 2, 3], 4, 2, 128), ([127, 128, 129], 2, 1, 128), ([300, 0, 5], 3, 3, 64), ([513], 6, 2, 128), ([64, 65, 63, 255, 257], 8, 2, 64),
    ([1000], 2, 1, 128), ([31] * 20, 5, 1, 64), ([384, 640], 1, 1, 128), ([700], 7, 7, 64),
])
def test_prompt(lens, heads, kv, d):
    at = _starts(lens, 3)
    rows = at[-1] + 2
    qkv = _normal(150, rows, heads + 2 * kv, d).to(DEV)
    q, k, v = qkv.split([heads, kv, kv], 1)
    q *= 2
    out = torch.full((rows, heads, d), 9.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((rows, heads), 9.0, device=DEV)
    _, _, st = binding.polyspec_prompt_attention(q, k, v, _i32(at), out=out, lse=lse)
    assert int(st) == 0
    want, want_lse, tol, tol_lse = plain.prompt(*(x.float().cpu().numpy() for x in (q, k, v)), at)
    mine = ~np.isnan(want_lse[:, 0])
    _close(out[torch.from_numpy(mine)], want[mine], tol[mine])
    _close(lse[torch.from_numpy(mine)], want_lse[mine], tol_lse[mine])
    assert (out[torch.from_numpy(~mine)] == 9).all() and (lse[torch.from_numpy(~mine)] == 9).all()


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_later_and_other_rows_never_reach_a_row(d):
    """NaN and infinities in keys and values behind a row, in other prompts and in rows of no prompt."""
    lens, heads, kv = [150, 200], 4, 2
    at = _starts(lens, 1)
    rows = at[-1] + 130
    q, k, v = _normal(160, rows, heads, d), _normal(161, rows, kv, d), _normal(162, rows, kv, d)
    want, _, tol, _ = plain.prompt(*(x.float().numpy() for x in (q, k, v)), at)
    k[0], v[0], q[0] = float("nan"), float("inf"), float("nan")
    k[at[-1]:], v[at[-1]:], q[at[-1]:] = float("nan"), float("nan"), float("inf")
    k[at[1] + 60:at[2]], v[at[1] + 60:at[2]] = float("nan"), float("inf")
    v[at[0] + 140, 1, 3] = float("-inf")
    v[at[0] + 145, 0, 5] = float("nan")
    out, _, st = binding.polyspec_prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), _i32(at))
    assert int(st) == 0
    good = list(range(at[0], at[0] + 140)) + list(range(at[1], at[1] + 60))
    _close(out[good], want[good], tol[good])
    assert torch.isnan(out[at[1] + 60:at[2]]).all()
    late = out[at[0] + 140:at[1]].cpu().float()
    assert (late[:, 2:, 3] == float("-inf")).all() and torch.isfinite(late[:, 2:, [0, 1, 2, 4, 5]]).all()
    assert torch.isnan(late[5:, :2, 5]).all() and torch.isfinite(late[:5, :2]).all() and torch.isfinite(late[5:, :2, :5]).all()


def test_prompt_scores_far_apart():
    lens, heads, kv, d = [300], 2, 2, 128
    q, k, v = _normal(170, 300, heads, d), _normal(171, 300, kv, d), _normal(172, 300, kv, d)
    k[5] = q[200] * 40
    k[250, 1] = q[260, 1] * 80
    lse = torch.zeros((300, heads), device=DEV)
    out, _, _ = binding.polyspec_prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), _i32([0, 300]), lse=lse)
    want, want_lse, tol, tol_lse = plain.prompt(*(x.float().numpy() for x in (q, k, v)), [0, 300])
    _close(out, want, tol)
    _close(lse, want_lse, tol_lse)


def test_prompt_bad_row_numbers():
    q = _normal(180, 20, 2, 64).to(DEV)
    for at in ([0, 30], [-1, 10], [5, 3, 20], [0, 2 ** 31 - 1]):
        out, _, st = binding.polyspec_prompt_attention(q, q, q, _i32(at))
        assert int(st) == BAD
    out = torch.full((20, 2, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    _, _, st = binding.polyspec_prompt_attention(q, q, q, _i32([4, 4, 4]), out=out)
    assert int(st) == 0 and (out == 9).all()


# ------------------------------------------------------------------ many sequences, several calls at once, one whole run
def test_more_sequences_than_a_block_has_threads():
    """The cursors over sequences go round more than once; every third sequence has no rows."""
    n, heads, kv, d, P = 700, 2, 1, 64, 8
    counts = [0 if b % 3 == 2 else 1 + b % 2 for b in range(n)]
    lens = [3 + b % 11 if c else b % 4 for b, c in enumerate(counts)]
    c = plain.Cache(lens, kv, d, P, 190)
    at, base = _starts(counts), [x - k for x, k in zip(lens, counts)]
    q = _normal(191, at[-1], heads, d)
    pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
    lse = torch.zeros((at[-1], heads), device=DEV)
    out, _, st = binding.polyspec_cache_attention(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse=lse)
    want, want_lse, tol, tol_lse, weights, tol_w = plain.attend(c, q.float().numpy(), at, base)
    _close(out, want, tol)
    _close(lse, want_lse, tol_lse)
    w = torch.zeros((n, c.cap), device=DEV)
    binding.polyspec_cache_weigh(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse, w)
    for b in range(n):
        _close(w[b, : lens[b]], weights[b], tol_w[b])
    assert int(st) == 0
    x = _normal(192, at[-1], kv, d)
    st = binding.polyspec_cache_append(pages, x.to(DEV), x.to(DEV), on, _i32(at), _i32(base))
    assert int(st) == 0
    pool = on.cpu().numpy().view(np.uint32).reshape(2, c.n_pages, kv, P // 8, d + 8)
    code, scale, offset, _ = plain.quantise(x.float().numpy())
    for p in range(2):
        want_pool = pool.copy()
        for b, k in enumerate(counts):
            c.put(want_pool, p, b, range(base[b], base[b] + k), code[at[b]:at[b] + k], scale[at[b]:at[b] + k], offset[at[b]:at[b] + k])
        assert (want_pool[p] == pool[p]).all()
    lens = [30 + 40 * (b % 5) for b in range(300)]
    at = _starts(lens)
    q, k, v = _normal(193, at[-1], 2, 64), _normal(194, at[-1], 1, 64), _normal(195, at[-1], 1, 64)
    out, _, st = binding.polyspec_prompt_attention(q.to(DEV), k.to(DEV), v.to(DEV), _i32(at))
    want, _, tol, _ = plain.prompt(*(x.float().numpy() for x in (q, k, v)), at)
    _close(out, want, tol)
    assert int(st) == 0


def test_a_page_larger_than_a_cache_and_wide_groups():
    """One page of 1024 tokens; 48 query heads on one key head, so that a sequence's rows fill several tiles."""
    lens, counts, heads, kv, P = [1000, 37], [3, 2], 48, 1, 1024
    for d in (64, 128):
        c = plain.Cache(lens, kv, d, P, 200)
        at, base = _starts(counts), [997, 35]
        q = _normal(201, 5, heads, d)
        lse = torch.zeros((5, heads), device=DEV)
        pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
        out, _, st = binding.polyspec_cache_attention(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse=lse)
        want, want_lse, tol, tol_lse, weights, tol_w = plain.attend(c, q.float().numpy(), at, base)
        _close(out, want, tol)
        _close(lse, want_lse, tol_lse)
        w = torch.zeros((2, c.cap), device=DEV)
        binding.polyspec_cache_weigh(pages, q.to(DEV), on, kv, _i32(at), _i32(base), lse, w)
        for b in range(2):
            _close(w[b, : lens[b]], weights[b], tol_w[b])


def test_two_calls_at_once_on_two_streams():
    """Attention of two layers, prompts and evictions side by side: nothing is shared between calls but what they are given."""
    lens, counts, heads, kv, d, P = [900, 300], [4, 4], 8, 2, 128, 16
    c = plain.Cache(lens, kv, d, P, 210)
    at, base = _i32(_starts(counts)), _i32(n - k for n, k in zip(lens, counts))
    pages, on = c.to(DEV), c.words_on(c.pool(4), DEV)
    q = [_normal(211 + i, 8, heads, d).to(DEV) for i in range(2)]
    prompt = _normal(213, 500, 4, 128).to(DEV)
    ends = _i32([0, 300, 500])
    alone = [binding.polyspec_cache_attention(pages, q[i], on[2 * i:2 * i + 2], kv, at, base)[0].clone() for i in range(2)]
    alone_prompt = binding.polyspec_prompt_attention(prompt, prompt, prompt, ends)[0].clone()
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got.append(binding.polyspec_cache_attention(pages, q[i], on[2 * i:2 * i + 2], kv, at, base)[0])
        with torch.cuda.stream(streams[2]):
            got.append(binding.polyspec_prompt_attention(prompt, prompt, prompt, ends)[0])
        torch.cuda.synchronize()
        assert torch.equal(got[0], alone[0]) and torch.equal(got[1], alone[1]) and torch.equal(got[2], alone_prompt)


def test_front_end_refuses_layouts_it_cannot_take():
    c = plain.Cache([9], 2, 64, 8, 220)
    pages, on = c.to(DEV), c.words_on(c.pool(), DEV)
    x = torch.zeros((9, 2, 64), dtype=torch.bfloat16, device=DEV)
    at, base = _i32([0, 9]), _i32([0])
    with pytest.raises(ValueError):
        binding.polyspec_cache_append(pages, x.transpose(0, 1), x, on, at, base)
    with pytest.raises(ValueError):
        binding.polyspec_cache_append(pages, x[:, :, ::2], x[:, :, ::2], on, at, base)
    with pytest.raises(ValueError):
        binding.polyspec_cache_append(pages, x, x, on[:1], at, base)
    with pytest.raises(ValueError):
        binding.polyspec_cache_attention(pages, x, on[:, :, :100], 2, at, base)
    with pytest.raises(ValueError):
        binding.polyspec_cache_attention(pages, x, on, 2, _i32([0, 3, 9]), base)
    with pytest.raises(TypeError):
        binding.polyspec_cache_attention(pages, x, on, 2, at.long(), base)
    with pytest.raises(TypeError):
        binding.polyspec_cache_weigh(pages, x, on, 2, at, base, torch.zeros((9, 2), device=DEV).double(), torch.zeros((1, c.cap), device=DEV))
    with pytest.raises(ValueError):
        binding.polyspec_cache_evict(pages, _i32([4]), torch.zeros((1, c.cap + 8), device=DEV), on, 2, 64)
    with pytest.raises(ValueError):
        binding.polyspec_prompt_attention(x, x, x, _i32([0]))
    with pytest.raises(ValueError):
        binding.polyspec_rotate_heads(x, None, None, torch.ones(32, device=DEV))
    with pytest.raises(binding.PolyspecError):
        binding.polyspec_rotate_heads(x[:, :, :8].contiguous(), None, None, None)


class Run:
    """A model's layer over a batch: prompts, then blocks of drafted tokens of which some are accepted, the cache kept to a budget."""

    def __init__(self, lens, heads, kv, d, P, seed):
        self.lens, self.heads, self.kv, self.d, self.P = lens, heads, kv, d, P
        self.rng = np.random.default_rng(seed)
        self.seed = seed
        B, most = len(lens), max(lens) + 80
        self.pages = binding.CachePages.new(B, -(-most // P), B * (-(-most // P)), P, DEV)
        self.pool = torch.zeros((2, self.pages.n_pages, binding.cache_page_bytes(kv, d, P)), dtype=torch.uint8, device=DEV)
        self.weights = torch.zeros((B, self.pages.max_pages * P), device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.freq = torch.from_numpy((10000.0 ** -(np.arange(d // 2) / (d // 2))).astype(np.float32)).to(DEV)
        self.norm = [(_normal(seed + i, d).float() * 0.1 + 1).to(torch.bfloat16).to(DEV) for i in range(2)]
        self.text = list(lens)                                          # positions: eviction does not move them
        # what the cache stands for, and the weights, in plain arrays
        self.codes = [[np.zeros((0, kv, d), int) for _ in lens] for _ in range(2)]
        self.scale = [[np.zeros((0, kv), np.float32) for _ in lens] for _ in range(2)]
        self.offset = [[np.zeros((0, kv), np.float32) for _ in lens] for _ in range(2)]
        self.w = [np.zeros(0) for _ in lens]

    def rows(self, counts):
        """A projection of new rows, rotated at their positions; the cache's room and its new tokens."""
        self.seed += 10
        H, K, d = self.heads, self.kv, self.d
        at = _starts(counts)
        qkv = _normal(self.seed, at[-1], H + 2 * K, d).to(DEV)
        q, k, v = qkv.split([H, K, K], 1)
        pos = np.concatenate([np.arange(t - n, t) for t, n in zip(self.text, counts)]).astype(np.int32)
        before = qkv.float().cpu().numpy()
        binding.polyspec_rotate_heads(q, k, torch.from_numpy(pos).to(DEV), self.freq, self.norm[0], self.norm[1], q_out=q, k_out=k)
        for x, part, w in ((q, before[:, :H], 0), (k, before[:, H:H + K], 1)):
            _close(x, *plain.rotate(part, self.norm[w].float().cpu().numpy(), pos, self.freq.cpu().numpy(), False))
        held = [len(x) for x in self.w]
        base = _i32(held)
        binding.polyspec_cache_reserve(self.pages, base, extra=_i32(counts), device_status=self.status)
        binding.polyspec_cache_append(self.pages, k, v, self.pool, _i32(at), base, weights=self.weights, device_status=self.status)
        for p, x in enumerate((k, v)):
            code, scale, offset, _ = plain.quantise(x.float().cpu().numpy())
            for b, n in enumerate(counts):
                s = slice(at[b], at[b] + n)
                for have, new in ((self.codes, code), (self.scale, scale), (self.offset, offset)):
                    have[p][b] = np.concatenate([have[p][b], new[s]])
        for b, n in enumerate(counts):
            self.w[b] = np.concatenate([self.w[b], np.zeros(n)])
        return at, q, k, v, held, base

    def cache(self):
        c = plain.Cache.__new__(plain.Cache)
        c.kv, c.d, c.P, c.lens = self.kv, self.d, self.P, [len(x) for x in self.w]
        c.codes, c.scale, c.offset = self.codes, self.scale, self.offset
        return c

    def prompt(self):
        at, q, k, v, _, _ = self.rows(self.lens)
        out, _, _ = binding.polyspec_prompt_attention(q, k, v, _i32(at), device_status=self.status)
        want, _, tol, _ = plain.prompt(*(x.float().cpu().numpy() for x in (q, k, v)), at)
        _close(out, want, tol)

    def block(self, counts):
        self.text = [t + n for t, n in zip(self.text, counts)]
        at, q, _, _, held, base = self.rows(counts)
        lse = torch.zeros((at[-1], self.heads), device=DEV)
        out, _, _ = binding.polyspec_cache_attention(self.pages, q, self.pool, self.kv, _i32(at), base, lse=lse, device_status=self.status)
        c, qn = self.cache(), q.float().cpu().numpy()
        want, want_lse, tol, tol_lse, _, _ = plain.attend(c, qn, at, held)
        _close(out, want, tol)
        _close(lse, want_lse, tol_lse)
        accepted = [int(self.rng.integers(0, n + 1)) for n in counts]
        kept = _i32(accepted)
        binding.polyspec_cache_weigh(self.pages, q, self.pool, self.kv, _i32(at), base, lse, self.weights, n_rows=kept, device_status=self.status)
        binding.polyspec_cache_rollback(self.pages, base, kept, device_status=self.status)
        _, _, _, _, more, tol_w = plain.attend(c, qn, at, held, n_rows=accepted)
        self.text = [t - n + a for t, n, a in zip(self.text, counts, accepted)]
        for b, a in enumerate(accepted):
            m = held[b] + a
            for have in (self.codes, self.scale, self.offset):
                for p in range(2):
                    have[p][b] = have[p][b][:m]
            _close(self.weights[b, :m], (self.w[b] + more[b])[:m], (tol_w[b] + 4 * plain.U32 * (self.w[b] + more[b]))[:m])
            self.w[b] = self.weights[b, :m].double().cpu().numpy()          # (the next comparison starts from what is there)

    def evict(self, budget):
        binding.polyspec_cache_evict(self.pages, _i32([budget] * len(self.lens)), self.weights, self.pool, self.kv, self.d, first=2, recent=8, device_status=self.status)
        for b in range(len(self.lens)):
            keep = plain.evict_slots(self.w[b].astype(np.float32), len(self.w[b]), budget, 2, 8)
            if keep is not None:
                self.w[b] = self.w[b][keep]
                for have in (self.codes, self.scale, self.offset):
                    for p in range(2):
                        have[p][b] = have[p][b][keep]
        assert self.pages.len.tolist() == [len(x) for x in self.w]


@pytest.mark.parametrize("lens,heads,kv,d,P", [([70, 33, 1], 4, 2, 64, 8), ([150, 40], 8, 2, 128, 16), ([130, 5, 64], 12, 4, 128, 24)])
def test_a_whole_run(lens, heads, kv, d, P):
    run = Run(lens, heads, kv, d, P, 300)
    run.prompt()
    for i in range(4):
        run.block([1 + (b + i) % 6 for b in range(len(lens))])
        if i % 2:
            run.evict(40)
    assert int(run.status) == 0
