"""The LM head with 4-bit weights against its 64-bit statement.

Tolerance per element: q - z is exact in bf16 and bf16 products are exact in fp32, so what is rounded are additions.  A group's
sum of G products takes at most G additions in any order, the sum over the groups one fused multiply-add each, each off by at
most 2^-23 (an addition inside the tensor core may truncate) of a partial sum that the sum of magnitudes bounds: (G + groups)
2^-23 sum |h| |w|.  A bf16 logit is rounded once more, by at most 2^-8 of its value."""
import threading

import pytest
import torch

from paper_2510_26527_b200 import binding, buildlib
from tests import plain_operators as plain
from tests.helpers import run_at_once

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _lib():
    buildlib.build()
    binding.load_library()
    assert torch.cuda.is_available()


def _case(rows, V, d, group, zeros, seed):
    g = torch.Generator().manual_seed(seed)
    hidden = torch.randn((rows, d), generator=g).to(torch.bfloat16)
    codes = torch.randint(0, 16, (V, d), generator=g, dtype=torch.uint8)
    scales = (torch.rand((V, d // group), generator=g) * 0.02 + 0.001).to(torch.bfloat16)
    zp = torch.randint(0, 16, (V, d // group), generator=g, dtype=torch.uint8) if zeros else None
    return hidden, codes, scales, zp


def _close(got, hidden, codes, scales, zp):
    ref, size = plain.head(hidden, codes, scales, zp)
    d = codes.shape[1]
    groups = scales.shape[1]
    tol = (d // groups + groups) * 2.0 ** -23 * size + 1e-30
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (ref.abs() + tol)
    err = (got.cpu().double() - ref).abs()
    worst = float((err / tol).max())
    assert worst <= 1.0, worst
    assert float(ref.abs().max()) > 0.01


def _to(*ts):
    return [None if t is None else t.to(DEV) for t in ts]


@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 15, 16, 17, 33, 64, 65, 100, 144, 193, 288, 300])
@pytest.mark.parametrize("V,d,group,zeros,dtype", [
    (257, 256, 128, True, torch.float32),
    (130, 96, 32, True, torch.bfloat16),
    (64, 192, 64, False, torch.float32),
])
def test_rows(rows, V, d, group, zeros, dtype):
    hidden, codes, scales, zp = _case(rows, V, d, group, zeros, rows * 7 + V)
    h, c, s, z = _to(hidden, codes, scales, zp)
    out, status = binding.polyspec_lm_head_quantized(h, binding.polyspec_pack_quantized(c), s, z, out_dtype=dtype)
    torch.cuda.synchronize()
    assert int(status) == 0 and out.dtype == dtype
    _close(out, hidden, codes, scales, zp)


@pytest.mark.parametrize("rows", [1, 9, 40])
@pytest.mark.parametrize("V,d,group", [
    (1, 32, 32), (1, 128, 128), (7, 64, 64), (31, 160, 32), (33, 128, 32), (127, 320, 64), (128, 384, 128), (129, 1152, 128),
    (1000, 2080, 32), (513, 4096, 128), (300, 8192, 64), (257, 16384, 128), (40, 12800, 32), (5000, 448, 64), (20001, 256, 32),
])
def test_shapes(rows, V, d, group):
    hidden, codes, scales, zp = _case(rows, V, d, group, V % 2 == 1, V + d)
    h, c, s, z = _to(hidden, codes, scales, zp)
    q = binding.polyspec_pack_quantized(c)
    out, status = binding.polyspec_lm_head_quantized(h, q, s, z)
    low, _ = binding.polyspec_lm_head_quantized(h, q, s, z, out_dtype=torch.bfloat16)
    torch.cuda.synchronize()
    assert int(status) == 0
    _close(out, hidden, codes, scales, zp)
    assert torch.equal(low, out.to(torch.bfloat16))


@pytest.mark.parametrize("rows,V,d,group", [(1, 3001, 1024, 128), (12, 3001, 1024, 64), (70, 3001, 1024, 128), (200, 3001, 1056, 32)])
def test_writes_nothing_else_and_repeats(rows, V, d, group):
    hidden, codes, scales, zp = _case(rows, V, d, group, True, 3)
    h, c, s, z = _to(hidden, codes, scales, zp)
    q = binding.polyspec_pack_quantized(c)
    room = torch.full((rows * V + 64,), -7.0, device=DEV)
    first = None
    for _ in range(3):
        out, _ = binding.polyspec_lm_head_quantized(h, q, s, z, out=room[: rows * V].view(rows, V))
        torch.cuda.synchronize()
        assert (room[rows * V:] == -7.0).all()
        assert first is None or torch.equal(first, out)
        first = out.clone()
    # slices of the vocabulary: the order in which a logit's partial sums are added depends on how the pieces fall to the
    # warps, so each slice is held to the same bound as the whole rather than to the whole's bits
    cut = 1504
    for a, b in ((0, cut), (cut, V)):
        part, _ = binding.polyspec_lm_head_quantized(h, q[a:b].contiguous(), s[a:b].contiguous(), z[a:b].contiguous())
        _close(part, hidden, codes[a:b], scales[a:b], zp[a:b])


def test_pack_layout_and_high_bits():
    codes = torch.arange(2 * 32, dtype=torch.uint8).view(2, 32)             # codes above 15: the low four bits count
    q = binding.polyspec_pack_quantized(codes.to(DEV)).cpu().numpy().view("uint32")
    for v in range(2):
        for k in range(32):
            e = k % 8
            assert (int(q[v, k // 8]) >> (4 * (e // 2) + 16 * (e % 2))) & 15 == int(codes[v, k]) & 15
    hidden, codes, scales, zp = _case(3, 40, 128, 32, True, 5)
    h, c, s, z = _to(hidden, codes, scales, zp)
    q = binding.polyspec_pack_quantized(c)
    a, _ = binding.polyspec_lm_head_quantized(h, q, s, z)
    b, _ = binding.polyspec_lm_head_quantized(h, q, s, z + 16)
    assert torch.equal(a, b)


@pytest.mark.parametrize("rows", [1, 20, 130])
def test_special_values_stay_in_their_rows_and_columns(rows):
    hidden, codes, scales, zp = _case(rows, 300, 256, 128, True, 11)
    hidden[0, 5] = float("inf")
    scales[17, 1] = float("nan")
    h, c, s, z = _to(hidden, codes, scales, zp)
    out, _ = binding.polyspec_lm_head_quantized(h, binding.polyspec_pack_quantized(c), s, z)
    out = out.cpu()
    assert out[:, 17].isnan().all()
    keep = torch.ones(300, dtype=torch.bool)
    keep[17] = False
    if rows > 1:
        ref, size = plain.head(hidden[1:], codes[keep], scales[keep], zp[keep])
        assert ((out[1:][:, keep].double() - ref).abs() <= (128 + 2) * 2.0 ** -23 * size).all()
    # inf * (q - z): +-inf by the sign of q - z, NaN where it is zero
    sign = (codes[:, 5].float() - zp[:, 0].float())
    assert torch.equal(out[0, keep & (sign > 0)], torch.full((int((keep & (sign > 0)).sum()),), float("inf")))
    assert out[0, keep & (sign == 0)].isnan().all()


@pytest.mark.parametrize("rows", [1, 36, 150])
def test_captured_and_on_another_stream(rows):
    hidden, codes, scales, zp = _case(rows, 2000, 512, 128, True, 21)
    h, c, s, z = _to(hidden, codes, scales, zp)
    q = binding.polyspec_pack_quantized(c)
    want, status = binding.polyspec_lm_head_quantized(h, q, s, z)
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.polyspec_lm_head_quantized(h, q, s, z, out=out, device_status=status)
    h2 = h.clone()
    h.mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want * 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _ = binding.polyspec_lm_head_quantized(h2, q, s, z, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("rows", [1, 5, 20, 150])
@pytest.mark.parametrize("zeros", [True, False])
def test_scales_and_zero_points_off_the_vector_boundary(rows, zeros):
    """Eight groups a row, so that only the address keeps the vector loads away: same bits as from an aligned copy."""
    hidden, codes, scales, zp = _case(rows, 300, 1024, 128, zeros, 31)
    h, c, s, z = _to(hidden, codes, scales, zp)
    q = binding.polyspec_pack_quantized(c)

    def off(t):
        if t is None:
            return None
        room = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
        room[1:] = t.flatten()
        return room[1:].view(t.shape)

    want, _ = binding.polyspec_lm_head_quantized(h, q, s, z)
    got, status = binding.polyspec_lm_head_quantized(h, q, off(s), off(z))
    torch.cuda.synchronize()
    assert int(status) == 0 and off(s).data_ptr() % 16 != 0
    _close(got, hidden, codes, scales, zp)
    assert torch.equal(got, want)


@pytest.mark.parametrize("rows", [4, 40, 200])
def test_two_calls_at_once_on_two_streams(rows):
    cases = [_case(rows, 9001, 1024, 128, True, 41 + i) for i in range(2)]
    args = []
    for hidden, codes, scales, zp in cases:
        h, c, s, z = _to(hidden, codes, scales, zp)
        args.append((h, binding.polyspec_pack_quantized(c), s, z))
    want = [binding.polyspec_lm_head_quantized(*a)[0] for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in args]
    got = [[] for _ in args]
    for _ in range(8):
        for i, (a, side) in enumerate(zip(args, streams)):
            got[i].append(binding.polyspec_lm_head_quantized(*a, stream=side))
    torch.cuda.synchronize()
    for outs, ref in zip(got, want):
        for out, status in outs:
            assert int(status) == 0 and torch.equal(out, ref)


def test_output_offsets_past_32_bits():
    """2.2 billion logits: the last rows are written where they belong, and nothing else is."""
    V, d, rows = 152064, 32, 14500
    hidden, codes, scales, zp = _case(rows, V, d, 32, True, 51)
    h, c, s, z = _to(hidden, codes, scales, zp)
    q = binding.polyspec_pack_quantized(c)
    out, status = binding.polyspec_lm_head_quantized(h, q, s, z, out_dtype=torch.bfloat16)
    torch.cuda.synchronize()
    assert int(status) == 0 and out.numel() > 1 << 31
    cols = torch.cat([torch.arange(200), torch.arange(V - 200, V)])
    for at in (0, 7000, rows - 30):
        part = out[at:at + 30][:, cols.to(DEV)]
        _close(part, hidden[at:at + 30], codes[cols], scales[cols], zp[cols])


@pytest.mark.parametrize("rows", [1, 40])
def test_a_host_thread_without_a_context(rows):
    """The C call as the first CUDA call of a thread, after another thread has made it already."""
    hidden, codes, scales, zp = _case(rows, 200, 512, 128, True, 81)
    h, c, s, z = _to(hidden, codes, scales, zp)
    q = binding.polyspec_pack_quantized(c)
    want, status = binding.polyspec_lm_head_quantized(h, q, s, z)
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    lib, stream, got = binding.load_library(), torch.cuda.current_stream().cuda_stream, []
    args = (h.data_ptr(), q.data_ptr(), s.data_ptr(), z.data_ptr(), rows, 200, 512, 128, binding.F32, out.data_ptr(), status.data_ptr(), stream)
    thread = threading.Thread(target=lambda: got.append(lib.polyspec_lm_head_quantized(*args)))
    thread.start()
    thread.join()
    torch.cuda.synchronize()
    assert got == [binding.OK] and int(status) == 0
    assert torch.equal(out, want)


def test_threads_with_narrow_and_wide_heads():
    """Same kernel, different shared memory: neither call may take the other's away between its set-up and its launch."""
    lib, stream = binding.load_library(), torch.cuda.current_stream().cuda_stream
    calls, kept = [], []
    for i, (V, d) in enumerate([(64, 1024), (64, 8192)]):
        hidden, codes, scales, zp = _case(4, V, d, 128, True, 61 + i)
        h, c, s, z = _to(hidden, codes, scales, zp)
        out, status, q = torch.empty((4, V), device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV), binding.polyspec_pack_quantized(c)
        kept.append((out, status, h, q, s, z, (hidden, codes, scales, zp)))
        args = (h.data_ptr(), q.data_ptr(), s.data_ptr(), z.data_ptr(), 4, V, d, 128, binding.F32, out.data_ptr(), status.data_ptr(), stream)
        calls.append(lambda a=args: lib.polyspec_lm_head_quantized(*a))
    torch.cuda.synchronize()
    assert run_at_once(calls, 3000) == []
    torch.cuda.synchronize()
    for out, status, *_, case in kept:
        assert int(status) == 0
        _close(out, *case)


def test_a_status_word_made_under_inference_mode_can_be_written_outside():
    hidden, codes, scales, zp = _case(2, 64, 128, 32, True, 71)
    h, c, s, z = _to(hidden, codes, scales, zp)
    q = binding.polyspec_pack_quantized(c)
    binding._status_words.clear()
    with torch.inference_mode():
        binding.polyspec_lm_head_quantized(h, q, s, z)
    _, status = binding.polyspec_lm_head_quantized(h, q, s, z)
    status.zero_()
    status.add_(1)
    assert int(status) == 1


def test_raw_handles_of_the_default_stream():
    """0 and cudaStreamLegacy (1) are the default stream."""
    hidden, codes, scales, zp = _case(2, 64, 128, 32, True, 72)
    h, c, s, z = _to(hidden, codes, scales, zp)
    for handle in (0, 1):
        out, status = binding.polyspec_lm_head_quantized(h, binding.polyspec_pack_quantized(c, stream=handle), s, z, stream=handle)
        torch.cuda.synchronize()
        assert int(status) == 0
        _close(out, hidden, codes, scales, zp)


@pytest.mark.parametrize("rows", [1, 8, 40, 200])
@pytest.mark.parametrize("V,d,group", [(300, 1024, 128), (9001, 1056, 32)])
def test_every_input_written_by_the_kernel_before(rows, V, d, group):
    """The kernel is set up while the one before it drains; what that one writes last is what is read."""
    cases = [_to(*_case(rows, V, d, group, True, 91 + i)) for i in range(2)]
    cases = [[h, binding.polyspec_pack_quantized(c), s, z] for h, c, s, z in cases]
    want = [binding.polyspec_lm_head_quantized(*a)[0] for a in cases]
    now = [t.clone() for t in cases[0]]
    got = []
    for n in range(24):
        for which in range(4):                              # another input written last each time
            for i in range(4):
                now[(which + 1 + i) % 4].copy_(cases[n % 2][(which + 1 + i) % 4])
            got.append((n % 2, binding.polyspec_lm_head_quantized(*now)[0]))
    torch.cuda.synchronize()
    assert all(torch.equal(out, want[i]) for i, out in got)
