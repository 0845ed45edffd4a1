"""Sampling controls on logits against their 64-bit statement.

Tolerance of a touched entry: a division or product, a product and two subtractions, and one addition per bias are each off by
at most 2^-24 of a value that the sum of the magnitudes involved bounds, so (4 + biases) 2^-24 of that sum (+ |z|); bf16 is
rounded once more, by at most 2^-8 of the value.  Entries that nothing touches keep their bits."""
import numpy as np
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


def _inputs(B, rows, V, dtype, history=0, bias=0, mask=False, draft=True, seed=0):
    rng = np.random.default_rng(seed + B * 1000 + V)
    z = torch.from_numpy(rng.normal(0, 3, (B, rows, V)).astype(np.float32)).to(dtype)
    kw = {}
    skew = lambda *shape: (rng.random(shape) ** 3 * V).astype(np.int32)
    if draft:
        kw["draft_tokens"] = skew(B, max(1, rows - 1))
    if history:
        kw["history"] = skew(B, history)
        kw["history_len"] = rng.integers(0, history + 1, B).astype(np.int32)
        kw["prompt_len"] = (kw["history_len"] * rng.random(B)).astype(np.int32)
    kw["repetition"] = rng.uniform(0.8, 1.5, B).astype(np.float32)
    kw["frequency"] = rng.uniform(-0.3, 0.6, B).astype(np.float32)
    kw["presence"] = rng.uniform(-0.5, 1.0, B).astype(np.float32)
    if bias:
        kw["bias_tokens"] = skew(B, bias)
        kw["bias_tokens"][:, 1::5] = -1
        kw["bias_values"] = rng.normal(0, 4, (B, bias)).astype(np.float32)
    allowed = None
    if mask:
        allowed = rng.random((B, rows, V)) < rng.choice([0.002, 0.5, 0.99], (B, rows, 1))
        allowed[0, 0] = False
        allowed[-1, -1] = True
    return z, kw, allowed


def _call(z, kw, allowed, **more):
    dev = {k: torch.from_numpy(np.ascontiguousarray(v)).to(DEV) for k, v in kw.items()}
    if allowed is not None:
        dev["mask"] = torch.from_numpy(plain.mask_words(allowed)).to(DEV)
    return binding.polyspec_process_logits(z, **dev, **more)


def _reference(z, kw, allowed, **more):
    names = {"draft_tokens": "draft"}
    return plain.controls(z.float().numpy(), allowed=allowed, **{names.get(k, k): v for k, v in kw.items()}, **more)


def _close(got, z, kw, allowed, **more):
    ref, touched, size = _reference(z, kw, allowed, **more)
    got = got.cpu()
    same = got.view(torch.int16 if got.dtype == torch.bfloat16 else torch.int32).numpy() == \
        z.view(torch.int16 if z.dtype == torch.bfloat16 else torch.int32).numpy()
    assert same[~touched].all()
    x = got.double().numpy()
    n = 4 + (kw["bias_tokens"].shape[1] if "bias_tokens" in kw else 0)
    tol = n * 2.0 ** -24 * (size + np.abs(z.double().numpy()))
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.where(np.isfinite(ref), np.abs(ref), 0) + tol)
    finite = np.isfinite(ref)
    assert (np.isneginf(x) == np.isneginf(ref)).all()
    assert (np.abs(x - ref)[finite] <= tol[finite]).all(), float((np.abs(x - ref) - tol)[finite].max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,rows,V,history,bias,mask,draft", [
    (1, 1, 8, 0, 0, False, False),
    (1, 1, 8, 3, 2, True, True),
    (1, 9, 1000, 50, 5, True, True),
    (2, 33, 2048, 300, 0, False, True),
    (3, 5, 2056, 1, 40, True, True),          # one vector past a slice of 2048
    (2, 4, 8200, 2500, 70, True, True),
    (5, 3, 16392, 9000, 33, False, True),
    (40, 7, 32000, 64, 8, True, True),        # enough CTAs for the widest slices
    (4, 6, 32000, 0, 0, True, False),         # masks alone
    (4, 6, 32000, 700, 0, False, False),      # a history alone
    (300, 2, 1024, 17, 1, True, True),
])
def test_against_plain(B, rows, V, history, bias, mask, draft, dtype):
    z, kw, allowed = _inputs(B, rows, V, dtype, history, bias, mask, draft)
    if not draft and not history and not bias:
        kw = {}
    zd = z.to(DEV)
    out, status = _call(zd, kw, allowed)
    torch.cuda.synchronize()
    assert int(status) == 0
    _close(out, z, kw, allowed)
    assert torch.equal(zd.cpu(), z)
    inside, _ = _call(zd, kw, allowed, out=zd)             # in place: the same bits
    assert inside is zd
    assert torch.equal(zd.view(torch.uint8), out.view(torch.uint8))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_special_values(dtype):
    B, rows, V = 1, 3, 64
    z = torch.randn((B, rows, V), generator=torch.Generator().manual_seed(1)).to(dtype)
    low = torch.finfo(dtype).min
    z[0, :, 0], z[0, :, 1], z[0, :, 2], z[0, :, 3], z[0, :, 4] = float("nan"), float("inf"), float("-inf"), low, 0.0
    z[0, :, 10], z[0, :, 11], z[0, :, 12] = float("nan"), float("inf"), low
    allowed = np.ones((B, rows, V), dtype=bool)
    allowed[0, 1, 10:13] = False                            # NaN, inf and the lowest value in masked places
    allowed[0, 2] = False                                   # a row that allows nothing
    kw = {"history": np.array([[1, 2, 3, 4, 5, 5]], dtype=np.int32), "repetition": np.array([2.0], dtype=np.float32),
          "bias_tokens": np.array([[6, 7]], dtype=np.int32), "bias_values": np.array([[float("-inf"), 1e30]], dtype=np.float32)}
    out, status = _call(z.to(DEV), kw, allowed)
    x = out.cpu().float()
    assert int(status) == 0
    assert x[0, 0, 0].isnan() and x[0, 0, 1] == float("inf") and x[0, 0, 2] == float("-inf")
    assert x[0, 0, 3] == float("-inf")                      # the lowest value times 2: out of the type's range
    assert x[0, 0, 4] == 0 and x[0, 0, 6] == float("-inf") and x[0, 0, 7] > 9e29
    assert x[0, 0, 10].isnan() and x[0, 0, 11] == float("inf") and x[0, 0, 12] == low
    assert (x[0, 1, 10:13] == float("-inf")).all() and (x[0, 2] == float("-inf")).all()
    # such a row is unusable for the verification, not a crash
    q = torch.zeros((B, 2, V), device=DEV, dtype=dtype)
    lv = binding.polyspec_verify_level(out, q, torch.tensor([[5, 5]], dtype=torch.int32, device=DEV), torch.full((1, 3), 0.5, device=DEV), 1.0)
    torch.cuda.synchronize()
    assert int(lv["accepted_len"][0]) == -1 and int(lv["device_status"]) == binding.ERR_BAD_INPUT_ON_DEVICE


def test_bad_tokens_lengths_and_factors_are_reported_and_left_out():
    V = 128
    z = torch.randn((2, 3, V), generator=torch.Generator().manual_seed(2))
    good = {"history": np.array([[1, 2, 2, -1, -5], [3, 3, 3, 3, 3]], dtype=np.int32), "frequency": np.array([0.5, 0.25], dtype=np.float32),
            "draft_tokens": np.array([[7, -1], [3, 9]], dtype=np.int32)}
    out, status = _call(z.to(DEV), good, None)
    assert int(status) == 0
    _close(out, z, good, None)
    for name, at, val in (("history", (0, 4), V), ("history", (1, 0), 2 ** 31 - 1), ("draft_tokens", (0, 1), V + 5)):
        kw = {k: v.copy() for k, v in good.items()}
        kw[name][at] = val
        out, status = _call(z.to(DEV), kw, None)
        assert int(status) == binding.ERR_BAD_INPUT_ON_DEVICE, name
        _close(out, z, kw, None)
    for more in ({"history_len": np.array([6, 2], dtype=np.int32)}, {"history_len": np.array([3, -1], dtype=np.int32)},
                 {"history_len": np.array([3, 2], dtype=np.int32), "prompt_len": np.array([1, 3], dtype=np.int32)},
                 {"repetition": np.array([1.5, 0.0], dtype=np.float32)}, {"repetition": np.array([np.nan, 1.0], dtype=np.float32)},
                 {"bias_tokens": np.array([[4], [V]], dtype=np.int32), "bias_values": np.ones((2, 1), dtype=np.float32)}):
        kw = {**good, **more}
        out, status = _call(z.to(DEV), kw, None)
        assert int(status) == binding.ERR_BAD_INPUT_ON_DEVICE, more
        _close(out, z, kw, None)


def test_a_token_listed_twice_counts_twice_in_list_order():
    V = 64
    z = torch.zeros((1, 1, V))
    rng = np.random.default_rng(3)
    toks = rng.choice([5, 9, 40], (1, 200)).astype(np.int32)
    vals = (rng.normal(0, 1, (1, 200)) * 10.0 ** rng.integers(-4, 4, (1, 200))).astype(np.float32)
    got, _ = _call(z.to(DEV), {"bias_tokens": toks, "bias_values": vals}, None)
    for v in (5, 9, 40):
        s = np.float32(0)
        for t, x in zip(toks[0], vals[0]):
            if t == v:
                s = np.float32(s + x)
        assert float(got[0, 0, v]) == float(s)
    for _ in range(5):
        again, _ = _call(z.to(DEV), {"bias_tokens": toks, "bias_values": vals}, None)
        assert torch.equal(again, got)


@pytest.mark.parametrize("ranks", [2, 4])
def test_slices_of_a_sharded_vocabulary_equal_the_whole(ranks):
    B, rows, V = 3, 5, 4096
    z, kw, allowed = _inputs(B, rows, V, torch.bfloat16, 200, 20, True, True)
    whole, _ = _call(z.to(DEV), kw, allowed)
    n = V // ranks
    for r in range(ranks):
        part = z[..., r * n:(r + 1) * n].contiguous().to(DEV)
        got, status = _call(part, kw, np.ascontiguousarray(allowed[..., r * n:(r + 1) * n]), vocab_begin=r * n, vocab_size=V)
        assert int(status) == 0
        assert torch.equal(got, whole[..., r * n:(r + 1) * n])


@pytest.mark.parametrize("history,bias", [(40, 5), (300, 256), (300, 257), (9000, 700)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_bias_lists_and_long_histories(history, bias, dtype):
    """Short and long bias lists, 16- and 32-bit counts, in every combination that the kernel tells apart."""
    z, kw, allowed = _inputs(2, 3, 4104, dtype, history, bias, True, True, seed=history)
    out, status = _call(z.to(DEV), kw, allowed)
    assert int(status) == 0
    _close(out, z, kw, allowed)
    only = {k: kw[k] for k in ("bias_tokens", "bias_values")}
    out, status = _call(z.to(DEV), only, None)
    assert int(status) == 0
    _close(out, z, only, None)


@pytest.mark.parametrize("dtype,V", [(torch.bfloat16, 16392), (torch.float32, 9000)])
def test_a_sequence_does_not_depend_on_its_batch(dtype, V):
    """Wide batches take other slice sizes than single sequences: the same bits."""
    B, rows = 620, 3
    z, kw, allowed = _inputs(B, rows, V, dtype, 64, 12, True, True, seed=9)
    whole, status = _call(z.to(DEV), kw, allowed)
    assert int(status) == 0
    for b in (0, 57, 301, B - 1):
        one, _ = _call(z[b:b + 1].to(DEV), {k: v[b:b + 1] for k, v in kw.items()}, allowed[b:b + 1])
        assert torch.equal(one[0], whole[b])
    some = slice(0, 3)
    _close(whole[some], z[some], {k: v[some] for k, v in kw.items()}, allowed[some])


def test_captured_on_another_stream_and_repeated():
    B, rows, V = 4, 5, 10000
    z, kw, allowed = _inputs(B, rows, V, torch.float32, 500, 30, True, True)
    dev = {k: torch.from_numpy(v).to(DEV) for k, v in kw.items()}
    dev["mask"] = torch.from_numpy(plain.mask_words(allowed)).to(DEV)
    zd = z.to(DEV)
    want, status = binding.polyspec_process_logits(zd, **dev)
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.polyspec_process_logits(zd, **dev, out=out, device_status=status)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _ = binding.polyspec_process_logits(zd, **dev, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_offsets_past_32_bits():
    """A batch whose logits pass 2^32 bytes: the last sequence is addressed like the first."""
    B, rows, V = 130, 9, 1 << 21                            # 4.9 GB of bf16
    z = torch.zeros((B, rows, V), dtype=torch.bfloat16, device=DEV)
    z[-1, -1, -8:] = 2.0
    hist = torch.full((B, 2), V - 3, dtype=torch.int32, device=DEV)
    out, status = binding.polyspec_process_logits(z, history=hist, frequency=torch.full((B,), 0.5, device=DEV), out=z)
    torch.cuda.synchronize()
    assert int(status) == 0
    assert z[-1, -1, -8:].tolist() == [2.0] * 5 + [1.0] + [2.0] * 2
    assert (z[:, :, V - 3] == torch.where(torch.arange(B * rows, device=DEV).view(B, rows) == B * rows - 1, 1.0, -1.0)).all()
    assert int((z != 0).sum()) == B * rows + 7


def test_threads_with_short_and_long_bias_lists():
    """Both take the widest slices with 32-bit counts and differ in shared memory only: neither may take the other's away."""
    B, rows, V, cap = 300, 1, 32768, 8192
    lib, stream = binding.load_library(), torch.cuda.current_stream().cuda_stream
    z = torch.randn((B, rows, V), generator=torch.Generator(device=DEV).manual_seed(4), device=DEV).to(torch.bfloat16)
    text = torch.arange(cap, device=DEV, dtype=torch.int32).repeat(B, 1)
    length = torch.full((B,), 4, dtype=torch.int32, device=DEV)
    calls, kept = [], []
    for n in (8, 300):
        kw = {"history": text, "history_len": length, "bias_tokens": torch.arange(n, device=DEV, dtype=torch.int32).repeat(B, 1),
              "bias_values": torch.ones((B, n), device=DEV)}
        out, status = torch.empty_like(z), torch.zeros(1, dtype=torch.int32, device=DEV)
        c = binding.LogitControls(history=text.data_ptr(), history_len=length.data_ptr(), bias_tokens=kw["bias_tokens"].data_ptr(),
                                  bias_values=kw["bias_values"].data_ptr(), history_cap=cap, n_bias=n)
        kept.append((n, out, status, kw, c))
        args = (z.data_ptr(), c, None, 0, B, rows, V, binding.BF16, out.data_ptr(), status.data_ptr(), stream)
        calls.append(lambda a=args: lib.polyspec_process_logits(*a))
    torch.cuda.synchronize()
    assert run_at_once(calls, 400) == []
    torch.cuda.synchronize()
    for n, out, status, *_ in kept:
        want = z.float()
        want[..., :n] += 1.0
        assert int(status) == 0 and torch.equal(out, want.to(torch.bfloat16))


@pytest.mark.parametrize("value", [0.0, -1.0, float("nan")])
def test_a_bad_repetition_is_reported_where_there_is_no_context(value):
    """Without a history, a draft or biases no entry is penalised, but the factor is looked at all the same."""
    B, rows, V = 3, 2, 5000
    z, _, allowed = _inputs(B, rows, V, torch.bfloat16, mask=True)
    for bad in range(B):
        rep = np.ones(B, dtype=np.float32)
        for masks in (allowed, None):
            out, status = _call(z.to(DEV), {"repetition": rep}, masks)
            assert int(status) == 0
        rep[bad] = value
        for masks in (allowed, None):
            out, status = _call(z.to(DEV), {"repetition": rep}, masks)
            assert int(status) == binding.ERR_BAD_INPUT_ON_DEVICE
            _close(out, z, {}, masks)
