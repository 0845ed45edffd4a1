"""The 4-bit LM head, the sampling controls and the cache pages on a machine without a GPU: refusals at the C entry points and
in the Python front end, and the plain page tables the GPU tests compare with."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest
import torch

from paper_2510_26527_b200 import binding, buildlib
from tests import plain_operators as plain

FAKE = 0x1000           # aligned, never dereferenced on the host
INVALID, UNSUPPORTED, WORKSPACE = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    buildlib.build()
    return binding.load_library()


def test_status_and_version(lib):
    assert binding.version() >= 400
    assert "pages" in binding.status_string(binding.ERR_NO_PAGES)


@pytest.mark.parametrize("change,status", [
    ({"hidden": None}, INVALID), ({"qweight": None}, INVALID), ({"scales": None}, INVALID), ({"logits": None}, INVALID),
    ({"hidden": FAKE + 8}, INVALID), ({"qweight": FAKE + 4}, INVALID), ({"logits": FAKE + 4}, INVALID), ({"scales": FAKE + 1}, INVALID),
    ({"rows": 0}, INVALID), ({"V": 0}, INVALID), ({"d": 0}, INVALID), ({"rows": -3}, INVALID), ({"dt": 2}, INVALID),
    ({"group": 16}, UNSUPPORTED), ({"group": 0}, UNSUPPORTED), ({"group": 256}, UNSUPPORTED), ({"d": 4096 + 64}, UNSUPPORTED),
    ({"V": 0x7fffffff}, UNSUPPORTED), ({"rows": 1 << 30, "V": 1 << 20}, UNSUPPORTED),
])
def test_quantized_head_refuses(lib, change, status):
    a = dict(hidden=FAKE, qweight=FAKE, scales=FAKE, zeros=None, rows=8, V=32000, d=4096, group=128, dt=binding.F32, logits=FAKE)
    a.update(change)
    assert lib.polyspec_lm_head_quantized(a["hidden"], a["qweight"], a["scales"], a["zeros"], a["rows"], a["V"], a["d"], a["group"],
                                          a["dt"], a["logits"], None, None) == status


def test_quantized_head_refuses_counts_at_the_end_of_int(lib):
    at = ctypes.c_void_p(1 << 20)                           # refused before it is read
    for rows, V in ((0x7fffffff, 1), (1, 0x7fffffff)):
        assert lib.polyspec_lm_head_quantized(at, at, at, None, rows, V, 32, 32, binding.F32, at, None, None) == binding.ERR_UNSUPPORTED


def test_pack_refuses(lib):
    assert lib.polyspec_pack_quantized(None, 8, 32, FAKE, None) == INVALID
    assert lib.polyspec_pack_quantized(FAKE, 8, 32, None, None) == INVALID
    assert lib.polyspec_pack_quantized(FAKE, 0, 32, FAKE, None) == INVALID
    assert lib.polyspec_pack_quantized(FAKE + 8, 8, 32, FAKE, None) == INVALID
    assert lib.polyspec_pack_quantized(FAKE, 8, 40, FAKE, None) == UNSUPPORTED


@pytest.mark.parametrize("change,status", [
    ({"logits": None}, INVALID), ({"out": None}, INVALID), ({"controls": None}, INVALID), ({"B": 0}, INVALID), ({"rows": 0}, INVALID),
    ({"V": 0}, INVALID), ({"dt": 5}, INVALID), ({"logits": FAKE + 8}, INVALID), ({"out": FAKE + (1 << 40) + 8}, INVALID),
    ({"V": 1004}, UNSUPPORTED), ({"V": 1 << 22}, UNSUPPORTED), ({"B": 1 << 20, "rows": 1 << 12}, UNSUPPORTED),
    ({"out": FAKE + 16}, INVALID),                                              # overlaps without being the same buffer
    ({"draft": FAKE, "k": 0}, INVALID), ({"draft": FAKE, "k": 33}, INVALID), ({"draft": FAKE, "k": 3, "rows": 5}, INVALID),
    ({"history": FAKE}, INVALID),                                               # history_cap 0
    ({"bias_tokens": FAKE, "n_bias": 3}, INVALID), ({"bias_values": FAKE, "n_bias": 3}, INVALID),
    ({"bias_tokens": FAKE, "bias_values": FAKE}, INVALID),
    ({"mask": FAKE + 2}, INVALID), ({"vocab_begin": -8, "vocab_size": 2000}, INVALID), ({"vocab_begin": 8}, INVALID),
    ({"vocab_begin": 1000, "vocab_size": 1999}, INVALID), ({"vocab_size": 999}, INVALID),
])
def test_process_logits_refuses(lib, change, status):
    a = dict(logits=FAKE, out=FAKE + (1 << 40), draft=None, k=0, B=2, rows=4, V=1000, dt=binding.BF16)
    c = binding.LogitControls()
    use = ctypes.byref(c)
    for key, val in change.items():
        if key == "controls":
            use = None
        elif key in a:
            a[key] = val
        else:
            setattr(c, key, val)
    assert lib.polyspec_process_logits(a["logits"], use, a["draft"], a["k"], a["B"], a["rows"], a["V"], a["dt"], a["out"], None, None) == status


def _pages(**change):
    s = binding.CachePagesStruct(4, 8, 100, 16, FAKE, FAKE, FAKE, FAKE)
    for key, val in change.items():
        setattr(s, key, val)
    return ctypes.byref(s)


@pytest.mark.parametrize("change,status", [
    ({"n_seqs": 0}, INVALID), ({"max_pages": 0}, INVALID), ({"n_pages": 0}, INVALID), ({"page_tokens": 0}, INVALID),
    ({"table": None}, INVALID), ({"len": None}, INVALID), ({"refs": None}, INVALID), ({"free_bits": None}, INVALID),
    ({"max_pages": 1 << 16, "page_tokens": 1 << 16}, UNSUPPORTED), ({"n_pages": (1 << 20) + 1}, UNSUPPORTED),
])
def test_cache_calls_refuse_bad_states(lib, change, status):
    s = _pages(**change)
    big = 1 << 40
    assert lib.polyspec_cache_init(s, None) == status
    assert lib.polyspec_cache_reserve(s, FAKE, None, 0, None, 0, None, FAKE, big, None) == status
    assert lib.polyspec_cache_rollback(s, FAKE, None, 0, None, None) == status
    assert lib.polyspec_cache_fork(s, FAKE, FAKE, 1, None, None) == status
    assert lib.polyspec_cache_compact(s, None, 0, None, FAKE, big, None) == status


def test_cache_calls_refuse_bad_arguments(lib):
    s, big = _pages(), 1 << 40
    n = ctypes.c_size_t(0)
    assert lib.polyspec_cache_workspace(4, 100, None) == INVALID
    assert lib.polyspec_cache_workspace(0, 100, ctypes.byref(n)) == INVALID
    assert lib.polyspec_cache_workspace(4, 100, ctypes.byref(n)) == binding.OK and n.value % 256 == 0
    assert lib.polyspec_cache_init(None, None) == INVALID
    assert lib.polyspec_cache_reserve(s, None, None, 0, None, 0, None, FAKE, big, None) == INVALID
    assert lib.polyspec_cache_reserve(s, FAKE, None, 0, None, 0, None, None, big, None) == INVALID
    assert lib.polyspec_cache_reserve(s, FAKE, None, 0, None, 0, None, FAKE + 128, big, None) == INVALID
    assert lib.polyspec_cache_reserve(s, FAKE, None, 0, None, 0, None, FAKE, n.value - 1, None) == WORKSPACE
    assert lib.polyspec_cache_reserve(s, FAKE, None, 0, None, 1, None, FAKE, big, None) == INVALID
    assert lib.polyspec_cache_rollback(s, None, None, 0, None, None) == INVALID
    assert lib.polyspec_cache_fork(s, None, FAKE, 1, None, None) == INVALID
    assert lib.polyspec_cache_fork(s, FAKE, FAKE, 0, None, None) == INVALID
    assert lib.polyspec_cache_compact(s, None, 0, None, FAKE, n.value - 1, None) == WORKSPACE
    for pool in ((None, 2, 64), (FAKE + 8, 2, 64), (FAKE, 0, 64), (FAKE, 2, 0), (FAKE, 2, 24)):
        p = (binding.CachePool * 1)(binding.CachePool(*pool))
        assert lib.polyspec_cache_reserve(s, FAKE, None, 0, p, 1, None, FAKE, big, None) == INVALID, pool
        assert lib.polyspec_cache_compact(s, p, 1, None, FAKE, big, None) == INVALID, pool
    p = (binding.CachePool * 9)(*[binding.CachePool(FAKE, 1, 16)] * 9)
    assert lib.polyspec_cache_reserve(s, FAKE, None, 0, p, 9, None, FAKE, big, None) == INVALID


def test_front_end_refuses(lib):
    h, q = torch.zeros((2, 64), dtype=torch.bfloat16), torch.zeros((8, 8), dtype=torch.int32)
    s = torch.zeros((8, 2), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        binding.polyspec_lm_head_quantized(h, q, s)
    with pytest.raises(TypeError):
        binding.polyspec_lm_head_quantized(h.float(), q, s)
    with pytest.raises(TypeError):
        binding.polyspec_lm_head_quantized(h, q, s, zero_points=torch.zeros((8, 2), dtype=torch.int32))
    with pytest.raises(ValueError, match="shapes"):
        binding.polyspec_lm_head_quantized(h, q[:, :4], s)
    with pytest.raises(ValueError, match="shapes"):
        binding.polyspec_lm_head_quantized(h, q, torch.zeros((8, 3), dtype=torch.bfloat16))
    z = torch.zeros((2, 3, 64))
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    for kw in ({"mask": i32(2, 3, 3)}, {"history_len": i32(2)}, {"history": i32(3, 5)}, {"bias_tokens": i32(2, 5)},
               {"repetition": torch.ones(3)}, {"draft_tokens": i32(2)}, {"out": torch.zeros(2, 3, 32)}):
        with pytest.raises(ValueError):
            binding.polyspec_process_logits(z, **kw)
    for kw in ({"mask": torch.zeros(2, 3, 2)}, {"out": z.double()}, {"repetition": torch.ones(2).double()},
               {"device_status": torch.zeros(1)}):
        with pytest.raises(TypeError):
            binding.polyspec_process_logits(z, **kw)
    with pytest.raises(ValueError, match="shapes"):
        binding.CachePages(i32(4, 8), i32(4), i32(100), i32(3), 16)
    with pytest.raises(ValueError, match="CUDA"):
        binding.CachePages(i32(4, 8), i32(4), i32(100), i32(4), 16)


def test_plain_pages_keep_their_invariants():
    rng = random.Random(7)
    p = plain.Pages(6, 9, 40, 4)
    for _ in range(400):
        what = rng.randrange(4)
        if what == 0:
            p.reserve([n + rng.randrange(-2, 9) for n in p.len])
        elif what == 1:
            p.rollback([rng.randrange(-1, 30) for _ in p.len])
        elif what == 2:
            p.fork([rng.randrange(-1, 7) for _ in range(2)], [rng.randrange(-1, 7) for _ in range(2)])
        else:
            p.compact()
            assert all(p.refs[i] for i in range(sum(c > 0 for c in p.refs)))
        held = [q for row in p.rows for q in row]
        assert all(held.count(i) == p.refs[i] for i in range(p.n_pages))
        assert all(len(row) == p.need(n) and len(set(row)) == len(row) for row, n in zip(p.rows, p.len))
    a = p.arrays()
    assert all(bool(a["free_bits"][i // 32] >> (i % 32) & 1) == (a["refs"][i] == 0) for i in range(p.n_pages))


def test_mask_words():
    rng = np.random.default_rng(0)
    allowed = rng.random((2, 3, 72)) < 0.5
    w = plain.mask_words(allowed)
    assert w.shape == (2, 3, 3)
    assert all(bool(w[b, j, v // 32] >> (v % 32) & 1) == allowed[b, j, v] for b in range(2) for j in range(3) for v in range(72))


def test_streaming_ring_leaves_no_copy_on_its_way(tmp_path):
    """The 4-bit head's ring on the host, given up at every point (a wait that runs out cannot be made to happen on the GPU)."""
    exe = str(tmp_path / "piece_ring")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=address,undefined", "-I", buildlib.CSRC, "-o", exe,
                    os.path.join(here, "piece_ring_driver.cpp")], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and "0 failed checks" in res.stdout, res.stdout


@pytest.mark.parametrize("shape,strides", [((2, 1, 64), (64, 64, 1)), ((1, 1, 64), (64, 1, 1)), ((2, 1, 64), (64, 999, 1)), ((1, 5, 4, 8), (160, 32, 8, 1)),
                                           ((3, 5, 32), (160, 32, 1))])
def test_page_sizes_of_contiguous_pools(shape, strides):
    """A contiguous tensor may have any stride in a dimension of size 1."""
    t = torch.empty(200 + strides[0] * shape[0], dtype=torch.bfloat16).as_strided(shape, strides)
    assert t.is_contiguous()
    pages = type("Pages", (), {"n_pages": shape[1]})
    (pool,) = binding._pools(pages, [t])
    assert pool.n_planes == shape[0] and pool.page_bytes == 2 * t[0, 0].numel()
    with pytest.raises(ValueError):
        binding._pools(pages, [torch.empty((0,) + shape[1:])])


@pytest.mark.parametrize("off", [1, 2, 3])
def test_arrays_of_words_off_their_boundary_are_refused(lib, off):
    at, big = FAKE + off, 1 << 40
    head = lambda status: lib.polyspec_lm_head_quantized(FAKE, FAKE, FAKE, None, 8, 32000, 4096, 128, binding.F32, FAKE, status, None)
    assert head(at) == INVALID

    def controls(draft=None, status=None, **fields):
        c = binding.LogitControls(history_cap=5, n_bias=3, **fields)
        return lib.polyspec_process_logits(FAKE, ctypes.byref(c), draft, 3, 2, 4, 1000, binding.BF16, FAKE + big, status, None)

    assert controls(draft=at) == INVALID and controls(status=at) == INVALID
    for name in ("history", "history_len", "prompt_len", "repetition", "frequency", "presence", "mask"):
        assert controls(**{name: at}) == INVALID, name
    assert controls(bias_tokens=at, bias_values=FAKE) == INVALID and controls(bias_tokens=FAKE, bias_values=at) == INVALID

    def pages(s, base=FAKE, extra=None, moved_to=None, status=None):
        return (lib.polyspec_cache_reserve(s, base, extra, 0, None, 0, status, FAKE, big, None), lib.polyspec_cache_rollback(s, base, extra, 0, status, None),
                lib.polyspec_cache_fork(s, base, FAKE, 1, status, None), lib.polyspec_cache_fork(s, FAKE, base, 1, status, None))

    for name in ("table", "len", "refs", "free_bits"):
        s = _pages(**{name: at})
        assert pages(s) == (INVALID,) * 4 and lib.polyspec_cache_init(s, None) == INVALID
        assert lib.polyspec_cache_compact(s, None, 0, None, FAKE, big, None) == INVALID
    s = _pages()
    assert pages(s, base=at) == (INVALID,) * 4 and pages(s, status=at) == (INVALID,) * 4
    assert pages(s, extra=at)[:2] == (INVALID,) * 2
    assert lib.polyspec_cache_compact(s, None, 0, at, FAKE, big, None) == INVALID
