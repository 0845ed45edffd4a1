"""The attention around the cache pages on a machine without a GPU: refusals at the C entry points and in the Python front end, and the plain
arithmetic that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2510_26527_b200 import binding, buildlib
from tests import plain_attention as plain

FAKE = 0x1000           # aligned, never dereferenced on the host
BIG = 1 << 40
INVALID, UNSUPPORTED, WORKSPACE = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    buildlib.build()
    return binding.load_library()


def _call(fn, defaults, change):
    a = dict(defaults)
    for key in change:
        assert key in a, key
    a.update(change)
    return fn(*a.values())


ROTATE = dict(q=FAKE, q_stride=6144, q_heads=32, k=FAKE, k_stride=6144, kv_heads=8, rows=9, d=128, rotary=128, interleaved=0, positions=FAKE, frequencies=FAKE,
              q_weight=FAKE, k_weight=None, eps=1e-6, q_out=FAKE + BIG, q_out_stride=4096, k_out=FAKE + BIG, k_out_stride=1024, stream=None)


@pytest.mark.parametrize("change,status", [
    ({"q": None}, INVALID), ({"q_out": None}, INVALID), ({"k": None}, INVALID), ({"k_out": None}, INVALID), ({"kv_heads": 0}, INVALID),
    ({"q": FAKE + 8}, INVALID), ({"k_out": FAKE + 2}, INVALID), ({"q_weight": FAKE + 4}, INVALID), ({"positions": None}, INVALID),
    ({"frequencies": None}, INVALID), ({"positions": FAKE + 2}, INVALID), ({"q_stride": 4088}, INVALID), ({"k_stride": 6140}, INVALID),
    ({"q_out_stride": 4100}, INVALID), ({"rows": 0}, INVALID), ({"rows": -1}, INVALID), ({"d": 0}, INVALID), ({"rotary": -16}, INVALID),
    ({"rotary": 144}, INVALID), ({"eps": -1.0}, INVALID), ({"eps": float("nan")}, INVALID), ({"eps": float("inf")}, INVALID), ({"q_heads": 0}, INVALID),
    ({"kv_heads": -1}, INVALID), ({"q_out": FAKE}, INVALID),                   # in place with another stride
    ({"d": 272, "q_stride": 32 * 272}, UNSUPPORTED), ({"rotary": 24}, UNSUPPORTED), ({"d": 120, "rotary": 96}, UNSUPPORTED), ({"rows": 1 << 25}, UNSUPPORTED),
    ({"q_heads": 5000}, UNSUPPORTED),
])
def test_rotate_refuses(lib, change, status):
    assert _call(lib.polyspec_rotate_heads, ROTATE, change) == status


PROMPT = dict(q=FAKE, q_stride=6144, k=FAKE, k_stride=6144, v=FAKE, v_stride=6144, rows_at=FAKE, n_seqs=3, rows=900, q_heads=32, kv_heads=8, d=128, scale=0.1,
              out=FAKE, lse=None, status=None, stream=None)


@pytest.mark.parametrize("change,status", [
    ({"q": None}, INVALID), ({"k": None}, INVALID), ({"v": None}, INVALID), ({"rows_at": None}, INVALID), ({"out": None}, INVALID), ({"out": FAKE + 8}, INVALID),
    ({"v": FAKE + 8}, INVALID), ({"lse": FAKE + 2}, INVALID), ({"n_seqs": 0}, INVALID), ({"rows": 0}, INVALID), ({"q_heads": 0}, INVALID), ({"kv_heads": 0}, INVALID),
    ({"q_stride": 4095}, INVALID), ({"k_stride": 1020}, INVALID), ({"scale": float("nan")}, INVALID), ({"scale": float("inf")}, INVALID), ({"scale": -0.1}, INVALID),
    ({"kv_heads": 5}, UNSUPPORTED), ({"d": 96}, UNSUPPORTED), ({"d": 256}, UNSUPPORTED), ({"rows": 1 << 25}, UNSUPPORTED), ({"q_heads": 2048, "kv_heads": 2048}, UNSUPPORTED),
    ({"n_seqs": (1 << 20) + 1}, UNSUPPORTED),
])
def test_prompt_attention_refuses(lib, change, status):
    assert _call(lib.polyspec_prompt_attention, PROMPT, change) == status


def _pages(**change):
    s = binding.CachePagesStruct(4, 8, 100, 16, FAKE, FAKE, FAKE, FAKE)
    for key, val in change.items():
        setattr(s, key, val)
    return ctypes.byref(s)


def _rows(**change):
    r = binding.BlockRows(FAKE, None, FAKE, None, 20)
    for key, val in change.items():
        setattr(r, key, val)
    return ctypes.byref(r)


def _all_calls(lib, s, r, **change):
    """append, attention and weigh with the same pages and rows"""
    a = dict(heads=8, kv=4, d=128)
    a.update(change)
    stride = a["heads"] * 128
    return {lib.polyspec_cache_append(s, r, FAKE, stride, FAKE, stride, a["kv"], a["d"], FAKE, None, None, None, None, None),
            lib.polyspec_cache_attention(s, r, FAKE, stride, a["heads"], a["kv"], a["d"], 0.1, FAKE, FAKE, None, None, FAKE, BIG, None),
            lib.polyspec_cache_weigh(s, r, FAKE, stride, a["heads"], a["kv"], a["d"], 0.1, FAKE, FAKE, 1.0, FAKE, None, None)}


@pytest.mark.parametrize("change,status", [
    ({"n_seqs": 0}, INVALID), ({"max_pages": 0}, INVALID), ({"n_pages": 0}, INVALID), ({"page_tokens": 0}, INVALID), ({"table": None}, INVALID),
    ({"len": None}, INVALID), ({"refs": FAKE + 2}, INVALID), ({"max_pages": 1 << 16, "page_tokens": 1 << 15}, UNSUPPORTED), ({"page_tokens": 12}, UNSUPPORTED),
    ({"page_tokens": 4}, UNSUPPORTED), ({"page_tokens": 32776}, UNSUPPORTED), ({"n_pages": (1 << 20) + 1}, UNSUPPORTED),
])
def test_calls_on_pages_refuse_bad_states(lib, change, status):
    assert _all_calls(lib, _pages(**change), _rows()) == {status}
    assert lib.polyspec_cache_evict(_pages(**change), FAKE, 0, 0, FAKE, FAKE, 2, 4, 128, None, None, FAKE, BIG, None) == status


def test_calls_on_pages_refuse_caches_whose_ends_counters_would_pass(lib):
    assert _all_calls(lib, _pages(max_pages=65535, page_tokens=32768), _rows()) == {UNSUPPORTED}
    assert lib.polyspec_cache_evict(_pages(max_pages=65535, page_tokens=32768), FAKE, 0, 0, FAKE, FAKE, 2, 4, 128, None, None, FAKE, BIG, None) == UNSUPPORTED
    assert lib.polyspec_cache_evict_workspace(4, 65535, 32768, ctypes.byref(ctypes.c_size_t(0))) == UNSUPPORTED
    assert lib.polyspec_cache_evict_workspace(4, 65534, 32768, ctypes.byref(ctypes.c_size_t(0))) == binding.OK


@pytest.mark.parametrize("change,status", [
    ({"rows_at": None}, INVALID), ({"base": None}, INVALID), ({"rows": 0}, INVALID), ({"n_rows": FAKE + 1}, INVALID), ({"extra": FAKE + 2}, INVALID), ({"rows": 1 << 25}, UNSUPPORTED),
])
def test_calls_on_pages_refuse_bad_rows(lib, change, status):
    assert _all_calls(lib, _pages(), _rows(**change)) == {status}


@pytest.mark.parametrize("change,status", [({"d": 80}, UNSUPPORTED), ({"d": 0}, INVALID), ({"kv": 0}, INVALID)])
def test_calls_on_pages_refuse_bad_heads(lib, change, status):
    assert _all_calls(lib, _pages(), _rows(), **change) == {status}
    assert lib.polyspec_cache_attention_workspace(8, change.get("kv", 4), change.get("d", 128), ctypes.byref(ctypes.c_size_t(0))) == status


def test_calls_on_pages_refuse_bad_arguments(lib):
    s, r = _pages(), _rows()
    n = ctypes.c_size_t(0)
    assert lib.polyspec_cache_attention_workspace(8, 4, 128, None) == INVALID
    assert lib.polyspec_cache_attention_workspace(8, 3, 128, ctypes.byref(n)) == UNSUPPORTED
    assert lib.polyspec_cache_attention_workspace(8, 4, 128, ctypes.byref(n)) == binding.OK and n.value % 256 == 0
    at = dict(s=s, r=r, q=FAKE, stride=1024, heads=8, kv=4, d=128, scale=0.1, pool=FAKE, out=FAKE, lse=None, status=None, ws=FAKE, bytes=n.value, stream=None)
    for change, want in (({"q": None}, INVALID), ({"stride": 1016}, INVALID), ({"stride": 1028}, INVALID), ({"pool": None}, INVALID), ({"pool": FAKE + 8}, INVALID),
                         ({"out": None}, INVALID), ({"lse": FAKE + 1}, INVALID), ({"status": FAKE + 1}, INVALID), ({"ws": None}, INVALID), ({"ws": FAKE + 128}, INVALID),
                         ({"bytes": n.value - 512}, WORKSPACE), ({"scale": float("nan")}, INVALID), ({"heads": 9, "stride": 2048}, UNSUPPORTED), ({"r": None}, INVALID), ({"s": None}, INVALID)):
        assert _call(lib.polyspec_cache_attention, at, change) == want, change
    ap = dict(s=s, r=r, k=FAKE, ks=512, v=FAKE, vs=512, kv=4, d=128, pool=FAKE, kh=None, vh=None, w=None, status=None, stream=None)
    for change in ({"k": None}, {"v": FAKE + 4}, {"ks": 504}, {"pool": None}, {"kh": FAKE + 8}, {"vh": FAKE + 2}, {"w": FAKE + 1}):
        assert _call(lib.polyspec_cache_append, ap, change) == INVALID, change
    we = dict(s=s, r=r, q=FAKE, stride=1024, heads=8, kv=4, d=128, scale=0.1, pool=FAKE, lse=FAKE, keep=1.0, w=FAKE, status=None, stream=None)
    for change in ({"lse": None}, {"w": None}, {"keep": -0.1}, {"keep": 1.5}, {"keep": float("nan")}, {"q": FAKE + 8}):
        assert _call(lib.polyspec_cache_weigh, we, change) == INVALID, change
    assert lib.polyspec_cache_evict_workspace(4, 8, 16, None) == INVALID
    assert lib.polyspec_cache_evict_workspace(0, 8, 16, ctypes.byref(n)) == INVALID
    assert lib.polyspec_cache_evict_workspace(4, 1 << 20, 1 << 12, ctypes.byref(n)) == UNSUPPORTED
    assert lib.polyspec_cache_evict_workspace(4, 8, 16, ctypes.byref(n)) == binding.OK
    ev = dict(s=s, budget=FAKE, first=0, recent=0, w=FAKE, pool=FAKE, planes=4, kv=4, d=128, kept=None, status=None, ws=FAKE, bytes=n.value, stream=None)
    for change, want in (({"budget": None}, INVALID), ({"first": -1}, INVALID), ({"recent": -2}, INVALID), ({"w": None}, INVALID), ({"pool": None}, INVALID), ({"planes": 3}, INVALID),
                         ({"planes": 0}, INVALID), ({"kept": FAKE + 2}, INVALID), ({"ws": None}, INVALID), ({"ws": FAKE + 64}, INVALID), ({"bytes": n.value - 1}, WORKSPACE),
                         ({"d": 32}, UNSUPPORTED)):
        assert _call(lib.polyspec_cache_evict, ev, change) == want, change


def test_front_end_refuses_host_tensors_and_wrong_types():
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    at = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.polyspec_prompt_attention(x, x, x, at)
    with pytest.raises(TypeError):
        binding.polyspec_prompt_attention(x.float(), x, x, at)
    with pytest.raises(ValueError):
        binding.polyspec_rotate_heads(x, None, torch.zeros(4, dtype=torch.int32), torch.zeros(32))
    with pytest.raises(TypeError):
        binding.polyspec_rotate_heads(x.half(), None, torch.zeros(4, dtype=torch.int32), torch.zeros(32))
    assert binding.cache_page_bytes(8, 128, 16) == 8 * 2 * 544


def test_plain_quantisation_keeps_to_half_a_step():
    x = torch.randn((50, 3, 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).float().numpy()
    x[0, 0] = 2.0
    code, scale, offset, held = plain.quantise(x)
    back = scale.astype(np.float64)[..., None] * code + offset.astype(np.float64)[..., None]
    assert code.min() == 0 and code.max() == 15
    # half a step, the division's and the difference's roundings
    assert (np.abs(back - x) <= scale[..., None] * (0.5 + 16 * plain.U32)).all()
    assert (back[0, 0] == 2.0).all() and scale[0, 0] == 1.0
    assert (np.abs(held - back) <= plain.UB * np.abs(back) + scale[..., None] * 32 * plain.U32).all()


def test_plain_pages_are_read_back_word_by_word():
    c = plain.Cache([21], 2, 128, 8, seed=2)
    pool = c.pool()
    for plane in range(2):
        for slot in (0, 7, 13, 20):
            unit = pool[plane, c.table[0, slot // 8], 1, 0]
            for dim in (0, 1, 9, 66, 127):
                w, r = dim // 8, slot % 8
                place = (8 * (w % 8) + r) * 2 + w // 8 if plane else r * 16 + w
                e = dim % 8
                assert int(unit[place]) >> (4 * (e // 2) + 16 * (e % 2)) & 15 == c.codes[plane][0][slot, 1, dim]


def test_plain_attention_rows_see_up_to_themselves():
    c = plain.Cache([6], 1, 64, 8, seed=3)
    q = np.zeros((2, 1, 64), np.float32)
    out, lse, _, _, weights, _ = plain.attend(c, q, [0, 2], [4])
    v = c.value(1, 0)[:, 0]
    np.testing.assert_allclose(out[0, 0], v[:5].mean(0))
    np.testing.assert_allclose(lse[:, 0], np.log([5, 6]))
    np.testing.assert_allclose(weights[0], [1 / 5 + 1 / 6] * 5 + [1 / 6])


def test_plain_eviction():
    w = np.array([0.0, 5, 1, 5, np.nan, 2, 9, 0], np.float32)
    assert plain.evict_slots(w, 8, 5, 1, 2) == [0, 1, 3, 6, 7]
    assert plain.evict_slots(w, 8, 4, 1, 2) == [0, 1, 6, 7]
    assert plain.evict_slots(w, 8, 8, 1, 2) is None and plain.evict_slots(w, 8, -1, 1, 2) is None
    assert plain.evict_slots(w, 8, 2, 1, 2) == "bad"
    assert plain.evict_slots(w, 6, 5, 0, 0) == [0, 1, 2, 3, 5]
