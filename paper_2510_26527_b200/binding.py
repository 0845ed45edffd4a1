"""Python front end of libpolyspec's C ABI (include/polyspec.h): argument marshalling only.

Each function here has the name and the arguments of the C entry point it calls; torch
is used for device memory and streams, nothing is computed in Python.  If the CUDA
library cannot be loaded the functions raise: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpolyspec.so")

OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT, ERR_BAD_INPUT_ON_DEVICE = 1, 2, 3, 4, 5, 6
ERR_SCRATCH_LIMIT, ERR_NO_PAGES = 7, 8
F32, BF16 = 0, 1
MAX_K, MAX_MODELS = 32, 8

EXPORTS = (
    "polyspec_status_string", "polyspec_version", "polyspec_last_cuda_error",
    "polyspec_verify_level_workspace", "polyspec_verify_level",
    "polyspec_verify_chain_workspace", "polyspec_verify_chain",
    "polyspec_chain_row_stats", "polyspec_chain_walk",
    "polyspec_verify_chain_greedy_workspace", "polyspec_verify_chain_greedy",
    "polyspec_verify_chain_host_workspace", "polyspec_verify_chain_host",
    "polyspec_verify_from_hidden_workspace", "polyspec_verify_from_hidden", "polyspec_lm_head",
    "polyspec_from_hidden_project", "polyspec_from_hidden_verify",
    "polyspec_static_scratch_bytes", "polyspec_verify_level_static",
    "polyspec_cost_total_time", "polyspec_cost_insertion", "polyspec_cost_insertion_drafter",
    "polyspec_sharded_level_sizes", "polyspec_sharded_level_stats", "polyspec_sharded_level_decide",
    "polyspec_sharded_level_pick",
    "polyspec_sharded_chain_sizes", "polyspec_sharded_chain_stats", "polyspec_sharded_chain_gather",
    "polyspec_sharded_chain_decide", "polyspec_sharded_chain_pick", "polyspec_sharded_chain_handoff",
    "polyspec_staged_init", "polyspec_staged_round_begin", "polyspec_staged_accumulate", "polyspec_staged_commit",
    "polyspec_pack_quantized", "polyspec_lm_head_quantized", "polyspec_process_logits",
    "polyspec_cache_workspace", "polyspec_cache_init", "polyspec_cache_reserve", "polyspec_cache_rollback", "polyspec_cache_fork",
    "polyspec_cache_compact",
    "polyspec_rotate_heads", "polyspec_prompt_attention", "polyspec_cache_append",
    "polyspec_cache_attention_workspace", "polyspec_cache_attention", "polyspec_cache_weigh",
    "polyspec_cache_evict_workspace", "polyspec_cache_evict",
)


class PolyspecError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        detail = ""
        if status == ERR_CUDA and _lib is not None:
            detail = ": " + _lib.polyspec_last_cuda_error().decode()
        super().__init__(f"{where}: {status_string(status)} (status {status}){detail}")


class ModelLogits(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("rows", ctypes.c_int)]


STAGED_ARRAYS = ("t", "cnt", "rounds", "cycles", "n_committed", "done", "accepted", "committed", "presented", "per_cycle", "remaining")
STAGED_FINISHED, STAGED_EXHAUSTED, STAGED_BAD_INPUT = 1, 2, 3


class StagedState(ctypes.Structure):
    """polyspec_staged_state: sizes, then the device pointers of the state arrays in STAGED_ARRAYS order."""
    _fields_ = [(n, ctypes.c_int) for n in ("B", "K", "mu", "kcap", "N", "R", "C", "cap", "n_tokens")] + \
               [(n, ctypes.c_void_p) for n in STAGED_ARRAYS]


class LogitControls(ctypes.Structure):
    """polyspec_logit_controls."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("history", "history_len", "prompt_len", "repetition", "frequency", "presence",
                                               "bias_tokens", "bias_values", "mask")] + \
               [(n, ctypes.c_int) for n in ("history_cap", "n_bias", "vocab_begin", "vocab_size")]


class CachePagesStruct(ctypes.Structure):
    """polyspec_cache_pages."""
    _fields_ = [(n, ctypes.c_int) for n in ("n_seqs", "max_pages", "n_pages", "page_tokens")] + \
               [(n, ctypes.c_void_p) for n in ("table", "len", "refs", "free_bits")]


class BlockRows(ctypes.Structure):
    """polyspec_block_rows"""
    _fields_ = [("rows_at", ctypes.c_void_p), ("n_rows", ctypes.c_void_p), ("base", ctypes.c_void_p), ("extra", ctypes.c_void_p),
                ("rows", ctypes.c_int)]


class CachePool(ctypes.Structure):
    """polyspec_cache_pool."""
    _fields_ = [("data", ctypes.c_void_p), ("n_planes", ctypes.c_int), ("page_bytes", ctypes.c_size_t)]


CACHE_MAX_POOLS = 8

_lib = None


def load_library() -> ctypes.CDLL:
    """Load libpolyspec.so from the package directory; raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2510_26527_b200.buildlib` "
                           "(needs nvcc); libpolyspec has no CPU fallback")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32p, f32p = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
    ci, cf, sz = ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    szp, cip = ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_int)
    lib.polyspec_status_string.restype = ctypes.c_char_p
    lib.polyspec_status_string.argtypes = [ci]
    lib.polyspec_last_cuda_error.restype = ctypes.c_char_p
    lib.polyspec_last_cuda_error.argtypes = []
    lib.polyspec_version.restype = ci
    lib.polyspec_version.argtypes = []
    lib.polyspec_verify_level_workspace.restype = ci
    lib.polyspec_verify_level_workspace.argtypes = [ci, ci, ci, ci, szp]
    lib.polyspec_verify_level.restype = ci
    lib.polyspec_verify_level.argtypes = [vp, vp, i32p, f32p, i32p, ci, ci, ci, ci, cf,
                                          i32p, i32p, f32p, f32p, i32p, vp, sz, vp]
    lib.polyspec_verify_chain_workspace.restype = ci
    lib.polyspec_verify_chain_workspace.argtypes = [ci, cip, cip, ci, ci, ci, szp]
    lib.polyspec_verify_chain.restype = ci
    lib.polyspec_verify_chain.argtypes = [ctypes.POINTER(ModelLogits), ci, cip, i32p, f32p, ci, ci, ci, cf,
                                          i32p, i32p, i32p, i32p, i32p, vp, sz, vp]
    lib.polyspec_verify_chain_greedy_workspace.restype = ci
    lib.polyspec_verify_chain_greedy_workspace.argtypes = [ci, cip, cip, ci, ci, ci, szp]
    lib.polyspec_verify_chain_greedy.restype = ci
    lib.polyspec_verify_chain_greedy.argtypes = [ctypes.POINTER(ModelLogits), ci, cip, i32p, ci, ci, ci,
                                                 i32p, i32p, i32p, i32p, i32p, vp, sz, vp]
    lib.polyspec_chain_row_stats.restype = ci
    lib.polyspec_chain_row_stats.argtypes = [ctypes.POINTER(ModelLogits), ci, cip, ci, ci, ci, cf, i32p, vp, sz, vp]
    lib.polyspec_chain_walk.restype = ci
    lib.polyspec_chain_walk.argtypes = lib.polyspec_verify_chain.argtypes
    lib.polyspec_verify_chain_host_workspace.restype = ci
    lib.polyspec_verify_chain_host_workspace.argtypes = [ci, cip, cip, ci, ci, ci, szp]
    lib.polyspec_verify_chain_host.restype = ci
    lib.polyspec_verify_chain_host.argtypes = [ctypes.POINTER(ModelLogits), ci, cip, i32p, f32p, ci, ci, ci, cf,
                                               i32p, i32p, i32p, i32p, i32p, vp, sz, vp]
    lib.polyspec_verify_from_hidden_workspace.restype = ci
    lib.polyspec_verify_from_hidden_workspace.argtypes = [ci, ci, ci, ci, ci, szp]
    lib.polyspec_verify_from_hidden.restype = ci
    lib.polyspec_verify_from_hidden.argtypes = [vp, vp, vp, vp, ci, i32p, f32p, i32p, ci, ci, ci, ci, ci, cf,
                                                i32p, i32p, f32p, f32p, i32p, vp, sz, vp]
    lib.polyspec_from_hidden_project.restype = ci
    lib.polyspec_from_hidden_project.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, cf, i32p, vp, sz, vp]
    lib.polyspec_from_hidden_verify.restype = ci
    lib.polyspec_from_hidden_verify.argtypes = [ci, i32p, f32p, i32p, ci, ci, ci, ci, ci, cf, i32p, i32p, f32p, f32p, i32p, vp, sz, vp]
    lib.polyspec_lm_head.restype = ci
    lib.polyspec_lm_head.argtypes = [vp, vp, ci, ci, ci, f32p, i32p, vp]
    lib.polyspec_cost_total_time.restype = ctypes.c_double
    lib.polyspec_cost_total_time.argtypes = [ci, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), ctypes.c_double, ctypes.c_double]
    lib.polyspec_cost_insertion.restype = ci
    lib.polyspec_cost_insertion.argtypes = [ctypes.c_double] * 5 + [ctypes.POINTER(ctypes.c_double)] * 2
    lib.polyspec_cost_insertion_drafter.restype = ci
    lib.polyspec_cost_insertion_drafter.argtypes = [ctypes.c_double] * 5 + [ctypes.POINTER(ctypes.c_double)] * 2
    lib.polyspec_static_scratch_bytes.restype = sz
    lib.polyspec_static_scratch_bytes.argtypes = []
    lib.polyspec_verify_level_static.restype = ci
    lib.polyspec_verify_level_static.argtypes = [vp, vp, i32p, f32p, i32p, ci, ci, ci, ci, cf,
                                                 i32p, i32p, f32p, f32p, i32p, vp]
    lib.polyspec_sharded_level_sizes.restype = ci
    lib.polyspec_sharded_level_sizes.argtypes = [ci, ci, ci, ci, ci, szp, szp, szp]
    lib.polyspec_sharded_level_stats.restype = ci
    lib.polyspec_sharded_level_stats.argtypes = [vp, vp, i32p, ci, ci, ci, ci, ci, ci, cf, vp, i32p, vp, sz, vp]
    lib.polyspec_sharded_level_decide.restype = ci
    lib.polyspec_sharded_level_decide.argtypes = [vp, vp, i32p, f32p, i32p, ci, ci, ci, ci, ci, ci, cf, vp,
                                                  i32p, f32p, f32p, vp, i32p, vp, sz, vp]
    lib.polyspec_sharded_level_pick.restype = ci
    lib.polyspec_sharded_level_pick.argtypes = [vp, vp, f32p, ci, ci, ci, ci, ci, ci, cf, vp, i32p, i32p, vp, sz, vp]
    mlp = ctypes.POINTER(ModelLogits)
    lib.polyspec_sharded_chain_sizes.restype = ci
    lib.polyspec_sharded_chain_sizes.argtypes = [ci, cip, cip, ci, ci, ci, ci, szp, szp, szp, szp]
    lib.polyspec_sharded_chain_stats.restype = ci
    lib.polyspec_sharded_chain_stats.argtypes = [mlp, ci, cip, ci, ci, ci, ci, ci, cf, vp, i32p, vp, sz, vp]
    lib.polyspec_sharded_chain_gather.restype = ci
    lib.polyspec_sharded_chain_gather.argtypes = [mlp, ci, cip, ci, i32p, i32p, ci, ci, ci, ci, ci, vp, vp, sz, vp]
    lib.polyspec_sharded_chain_decide.restype = ci
    lib.polyspec_sharded_chain_decide.argtypes = [mlp, ci, cip, ci, i32p, i32p, f32p, ci, ci, ci, ci, ci, cf, vp, vp, i32p, i32p, vp,
                                                  i32p, vp, sz, vp]
    lib.polyspec_sharded_chain_pick.restype = ci
    lib.polyspec_sharded_chain_pick.argtypes = [mlp, ci, cip, ci, f32p, ci, ci, ci, ci, ci, cf, vp, i32p, i32p, vp, sz, vp]
    lib.polyspec_sharded_chain_handoff.restype = ci
    lib.polyspec_sharded_chain_handoff.argtypes = [ci, cip, ci, ci, i32p, i32p, i32p, i32p, i32p, i32p, vp]
    ssp = ctypes.POINTER(StagedState)
    lib.polyspec_staged_init.restype = ci
    lib.polyspec_staged_init.argtypes = [ssp, vp]
    lib.polyspec_staged_round_begin.restype = ci
    lib.polyspec_staged_round_begin.argtypes = [ssp, i32p, f32p, i32p, i32p, f32p, i32p, vp]
    lib.polyspec_staged_accumulate.restype = ci
    lib.polyspec_staged_accumulate.argtypes = [ssp, i32p, i32p, i32p, i32p, f32p, i32p, i32p, f32p, i32p, vp]
    lib.polyspec_staged_commit.restype = ci
    lib.polyspec_staged_commit.argtypes = [ssp, i32p, i32p, i32p, vp]
    lib.polyspec_pack_quantized.restype = ci
    lib.polyspec_pack_quantized.argtypes = [vp, ci, ci, vp, vp]
    lib.polyspec_lm_head_quantized.restype = ci
    lib.polyspec_lm_head_quantized.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, vp, i32p, vp]
    lib.polyspec_process_logits.restype = ci
    lib.polyspec_process_logits.argtypes = [vp, ctypes.POINTER(LogitControls), i32p, ci, ci, ci, ci, ci, vp, i32p, vp]
    cpp, poolp = ctypes.POINTER(CachePagesStruct), ctypes.POINTER(CachePool)
    lib.polyspec_cache_workspace.restype = ci
    lib.polyspec_cache_workspace.argtypes = [ci, ci, szp]
    lib.polyspec_cache_init.restype = ci
    lib.polyspec_cache_init.argtypes = [cpp, vp]
    lib.polyspec_cache_reserve.restype = ci
    lib.polyspec_cache_reserve.argtypes = [cpp, i32p, i32p, ci, poolp, ci, i32p, vp, sz, vp]
    lib.polyspec_cache_rollback.restype = ci
    lib.polyspec_cache_rollback.argtypes = [cpp, i32p, i32p, ci, i32p, vp]
    lib.polyspec_cache_fork.restype = ci
    lib.polyspec_cache_fork.argtypes = [cpp, i32p, i32p, ci, i32p, vp]
    lib.polyspec_cache_compact.restype = ci
    lib.polyspec_cache_compact.argtypes = [cpp, poolp, ci, i32p, vp, sz, vp]
    brp, ll = ctypes.POINTER(BlockRows), ctypes.c_longlong
    lib.polyspec_rotate_heads.restype = ci
    lib.polyspec_rotate_heads.argtypes = [vp, ll, ci, vp, ll, ci, ci, ci, ci, ci, i32p, f32p, vp, vp, cf, vp, ll, vp, ll, vp]
    lib.polyspec_prompt_attention.restype = ci
    lib.polyspec_prompt_attention.argtypes = [vp, ll, vp, ll, vp, ll, i32p, ci, ci, ci, ci, ci, cf, vp, f32p, i32p, vp]
    lib.polyspec_cache_append.restype = ci
    lib.polyspec_cache_append.argtypes = [cpp, brp, vp, ll, vp, ll, ci, ci, vp, vp, vp, f32p, i32p, vp]
    lib.polyspec_cache_attention_workspace.restype = ci
    lib.polyspec_cache_attention_workspace.argtypes = [ci, ci, ci, szp]
    lib.polyspec_cache_attention.restype = ci
    lib.polyspec_cache_attention.argtypes = [cpp, brp, vp, ll, ci, ci, ci, cf, vp, vp, f32p, i32p, vp, sz, vp]
    lib.polyspec_cache_weigh.restype = ci
    lib.polyspec_cache_weigh.argtypes = [cpp, brp, vp, ll, ci, ci, ci, cf, vp, f32p, cf, f32p, i32p, vp]
    lib.polyspec_cache_evict_workspace.restype = ci
    lib.polyspec_cache_evict_workspace.argtypes = [ci, ci, ci, szp]
    lib.polyspec_cache_evict.restype = ci
    lib.polyspec_cache_evict.argtypes = [cpp, i32p, ci, ci, f32p, vp, ci, ci, ci, i32p, i32p, vp, sz, vp]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().polyspec_status_string(int(status)).decode()


def version() -> int:
    return load_library().polyspec_version()


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"logits must be float32 or bfloat16, got {t.dtype}")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(st: int, where: str):
    if st != OK:
        raise PolyspecError(st, where)


def _dev_check(*tensors):
    for t in tensors:
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("device-pointer arguments must be contiguous CUDA tensors")


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


# ------------------------------------------------------------------ verify_level
def polyspec_verify_level_workspace(B: int, k: int, V: int, dt: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().polyspec_verify_level_workspace(B, k, V, dt, ctypes.byref(n)), "polyspec_verify_level_workspace")
    return n.value


def polyspec_verify_level(logits_p, logits_q, draft_tokens, uniforms, temperature, block_len=None,
                          want_probs=False, workspace=None, out=None, device_status=None, stream=None):
    """One adjacent pair over a batch.  logits_p [B,k+1,V], logits_q [B,k,V], draft_tokens [B,k] int32,
    uniforms [B,k+1] float32; returns device tensors accepted_len [B], next_token [B] (and p_at_draft,
    q_at_draft [B,k] if want_probs) plus the device status word."""
    lib = load_library()
    _dev_check(logits_p, logits_q, draft_tokens, uniforms, block_len)
    B, rows_p, V = logits_p.shape
    k = draft_tokens.shape[1]
    if rows_p != k + 1 or tuple(logits_q.shape) != (B, k, V) or tuple(uniforms.shape) != (B, k + 1):
        raise ValueError("shapes must be logits_p [B,k+1,V], logits_q [B,k,V], draft_tokens [B,k], uniforms [B,k+1]")
    if draft_tokens.dtype != torch.int32 or uniforms.dtype != torch.float32 or logits_q.dtype != logits_p.dtype:
        raise TypeError("draft_tokens int32, uniforms float32, logits_p/logits_q one dtype")
    dev = logits_p.device
    dt = _dt(logits_p)
    if workspace is None:
        workspace = _workspace(polyspec_verify_level_workspace(B, k, V, dt), dev)
    if out is None:
        out = {"accepted_len": torch.empty(B, dtype=torch.int32, device=dev),
               "next_token": torch.empty(B, dtype=torch.int32, device=dev)}
        if want_probs:
            out["p_at_draft"] = torch.empty((B, k), dtype=torch.float32, device=dev)
            out["q_at_draft"] = torch.empty((B, k), dtype=torch.float32, device=dev)
    if device_status is None:
        device_status = torch.zeros(1, dtype=torch.int32, device=dev)
    st = lib.polyspec_verify_level(
        _ptr(logits_p), _ptr(logits_q), _ptr(draft_tokens), _ptr(uniforms), _ptr(block_len),
        B, k, V, dt, float(temperature), _ptr(out["accepted_len"]), _ptr(out["next_token"]),
        _ptr(out.get("p_at_draft")), _ptr(out.get("q_at_draft")), _ptr(device_status),
        _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "polyspec_verify_level")
    out["device_status"] = device_status
    return out


# ------------------------------------------------------------------ verify_chain
def _int_array(vals: Sequence[int]):
    return (ctypes.c_int * len(vals))(*[int(v) for v in vals])


def polyspec_verify_chain_workspace(k: Sequence[int], rows: Sequence[int], B: int, V: int, dt: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().polyspec_verify_chain_workspace(len(rows), _int_array(k), _int_array(rows), B, V, dt, ctypes.byref(n)),
           "polyspec_verify_chain_workspace")
    return n.value


def chain_outputs(L: int, B: int, kmax: int, device, pin=False) -> dict:
    kw = {"dtype": torch.int32, "device": device}
    if pin:
        kw["pin_memory"] = True
    return {"accepted_len": torch.empty((L, B), **kw), "block_len": torch.empty((L, B), **kw),
            "out_tokens": torch.empty((L, B, kmax + 1), **kw), "out_len": torch.empty((L, B), **kw)}


def polyspec_verify_chain(models, k, draft_tokens, uniforms, temperature, workspace=None, out=None,
                          device_status=None, stream=None):
    """n models (models[0] = M_1 ... models[-1] = M_n, each [B, rows_i, V]), n-1 levels verified bottom-up.
    k[l] = largest block level l verifies; draft_tokens [B, k[-1]]; uniforms [n-1, B, max(k)+1]."""
    lib = load_library()
    _dev_check(*models, draft_tokens, uniforms)
    n = len(models)
    L = n - 1
    B, _, V = models[0].shape
    dt = _dt(models[0])
    rows = [int(m.shape[1]) for m in models]
    kmax = max(int(x) for x in k)
    if any(m.dtype != models[0].dtype or m.shape[0] != B or m.shape[2] != V for m in models):
        raise ValueError("all models must share dtype, batch and vocabulary")
    if tuple(uniforms.shape) != (L, B, kmax + 1) or tuple(draft_tokens.shape) != (B, int(k[-1])):
        raise ValueError("uniforms must be [n-1, B, max(k)+1] and draft_tokens [B, k[-1]]")
    if draft_tokens.dtype != torch.int32 or uniforms.dtype != torch.float32:
        raise TypeError("draft_tokens int32, uniforms float32")
    dev = models[0].device
    if workspace is None:
        workspace = _workspace(polyspec_verify_chain_workspace(k, rows, B, V, dt), dev)
    if out is None:
        out = chain_outputs(L, B, kmax, dev)
    if device_status is None:
        device_status = torch.zeros(1, dtype=torch.int32, device=dev)
    arr = (ModelLogits * n)(*[ModelLogits(m.data_ptr(), r) for m, r in zip(models, rows)])
    st = lib.polyspec_verify_chain(arr, n, _int_array(k), _ptr(draft_tokens), _ptr(uniforms), B, V, dt, float(temperature),
                                   _ptr(out["accepted_len"]), _ptr(out["block_len"]), _ptr(out["out_tokens"]),
                                   _ptr(out["out_len"]), _ptr(device_status), _ptr(workspace), workspace.numel(),
                                   _stream(stream))
    _check(st, "polyspec_verify_chain")
    out["device_status"] = device_status
    return out


def polyspec_verify_chain_greedy_workspace(k: Sequence[int], rows: Sequence[int], B: int, V: int, dt: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().polyspec_verify_chain_greedy_workspace(len(rows), _int_array(k), _int_array(rows), B, V, dt, ctypes.byref(n)),
           "polyspec_verify_chain_greedy_workspace")
    return n.value


def polyspec_verify_chain_greedy(models, k, draft_tokens, workspace=None, out=None, device_status=None, stream=None):
    """The chain under greedy matching.  models as in polyspec_verify_chain; the last entry (the drafter's logits)
    is not read and may be None.  Returns the same four outputs plus the device status word."""
    lib = load_library()
    verifiers = list(models[:-1])
    _dev_check(*verifiers, draft_tokens)
    n = len(models)
    L = n - 1
    B, _, V = verifiers[0].shape
    dt = _dt(verifiers[0])
    rows = [int(m.shape[1]) for m in verifiers] + [int(k[-1])]
    kmax = max(int(x) for x in k)
    if any(m.dtype != verifiers[0].dtype or m.shape[0] != B or m.shape[2] != V for m in verifiers):
        raise ValueError("all verifiers must share dtype, batch and vocabulary")
    if tuple(draft_tokens.shape) != (B, int(k[-1])) or draft_tokens.dtype != torch.int32:
        raise ValueError("draft_tokens must be int32 [B, k[-1]]")
    dev = verifiers[0].device
    if workspace is None:
        workspace = _workspace(polyspec_verify_chain_greedy_workspace(k, rows, B, V, dt), dev)
    if out is None:
        out = chain_outputs(L, B, kmax, dev)
    if device_status is None:
        device_status = torch.zeros(1, dtype=torch.int32, device=dev)
    ptrs = [m.data_ptr() for m in verifiers] + [models[-1].data_ptr() if models[-1] is not None else None]
    arr = (ModelLogits * n)(*[ModelLogits(pt, r) for pt, r in zip(ptrs, rows)])
    with torch.cuda.device(dev):
        st = lib.polyspec_verify_chain_greedy(arr, n, _int_array(k), _ptr(draft_tokens), B, V, dt,
                                              _ptr(out["accepted_len"]), _ptr(out["block_len"]), _ptr(out["out_tokens"]),
                                              _ptr(out["out_len"]), _ptr(device_status), _ptr(workspace), workspace.numel(),
                                              _stream(stream))
    _check(st, "polyspec_verify_chain_greedy")
    out["device_status"] = device_status
    return out


class ChainCall:
    """A prepared polyspec_verify_chain call: arguments marshalled once, outputs and workspace allocated once.

    launch() is the single C-ABI call; row_stats() and walk() are its two halves
    (polyspec_chain_row_stats / polyspec_chain_walk)."""

    def __init__(self, models, k, draft_tokens, uniforms, temperature, stream=None):
        self.lib = load_library()
        _dev_check(*models, draft_tokens, uniforms)
        self.models, self.draft_tokens, self.uniforms = list(models), draft_tokens, uniforms
        self.n = len(models)
        self.B, _, self.V = models[0].shape
        self.dt = _dt(models[0])
        self.rows = [int(m.shape[1]) for m in models]
        self.k = [int(x) for x in k]
        self.kmax = max(self.k)
        self.temperature = float(temperature)
        dev = models[0].device
        self.workspace = _workspace(polyspec_verify_chain_workspace(self.k, self.rows, self.B, self.V, self.dt), dev)
        self.out = chain_outputs(self.n - 1, self.B, self.kmax, dev)
        self.device_status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.out["device_status"] = self.device_status
        self._arr = (ModelLogits * self.n)(*[ModelLogits(m.data_ptr(), r) for m, r in zip(models, self.rows)])
        self._k = _int_array(self.k)
        self.stream = stream

    def _tail(self):
        o = self.out
        return (_ptr(o["accepted_len"]), _ptr(o["block_len"]), _ptr(o["out_tokens"]), _ptr(o["out_len"]),
                _ptr(self.device_status), _ptr(self.workspace), self.workspace.numel(), _stream(self.stream))

    def launch(self):
        _check(self.lib.polyspec_verify_chain(self._arr, self.n, self._k, _ptr(self.draft_tokens), _ptr(self.uniforms),
                                              self.B, self.V, self.dt, self.temperature, *self._tail()), "polyspec_verify_chain")
        return self.out

    def row_stats(self):
        _check(self.lib.polyspec_chain_row_stats(self._arr, self.n, self._k, self.B, self.V, self.dt, self.temperature,
                                                 _ptr(self.device_status), _ptr(self.workspace), self.workspace.numel(), _stream(self.stream)),
               "polyspec_chain_row_stats")

    def walk(self):
        _check(self.lib.polyspec_chain_walk(self._arr, self.n, self._k, _ptr(self.draft_tokens), _ptr(self.uniforms),
                                            self.B, self.V, self.dt, self.temperature, *self._tail()), "polyspec_chain_walk")
        return self.out


def polyspec_verify_chain_host_workspace(k: Sequence[int], rows: Sequence[int], B: int, V: int, dt: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().polyspec_verify_chain_host_workspace(len(rows), _int_array(k), _int_array(rows), B, V, dt, ctypes.byref(n)),
           "polyspec_verify_chain_host_workspace")
    return n.value


def polyspec_verify_chain_host(models, k, draft_tokens, uniforms, temperature, workspace, out=None,
                               host_status=None, stream=None):
    """The chain for HOST buffers (CPU tensors, ideally pinned); `workspace` is a device tensor of at least
    polyspec_verify_chain_host_workspace bytes.  Outputs are CPU tensors, valid after the stream synchronises."""
    lib = load_library()
    n = len(models)
    L = n - 1
    B, _, V = models[0].shape
    dt = _dt(models[0])
    rows = [int(m.shape[1]) for m in models]
    kmax = max(int(x) for x in k)
    for t in list(models) + [draft_tokens, uniforms]:
        if t.is_cuda or not t.is_contiguous():
            raise ValueError("polyspec_verify_chain_host takes contiguous CPU tensors")
    if not workspace.is_cuda:
        raise ValueError("the workspace must be a CUDA tensor")
    if out is None:
        out = chain_outputs(L, B, kmax, "cpu", pin=True)
    if host_status is None:
        host_status = torch.zeros(1, dtype=torch.int32, pin_memory=True)
    arr = (ModelLogits * n)(*[ModelLogits(m.data_ptr(), r) for m, r in zip(models, rows)])
    with torch.cuda.device(workspace.device):
        st = lib.polyspec_verify_chain_host(arr, n, _int_array(k), _ptr(draft_tokens), _ptr(uniforms), B, V, dt,
                                            float(temperature), _ptr(out["accepted_len"]), _ptr(out["block_len"]),
                                            _ptr(out["out_tokens"]), _ptr(out["out_len"]), _ptr(host_status),
                                            _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "polyspec_verify_chain_host")
    out["host_status"] = host_status
    return out


# ------------------------------------------------------------------ verify_from_hidden
def polyspec_verify_from_hidden_workspace(B: int, k: int, V: int, d_p: int, d_q: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().polyspec_verify_from_hidden_workspace(B, k, V, d_p, d_q, ctypes.byref(n)),
           "polyspec_verify_from_hidden_workspace")
    return n.value


def polyspec_verify_from_hidden(hidden_p, W_p, hidden_q, W_q, draft_tokens, uniforms, temperature, block_len=None,
                                want_probs=False, workspace=None, out=None, device_status=None, stream=None):
    """verify_level with the LM-head projection fused in front: hidden_p [B,k+1,d_p], W_p [V,d_p],
    hidden_q [B,rows_q>=k,d_q], W_q [V,d_q], all bf16."""
    lib = load_library()
    _dev_check(hidden_p, W_p, hidden_q, W_q, draft_tokens, uniforms, block_len)
    B, rows_p, d_p = hidden_p.shape
    _, rows_q, d_q = hidden_q.shape
    V = W_p.shape[0]
    k = draft_tokens.shape[1]
    if rows_p != k + 1 or W_q.shape[0] != V or W_p.shape[1] != d_p or W_q.shape[1] != d_q or hidden_q.shape[0] != B:
        raise ValueError("shapes must be hidden_p [B,k+1,d_p], W_p [V,d_p], hidden_q [B,rows_q,d_q], W_q [V,d_q]")
    if any(t.dtype != torch.bfloat16 for t in (hidden_p, W_p, hidden_q, W_q)):
        raise TypeError("hidden states and LM-head weights must be bfloat16")
    dev = hidden_p.device
    if workspace is None:
        workspace = _workspace(polyspec_verify_from_hidden_workspace(B, k, V, d_p, d_q), dev)
    if out is None:
        out = {"accepted_len": torch.empty(B, dtype=torch.int32, device=dev),
               "next_token": torch.empty(B, dtype=torch.int32, device=dev)}
        if want_probs:
            out["p_at_draft"] = torch.empty((B, k), dtype=torch.float32, device=dev)
            out["q_at_draft"] = torch.empty((B, k), dtype=torch.float32, device=dev)
    if device_status is None:
        device_status = torch.zeros(1, dtype=torch.int32, device=dev)
    st = lib.polyspec_verify_from_hidden(
        _ptr(hidden_p), _ptr(W_p), _ptr(hidden_q), _ptr(W_q), rows_q, _ptr(draft_tokens), _ptr(uniforms), _ptr(block_len),
        B, k, V, d_p, d_q, float(temperature), _ptr(out["accepted_len"]), _ptr(out["next_token"]),
        _ptr(out.get("p_at_draft")), _ptr(out.get("q_at_draft")), _ptr(device_status),
        _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "polyspec_verify_from_hidden")
    out["device_status"] = device_status
    return out


class FusedCall:
    """A prepared polyspec_verify_from_hidden call: arguments marshalled once, outputs and workspace allocated once.

    launch() is the single C-ABI call; project() and verify() are its two halves
    (polyspec_from_hidden_project / polyspec_from_hidden_verify)."""

    def __init__(self, hidden_p, W_p, hidden_q, W_q, draft_tokens, uniforms, temperature, block_len=None, stream=None):
        self.lib = load_library()
        _dev_check(hidden_p, W_p, hidden_q, W_q, draft_tokens, uniforms, block_len)
        if any(t.dtype != torch.bfloat16 for t in (hidden_p, W_p, hidden_q, W_q)):
            raise TypeError("hidden states and LM-head weights must be bfloat16")
        self.t = (hidden_p, W_p, hidden_q, W_q, draft_tokens, uniforms, block_len)
        self.B, rows_p, self.d_p = hidden_p.shape
        _, self.rows_q, self.d_q = hidden_q.shape
        self.V = W_p.shape[0]
        self.k = draft_tokens.shape[1]
        if rows_p != self.k + 1 or W_q.shape[0] != self.V or W_p.shape[1] != self.d_p or W_q.shape[1] != self.d_q:
            raise ValueError("shapes must be hidden_p [B,k+1,d_p], W_p [V,d_p], hidden_q [B,rows_q,d_q], W_q [V,d_q]")
        self.temperature = float(temperature)
        dev = hidden_p.device
        self.workspace = _workspace(polyspec_verify_from_hidden_workspace(self.B, self.k, self.V, self.d_p, self.d_q), dev)
        self.out = {"accepted_len": torch.empty(self.B, dtype=torch.int32, device=dev),
                    "next_token": torch.empty(self.B, dtype=torch.int32, device=dev)}
        self.device_status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.out["device_status"] = self.device_status
        self.stream = stream

    def _sizes(self):
        return (self.B, self.k, self.V, self.d_p, self.d_q)

    def launch(self):
        hp, wp, hq, wq, tok, u, bl = self.t
        _check(self.lib.polyspec_verify_from_hidden(
            _ptr(hp), _ptr(wp), _ptr(hq), _ptr(wq), self.rows_q, _ptr(tok), _ptr(u), _ptr(bl), *self._sizes(), self.temperature,
            _ptr(self.out["accepted_len"]), _ptr(self.out["next_token"]), None, None, _ptr(self.device_status),
            _ptr(self.workspace), self.workspace.numel(), _stream(self.stream)), "polyspec_verify_from_hidden")
        return self.out

    def project(self):
        hp, wp, hq, wq, _, _, _ = self.t
        _check(self.lib.polyspec_from_hidden_project(
            _ptr(hp), _ptr(wp), _ptr(hq), _ptr(wq), self.rows_q, *self._sizes(), self.temperature, _ptr(self.device_status),
            _ptr(self.workspace), self.workspace.numel(), _stream(self.stream)), "polyspec_from_hidden_project")

    def verify(self):
        _, _, _, _, tok, u, bl = self.t
        _check(self.lib.polyspec_from_hidden_verify(
            self.rows_q, _ptr(tok), _ptr(u), _ptr(bl), *self._sizes(), self.temperature,
            _ptr(self.out["accepted_len"]), _ptr(self.out["next_token"]), None, None, _ptr(self.device_status),
            _ptr(self.workspace), self.workspace.numel(), _stream(self.stream)), "polyspec_from_hidden_verify")
        return self.out


def polyspec_lm_head(hidden, W, out=None, device_status=None, stream=None):
    """The projection alone: hidden [..., d] bf16, W [V, d] bf16 -> fp32 logits [..., V]."""
    lib = load_library()
    _dev_check(hidden, W, out)
    if hidden.dtype != torch.bfloat16 or W.dtype != torch.bfloat16:
        raise TypeError("hidden states and LM-head weights must be bfloat16")
    d = hidden.shape[-1]
    rows = hidden.numel() // d
    V = W.shape[0]
    if W.shape[1] != d:
        raise ValueError("hidden [..., d] and W [V, d] must share d")
    if out is None:
        out = torch.empty(tuple(hidden.shape[:-1]) + (V,), dtype=torch.float32, device=hidden.device)
    if device_status is None:
        device_status = torch.zeros(1, dtype=torch.int32, device=hidden.device)
    with torch.cuda.device(hidden.device):
        st = lib.polyspec_lm_head(_ptr(hidden), _ptr(W), rows, V, d, _ptr(out), _ptr(device_status), _stream(stream))
    _check(st, "polyspec_lm_head")
    return out, device_status


# ------------------------------------------------------------------ verify_level without a workspace
def polyspec_static_scratch_bytes() -> int:
    return int(load_library().polyspec_static_scratch_bytes())


def polyspec_verify_level_static(logits_p, logits_q, draft_tokens, uniforms, temperature, out, block_len=None,
                                 device_status=None, stream=None):
    """polyspec_verify_level for callers that cannot allocate device memory: no workspace is passed, the
    library's built-in scratch array is used, and this wrapper allocates nothing either -- `out` must hold
    the caller's own accepted_len / next_token (and optionally p_at_draft / q_at_draft) device tensors.
    Raises PolyspecError(ERR_SCRATCH_LIMIT) when the problem needs more than polyspec_static_scratch_bytes()."""
    lib = load_library()
    _dev_check(logits_p, logits_q, draft_tokens, uniforms, block_len)
    B, rows_p, V = logits_p.shape
    k = draft_tokens.shape[1]
    if rows_p != k + 1 or tuple(logits_q.shape) != (B, k, V) or tuple(uniforms.shape) != (B, k + 1):
        raise ValueError("shapes must be logits_p [B,k+1,V], logits_q [B,k,V], draft_tokens [B,k], uniforms [B,k+1]")
    with torch.cuda.device(logits_p.device):
        st = lib.polyspec_verify_level_static(
            _ptr(logits_p), _ptr(logits_q), _ptr(draft_tokens), _ptr(uniforms), _ptr(block_len),
            B, k, V, _dt(logits_p), float(temperature), _ptr(out["accepted_len"]), _ptr(out["next_token"]),
            _ptr(out.get("p_at_draft")), _ptr(out.get("q_at_draft")), _ptr(device_status), _stream(stream))
    _check(st, "polyspec_verify_level_static")
    return out


# ------------------------------------------------------------------ cost model (host arithmetic)
def polyspec_cost_total_time(T: Sequence[float], L: Sequence[float], beta: float, N: float) -> float:
    """Lemma 3.1 (Eq. 3): T = sum_{i<n} (N / L_i) T_i + beta (N / L_{n-1}) T_n."""
    n = len(T)
    if len(L) != n - 1:
        raise ValueError("L must hold n - 1 acceptance lengths")
    Ta = (ctypes.c_double * n)(*[float(x) for x in T])
    La = (ctypes.c_double * max(n - 1, 1))(*[float(x) for x in L])
    return float(load_library().polyspec_cost_total_time(n, Ta, La, float(beta), float(N)))


def polyspec_cost_insertion(T_new: float, T_i: float, L_new: float, L_i: float, L_i_new: float):
    """Theorem 3.2, first condition: (improves, T_new / T_i, L_new (1 / L_i - 1 / L_{i-new}))."""
    lhs, rhs = ctypes.c_double(0.0), ctypes.c_double(0.0)
    r = load_library().polyspec_cost_insertion(float(T_new), float(T_i), float(L_new), float(L_i), float(L_i_new),
                                               ctypes.byref(lhs), ctypes.byref(rhs))
    if r < 0:
        raise ValueError("all five quantities must be positive")
    return bool(r), lhs.value, rhs.value


def polyspec_cost_insertion_drafter(T_new: float, T_next: float, L_new: float, L_i: float, beta: float):
    """Theorem 3.2, second condition (as its proof derives it): (improves, T_new / T_{i+1}, beta (L_new / L_i - 1))."""
    lhs, rhs = ctypes.c_double(0.0), ctypes.c_double(0.0)
    r = load_library().polyspec_cost_insertion_drafter(float(T_new), float(T_next), float(L_new), float(L_i), float(beta),
                                                       ctypes.byref(lhs), ctypes.byref(rhs))
    if r < 0:
        raise ValueError("all five quantities must be positive")
    return bool(r), lhs.value, rhs.value


# ------------------------------------------------------------------ one level, vocabulary sharded over ranks
def polyspec_sharded_level_sizes(B: int, k: int, V_local: int, dt: int, n_ranks: int):
    """(workspace bytes, stats record bytes, mass record bytes) of the sharded level calls."""
    w, a, m = ctypes.c_size_t(0), ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(load_library().polyspec_sharded_level_sizes(B, k, V_local, dt, n_ranks, ctypes.byref(w), ctypes.byref(a), ctypes.byref(m)),
           "polyspec_sharded_level_sizes")
    return w.value, a.value, m.value


class ShardedLevelCall:
    """One rank's side of a vocabulary-sharded level: its slices of the logits, its workspace and records.

    stats() -> this rank's stats record; decide(all ranks' stats records) -> (accepted_len, this rank's mass
    record); pick(all ranks' mass records) -> next_token, -1 unless this rank's slice holds the token.  The
    exchanges between the calls are the caller's (see paper_2510_26527_b200.sharded)."""

    def __init__(self, logits_p, logits_q, draft_tokens, uniforms, temperature, rank, n_ranks, block_len=None,
                 want_probs=False, stream=None):
        self.lib = load_library()
        _dev_check(logits_p, logits_q, draft_tokens, uniforms, block_len)
        self.B, rows_p, self.V_local = logits_p.shape
        self.k = int(draft_tokens.shape[1])
        if rows_p != self.k + 1 or tuple(logits_q.shape) != (self.B, self.k, self.V_local) or logits_q.dtype != logits_p.dtype:
            raise ValueError("shapes must be logits_p [B,k+1,V_local], logits_q [B,k,V_local] of one dtype")
        self.dt = _dt(logits_p)
        self.t = (logits_p, logits_q, draft_tokens, uniforms, block_len)
        self.rank, self.n_ranks = int(rank), int(n_ranks)
        self.temperature = float(temperature)
        dev = logits_p.device
        wbytes, self.stats_bytes, self.mass_bytes = polyspec_sharded_level_sizes(self.B, self.k, self.V_local, self.dt, self.n_ranks)
        self.workspace = _workspace(wbytes, dev)
        self.stats_record = torch.zeros(self.stats_bytes, dtype=torch.uint8, device=dev)
        self.mass_record = torch.zeros(self.mass_bytes, dtype=torch.uint8, device=dev)
        self.accepted_len = torch.empty(self.B, dtype=torch.int32, device=dev)
        self.next_token = torch.empty(self.B, dtype=torch.int32, device=dev)
        self.p_at = torch.zeros((self.B, self.k), dtype=torch.float32, device=dev) if want_probs else None
        self.q_at = torch.zeros((self.B, self.k), dtype=torch.float32, device=dev) if want_probs else None
        self.device_status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.stream = stream

    def _sizes(self):
        return (self.B, self.k, self.V_local, self.rank, self.n_ranks, self.dt, self.temperature)

    def _tail(self):
        return (_ptr(self.device_status), _ptr(self.workspace), self.workspace.numel(), _stream(self.stream))

    def stats(self):
        lp, lq, tok, _, _ = self.t
        _check(self.lib.polyspec_sharded_level_stats(_ptr(lp), _ptr(lq), _ptr(tok), *self._sizes(), _ptr(self.stats_record), *self._tail()),
               "polyspec_sharded_level_stats")
        return self.stats_record

    def decide(self, stats_records):
        lp, lq, tok, u, bl = self.t
        _dev_check(stats_records)
        if stats_records.numel() != self.n_ranks * self.stats_bytes:
            raise ValueError("need every rank's stats record, in rank order")
        _check(self.lib.polyspec_sharded_level_decide(_ptr(lp), _ptr(lq), _ptr(tok), _ptr(u), _ptr(bl), *self._sizes(), _ptr(stats_records),
                                                      _ptr(self.accepted_len), _ptr(self.p_at), _ptr(self.q_at), _ptr(self.mass_record),
                                                      *self._tail()), "polyspec_sharded_level_decide")
        return self.accepted_len, self.mass_record

    def pick(self, mass_records):
        lp, lq, _, u, _ = self.t
        _dev_check(mass_records)
        if mass_records.numel() != self.n_ranks * self.mass_bytes:
            raise ValueError("need every rank's mass record, in rank order")
        _check(self.lib.polyspec_sharded_level_pick(_ptr(lp), _ptr(lq), _ptr(u), *self._sizes(), _ptr(mass_records), _ptr(self.next_token),
                                                    *self._tail()), "polyspec_sharded_level_pick")
        return self.next_token


def polyspec_sharded_chain_sizes(k: Sequence[int], rows: Sequence[int], B: int, V_local: int, dt: int, n_ranks: int):
    """(workspace, stats record, gather record, mass record) bytes of the sharded chain calls."""
    w, a, g, m = (ctypes.c_size_t(0) for _ in range(4))
    _check(load_library().polyspec_sharded_chain_sizes(len(rows), _int_array(k), _int_array(rows), B, V_local, dt, n_ranks,
                                                       ctypes.byref(w), ctypes.byref(a), ctypes.byref(g), ctypes.byref(m)),
           "polyspec_sharded_chain_sizes")
    return w.value, a.value, g.value, m.value


class ShardedChainCall:
    """One rank's side of a vocabulary-sharded chain: its slices of every model's logits, its workspace, records,
    the block being verified and the chain's outputs (identical on every rank once a level is handed off).

    stats() once; then per level, bottom-up: gather(level), decide(level, stats records, gather records),
    pick(level, mass records), handoff(level, token after the max over ranks)."""

    def __init__(self, models, k, draft_tokens, uniforms, temperature, rank, n_ranks, stream=None):
        self.lib = load_library()
        _dev_check(*models, draft_tokens, uniforms)
        self.models = list(models)
        self.n = len(models)
        self.L = self.n - 1
        self.B, _, self.V_local = models[0].shape
        self.dt = _dt(models[0])
        self.rows = [int(m.shape[1]) for m in models]
        self.k = [int(x) for x in k]
        self.kmax = max(self.k)
        if any(m.dtype != models[0].dtype or m.shape[0] != self.B or m.shape[2] != self.V_local for m in models):
            raise ValueError("every model's slice must be [B, rows, V_local] of one dtype")
        if tuple(draft_tokens.shape) != (self.B, self.k[-1]) or tuple(uniforms.shape) != (self.L, self.B, self.kmax + 1):
            raise ValueError("shapes must be draft_tokens [B, k[-1]], uniforms [n_models-1, B, kmax+1]")
        self.rank, self.n_ranks = int(rank), int(n_ranks)
        self.temperature = float(temperature)
        self.uniforms = uniforms
        dev = models[0].device
        wbytes, self.stats_bytes, self.gather_bytes, self.mass_bytes = polyspec_sharded_chain_sizes(
            self.k, self.rows, self.B, self.V_local, self.dt, self.n_ranks)
        self.workspace = _workspace(wbytes, dev)
        self.stats_record = torch.zeros(self.stats_bytes, dtype=torch.uint8, device=dev)
        self.gather_record = torch.zeros(self.gather_bytes, dtype=torch.uint8, device=dev)
        self.mass_record = torch.zeros(self.mass_bytes, dtype=torch.uint8, device=dev)
        self.block_tokens = torch.full((self.B, self.kmax + 1), -1, dtype=torch.int32, device=dev)
        self.block_tokens[:, : self.k[-1]] = draft_tokens
        self.block_len = torch.full((self.B,), self.k[-1], dtype=torch.int32, device=dev)
        self.next_token = torch.empty(self.B, dtype=torch.int32, device=dev)
        self.out = chain_outputs(self.L, self.B, self.kmax, dev)
        self.device_status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.out["device_status"] = self.device_status
        self._arr = (ModelLogits * self.n)(*[ModelLogits(m.data_ptr(), r) for m, r in zip(models, self.rows)])
        self._k = _int_array(self.k)
        self.stream = stream

    def _head(self):
        return (self._arr, self.n, self._k)

    def _geom(self):
        return (self.B, self.V_local, self.rank, self.n_ranks, self.dt)

    def _ws(self):
        return (_ptr(self.workspace), self.workspace.numel(), _stream(self.stream))

    def stats(self):
        _check(self.lib.polyspec_sharded_chain_stats(*self._head(), *self._geom(), self.temperature, _ptr(self.stats_record),
                                                     _ptr(self.device_status), *self._ws()), "polyspec_sharded_chain_stats")
        return self.stats_record

    def gather(self, level):
        _check(self.lib.polyspec_sharded_chain_gather(*self._head(), level, _ptr(self.block_tokens), _ptr(self.block_len), *self._geom(),
                                                      _ptr(self.gather_record), *self._ws()), "polyspec_sharded_chain_gather")
        return self.gather_record

    def decide(self, level, stats_records, gather_records):
        _dev_check(stats_records, gather_records)
        if stats_records.numel() != self.n_ranks * self.stats_bytes or gather_records.numel() != self.n_ranks * self.gather_bytes:
            raise ValueError("need every rank's records, in rank order")
        _check(self.lib.polyspec_sharded_chain_decide(*self._head(), level, _ptr(self.block_tokens), _ptr(self.block_len), _ptr(self.uniforms),
                                                      *self._geom(), self.temperature, _ptr(stats_records), _ptr(gather_records),
                                                      _ptr(self.out["accepted_len"]), _ptr(self.out["block_len"]), _ptr(self.mass_record),
                                                      _ptr(self.device_status), *self._ws()), "polyspec_sharded_chain_decide")
        return self.mass_record

    def pick(self, level, mass_records):
        _dev_check(mass_records)
        if mass_records.numel() != self.n_ranks * self.mass_bytes:
            raise ValueError("need every rank's mass record, in rank order")
        _check(self.lib.polyspec_sharded_chain_pick(*self._head(), level, _ptr(self.uniforms), *self._geom(), self.temperature,
                                                    _ptr(mass_records), _ptr(self.next_token), _ptr(self.device_status), *self._ws()),
               "polyspec_sharded_chain_pick")
        return self.next_token

    def handoff(self, level, token):
        _dev_check(token)
        _check(self.lib.polyspec_sharded_chain_handoff(self.n, self._k, level, self.B, _ptr(self.out["accepted_len"]), _ptr(token),
                                                       _ptr(self.block_tokens), _ptr(self.block_len), _ptr(self.out["out_tokens"]),
                                                       _ptr(self.out["out_len"]), _stream(self.stream)), "polyspec_sharded_chain_handoff")


# ------------------------------------------------------------------ 4-bit LM head, sampling controls, cache pages
# These calls are short on the device (a few microseconds for one sequence), so the checks below read each tensor's device,
# layout and type once and nothing else.
def _one_device(*tensors) -> int:
    """The one CUDA device all tensors are on, each contiguous."""
    dev = -1
    for t in tensors:
        if t is not None:
            d = t.get_device()
            if d < 0 or not t.is_contiguous():
                raise ValueError("device-pointer arguments must be contiguous CUDA tensors")
            if d != dev:
                if dev >= 0:
                    raise ValueError("all tensors of a call must be on one device")
                dev = d
    return dev


def _expect(name, t, dtype, shape=None):
    if t is not None:
        if t.dtype is not dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if shape is not None and t.shape != shape:
            raise ValueError(f"shapes do not fit: {name} must be {list(shape)}, got {list(t.shape)}")


def _on_stream(stream, dev: int):
    """Context in which allocations belong to `stream` (a torch stream or a raw handle) of device `dev`."""
    if stream is None:
        return torch.cuda.device(dev)
    if not isinstance(stream, torch.cuda.Stream):
        handle = _stream(stream)
        # cudaStreamLegacy (1) is the default stream by another name, which torch refuses as an external one
        stream = torch.cuda.ExternalStream(0 if handle == 1 else handle, device=torch.device("cuda", dev))
    return torch.cuda.stream(stream)


@functools.lru_cache(maxsize=None)
def _device(dev: int) -> torch.device:
    return torch.device("cuda", dev)


def _empty(shape, dtype, dev: int, stream) -> torch.Tensor:
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=_device(dev))
    with _on_stream(stream, dev):
        return torch.empty(shape, dtype=dtype, device=_device(dev))


def _handle(stream, dev: int) -> int:
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream(stream)


_status_words = {}          # (device, stream) -> status words zeroed on that stream and not handed out yet


def _status_word(device_status, dev: int, stream) -> torch.Tensor:
    """The caller's status word, or a fresh zeroed one.  Fresh ones are zeroed 256 at a time; while a graph is captured, and for a
    stream other than the current one, each is a tensor of its own (a graph keeps alive what is allocated during its capture)."""
    if device_status is not None:
        return device_status
    if stream is not None:
        with _on_stream(stream, dev):
            return torch.zeros(1, dtype=torch.int32, device=torch.device("cuda", dev))
    if torch._C._cuda_isCurrentStreamCapturing():
        return torch.zeros(1, dtype=torch.int32, device=torch.device("cuda", dev))
    key = (dev, torch._C._cuda_getCurrentRawStream(dev))
    try:
        return _status_words[key].pop()
    except (KeyError, IndexError):
        with torch.inference_mode(False):       # words outlive the mode they are made under: later callers may write to theirs
            words = list(torch.zeros(256, dtype=torch.int32, device=torch.device("cuda", dev)).split(1))
        word = words.pop()
        _status_words[key] = words
        return word


def _call(where: str, fn, dev: int, *args):
    """fn(*args) with device `dev` current."""
    if torch._C._cuda_getDevice() == dev:
        st = fn(*args)
    else:
        with torch.cuda.device(dev):
            st = fn(*args)
    if st != OK:
        raise PolyspecError(st, where)


def polyspec_pack_quantized(codes, out=None, stream=None):
    """codes [V, d] uint8 (one 4-bit code per byte, d a multiple of 32) -> qweight [V, d/8] int32, the words
    polyspec_lm_head_quantized reads."""
    V, d = codes.shape
    _expect("codes", codes, torch.uint8)
    _expect("out", out, torch.int32, (V, d // 8))
    dev = _one_device(codes, out)
    if out is None:
        out = _empty((V, d // 8), torch.int32, dev, stream)
    _call("polyspec_pack_quantized", load_library().polyspec_pack_quantized, dev, codes.data_ptr(), V, d, out.data_ptr(), _handle(stream, dev))
    return out


def polyspec_lm_head_quantized(hidden, qweight, scales, zero_points=None, out=None, out_dtype=torch.float32, device_status=None, stream=None):
    """logits[r, v] = sum_d hidden[r, d] * scales[v, d // group] * (code[v, d] - zero_point[v, d // group]).

    hidden [rows, d] bf16, qweight [V, d/8] int32 (polyspec_pack_quantized), scales [V, d/group] bf16, zero_points
    [V, d/group] uint8 or None (8 everywhere); out [rows, V] fp32 or bf16 (out_dtype, where out is not given).
    Returns (out, status word)."""
    rows, d = hidden.shape
    V, groups = scales.shape
    _expect("hidden", hidden, torch.bfloat16)
    _expect("scales", scales, torch.bfloat16)
    _expect("qweight", qweight, torch.int32)
    _expect("zero_points", zero_points, torch.uint8)
    if qweight.shape != (V, d // 8) or groups < 1 or d % groups or (zero_points is not None and zero_points.shape != scales.shape):
        raise ValueError("shapes must be hidden [rows,d], qweight [V,d/8], scales [V,d/group], zero_points [V,d/group]")
    _expect("device_status", device_status, torch.int32)
    dev = _one_device(hidden, qweight, scales, zero_points, out, device_status)
    if out is None:
        out = _empty((rows, V), out_dtype, dev, stream)
    elif out.shape != (rows, V):
        raise ValueError("out must be [rows, V]")
    dt = _dt(out)
    device_status = _status_word(device_status, dev, stream)
    _call("polyspec_lm_head_quantized", load_library().polyspec_lm_head_quantized, dev, hidden.data_ptr(), qweight.data_ptr(),
          scales.data_ptr(), _ptr(zero_points), rows, V, d, d // groups, dt, out.data_ptr(), device_status.data_ptr(), _handle(stream, dev))
    return out, device_status


def polyspec_process_logits(logits, draft_tokens=None, history=None, history_len=None, prompt_len=None, repetition=None, frequency=None,
                            presence=None, bias_tokens=None, bias_values=None, mask=None, out=None, vocab_begin=0, vocab_size=0,
                            device_status=None, stream=None):
    """Sampling controls on logits [B, rows, V] of a block: penalties for repeated tokens, biases, allowed-token masks; row j has
    the history and draft_tokens[:, :j] as its context.

    draft_tokens [B, k >= rows-1], history [B, cap], history_len and prompt_len [B], bias_tokens [B, n]: int32; repetition,
    frequency, presence [B], bias_values [B, n]: float32; mask [B, rows, ceil(V/32)] int32 (bit v % 32 of word v // 32 set:
    allowed).  out: a tensor of its own (made if None) or logits itself.  Returns (out, status word)."""
    if logits.dim() != 3:
        raise ValueError("logits must be [B, rows, V]")
    B, rows, V = logits.shape
    dt = _dt(logits)
    i32, f32, per_seq = torch.int32, torch.float32, (B,)
    k = cap = n_bias = 0
    if draft_tokens is not None:
        k = draft_tokens.shape[-1]
        _expect("draft_tokens", draft_tokens, i32, (B, k))
    if history is not None:
        cap = history.shape[-1]
        _expect("history", history, i32, (B, cap))
        _expect("history_len", history_len, i32, per_seq)
        _expect("prompt_len", prompt_len, i32, per_seq)
        if cap == 0:
            history = history_len = prompt_len = None
    elif history_len is not None or prompt_len is not None:
        raise ValueError("history_len and prompt_len need a history")
    _expect("repetition", repetition, f32, per_seq)
    _expect("frequency", frequency, f32, per_seq)
    _expect("presence", presence, f32, per_seq)
    if (bias_tokens is None) != (bias_values is None):
        raise ValueError("bias_tokens and bias_values go together")
    if bias_tokens is not None:
        n_bias = bias_tokens.shape[-1]
        _expect("bias_tokens", bias_tokens, i32, (B, n_bias))
        _expect("bias_values", bias_values, f32, (B, n_bias))
        if n_bias == 0:
            bias_tokens = bias_values = None
    _expect("mask", mask, i32, (B, rows, (V + 31) // 32))
    _expect("out", out, logits.dtype, logits.shape)
    _expect("device_status", device_status, torch.int32)
    dev = _one_device(logits, draft_tokens, history, history_len, prompt_len, repetition, frequency, presence, bias_tokens, bias_values,
                      mask, out, device_status)
    if out is None:
        out = _empty(logits.shape, logits.dtype, dev, stream)
    device_status = _status_word(device_status, dev, stream)
    c = LogitControls(_ptr(history), _ptr(history_len), _ptr(prompt_len), _ptr(repetition), _ptr(frequency), _ptr(presence),
                      _ptr(bias_tokens), _ptr(bias_values), _ptr(mask), cap, n_bias, vocab_begin, vocab_size)
    _call("polyspec_process_logits", load_library().polyspec_process_logits, dev, logits.data_ptr(), c, _ptr(draft_tokens), k, B, rows, V,
          dt, out.data_ptr(), device_status.data_ptr(), _handle(stream, dev))
    return out, device_status


def polyspec_cache_workspace(n_seqs: int, n_pages: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().polyspec_cache_workspace(n_seqs, n_pages, n), "polyspec_cache_workspace")
    return n.value


class CachePages:
    """Page tables of one model's cache: table [n_seqs, max_pages], len [n_seqs], refs [n_pages] (int32) and free_bits
    [ceil(n_pages/32)] (int32), on the device.  CachePages.new allocates and initialises them; the constructor takes tensors
    that hold a state already.  The calls' workspace is allocated at the first call that needs one and belongs to the state:
    calls on one state are ordered anyway.  Streams of torch's own that it is used on besides the one it was allocated on are
    recorded, so that its memory is not handed out again before their work is done; for raw handles and external streams, which may be
    destroyed before the state is, and for the state's tensors that is the caller's to see to."""

    def __init__(self, table, len, refs, free_bits, page_tokens):
        i32 = torch.int32
        if table.dtype is not i32 or len.dtype is not i32 or refs.dtype is not i32 or free_bits.dtype is not i32:
            raise TypeError("table, len, refs and free_bits must be int32")
        n_seqs, max_pages = table.shape
        n_pages = refs.numel()
        if len.shape != (n_seqs,) or refs.dim() != 1 or free_bits.shape != ((n_pages + 31) // 32,):
            raise ValueError("shapes must be table [n_seqs,max_pages], len [n_seqs], refs [n_pages], free_bits [ceil(n_pages/32)]")
        self.dev = _one_device(table, len, refs, free_bits)
        self.table, self.len, self.refs, self.free_bits = table, len, refs, free_bits
        self.n_seqs, self.max_pages, self.n_pages, self.page_tokens = n_seqs, max_pages, n_pages, int(page_tokens)
        self.c = CachePagesStruct(n_seqs, max_pages, n_pages, self.page_tokens, table.data_ptr(), len.data_ptr(), refs.data_ptr(),
                                  free_bits.data_ptr())
        self._workspace, self._workspace_streams = None, set()          # the streams it belongs to: allocated on, recorded

    @classmethod
    def new(cls, n_seqs, max_pages, n_pages, page_tokens, device="cuda", stream=None):
        device = torch.empty(0, device=device).device
        i32 = lambda *shape: _empty(shape, torch.int32, device.index, stream)
        pages = cls(i32(n_seqs, max_pages), i32(n_seqs), i32(n_pages), i32((n_pages + 31) // 32), page_tokens)
        _call("polyspec_cache_init", load_library().polyspec_cache_init, pages.dev, pages.c, _handle(stream, pages.dev))
        return pages

    def workspace(self, stream=None):
        handle = _handle(stream, self.dev)
        if self._workspace is None:
            self._workspace = _empty(polyspec_cache_workspace(self.n_seqs, self.n_pages), torch.uint8, self.dev, stream)
            self._workspace_streams = {handle}
        elif handle not in self._workspace_streams and (stream is None or isinstance(stream, torch.cuda.Stream)):
            used = torch.cuda.current_stream(self.dev) if stream is None else stream
            if handle == 0 or used.stream_id != handle:     # an external stream's id is its handle
                self._workspace.record_stream(used)
                self._workspace_streams.add(handle)
        return self._workspace


def _same_device(pages, *tensors):
    dev = _one_device(*tensors)
    if dev >= 0 and dev != pages.dev:
        raise ValueError("all tensors of a call must be on one device")
    return pages.dev


def _targets(pages, base, extra):
    if base.dtype is not torch.int32 or (extra is not None and extra.dtype is not torch.int32):
        raise TypeError("base and extra must be int32")
    n = (pages.n_seqs,)
    if base.shape != n or (extra is not None and extra.shape != n):
        raise ValueError("base and extra must be [n_seqs]")


def _pools(pages, pools):
    """pools: tensors [n_planes, n_pages, ...], each plane's page contiguous."""
    if len(pools) > CACHE_MAX_POOLS:
        raise ValueError(f"at most {CACHE_MAX_POOLS} pools")
    for t in pools:
        if t.dim() < 3 or t.shape[0] < 1 or t.shape[1] != pages.n_pages:
            raise ValueError("a pool must be [n_planes, n_pages, ...]")
    # (a stride says nothing of a dimension of size 1, so the size of a page is not read from it)
    return (CachePool * len(pools))(*[CachePool(t.data_ptr(), t.shape[0], t.nbytes // (t.shape[0] * t.shape[1])) for t in pools]) if pools else None


def polyspec_cache_reserve(pages, base, extra=None, plus=0, pools=(), device_status=None, workspace=None, stream=None):
    """Grow every sequence to base[b] + extra[b] + plus tokens; a last page that others hold too is replaced by a copy of its
    own, in every pool ([n_planes, n_pages, ...] tensors).  pages.len tells what was granted.  Returns the status word."""
    _targets(pages, base, extra)
    _expect("device_status", device_status, torch.int32)
    dev = _same_device(pages, base, extra, workspace, device_status, *pools)
    if workspace is None:
        workspace = pages.workspace(stream)
    device_status = _status_word(device_status, dev, stream)
    _call("polyspec_cache_reserve", load_library().polyspec_cache_reserve, dev, pages.c, base.data_ptr(), _ptr(extra), plus,
          _pools(pages, pools), len(pools), device_status.data_ptr(), workspace.data_ptr(), workspace.nbytes, _handle(stream, dev))
    return device_status


def polyspec_cache_rollback(pages, base, extra=None, plus=0, device_status=None, stream=None):
    """Let every sequence fall back to base[b] + extra[b] + plus tokens (never up); returns the status word."""
    _targets(pages, base, extra)
    _expect("device_status", device_status, torch.int32)
    dev = _same_device(pages, base, extra, device_status)
    device_status = _status_word(device_status, dev, stream)
    _call("polyspec_cache_rollback", load_library().polyspec_cache_rollback, dev, pages.c, base.data_ptr(), _ptr(extra), plus,
          device_status.data_ptr(), _handle(stream, dev))
    return device_status


def polyspec_cache_fork(pages, src, dst, device_status=None, stream=None):
    """Sequence dst[i], which holds nothing, becomes a copy of src[i] on the same pages; returns the status word."""
    n = src.numel()
    _expect("src", src, torch.int32, (n,))
    _expect("dst", dst, torch.int32, (n,))
    _expect("device_status", device_status, torch.int32)
    dev = _same_device(pages, src, dst, device_status)
    device_status = _status_word(device_status, dev, stream)
    _call("polyspec_cache_fork", load_library().polyspec_cache_fork, dev, pages.c, src.data_ptr(), dst.data_ptr(), n,
          device_status.data_ptr(), _handle(stream, dev))
    return device_status


def polyspec_cache_compact(pages, pools=(), moved_to=None, workspace=None, stream=None):
    """Renumber the pages in use to 0 .. n_live-1, moving their contents in every pool; moved_to [n_pages] int32 takes the new
    numbers (-1 for free pages)."""
    _expect("moved_to", moved_to, torch.int32, (pages.n_pages,))
    dev = _same_device(pages, moved_to, workspace, *pools)
    if workspace is None:
        workspace = pages.workspace(stream)
    _call("polyspec_cache_compact", load_library().polyspec_cache_compact, dev, pages.c, _pools(pages, pools), len(pools), _ptr(moved_to),
          workspace.data_ptr(), workspace.nbytes, _handle(stream, dev))


# ------------------------------------------------------------------ a model's attention around the cache pages
# (Short calls again: each tensor's type, shape, strides and device are read once.)
_BF16, _F32T, _I32T = torch.bfloat16, torch.float32, torch.int32


def _head_rows(name, t, shape, dev):
    """Checks rows of heads, [rows, heads, head_dim] bf16 whose rows may lie apart (parts of a fused projection), of a given shape or (None) any;
    dev: the device of the call's other tensors, -1 for the first.  Returns (row stride, device)."""
    if t.dtype is not _BF16:
        raise TypeError(f"{name} must be torch.bfloat16, got {t.dtype}")
    size = t.shape
    if len(size) != 3 or (shape is not None and size != shape):
        raise ValueError(f"shapes do not fit: {name} must be {'[rows, heads, head_dim]' if shape is None else list(shape)}, got {list(size)}")
    stride, at = t.stride(), t.get_device()
    # (a stride says nothing of a dimension of size 1)
    if at < 0 or (stride[2] != 1 and size[2] > 1) or (stride[1] != size[2] and size[1] > 1):
        raise ValueError(f"{name} must be a CUDA tensor with the heads of a row behind one another")
    if at != dev and dev >= 0:
        raise ValueError("all tensors of a call must be on one device")
    return (stride[0] if size[0] > 1 else size[1] * size[2]), at


def _flat(name, t, dtype, shape, dev):
    """Checks a contiguous tensor of a call on device dev; returns its address, None for None."""
    if t is None:
        return None
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"shapes do not fit: {name} must be {list(shape)}, got {list(t.shape)}")
    if t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor on the device of the call's other tensors")
    return t.data_ptr()


def polyspec_rotate_heads(q, k, positions, frequencies, q_weight=None, k_weight=None, interleaved=False, eps=1e-6, q_out=None, k_out=None, stream=None):
    """RMS norm (where weights are given) of every head of q [rows, q_heads, d] and k [rows, kv_heads, d] (or None), then the rotation of the
    first 2 * len(frequencies) elements by positions[row] * frequencies[i].

    bf16; rows may lie apart, as parts of one projection's rows do.  positions [rows] int32, frequencies [rotary/2] fp32, weights [d] bf16.
    q_out, k_out: tensors of their own (made if None) or q and k themselves.  Returns (q_out, k_out)."""
    qs, dev = _head_rows("q", q, None, -1)
    shape = rows, heads, d = q.shape
    ks = kv_heads = kos = rotary = 0
    k_ptr = k_out_ptr = None
    if frequencies is not None:
        rotary = 2 * frequencies.numel()
        if positions is None:
            raise ValueError("frequencies need positions")
    if q_out is None:
        q_out = _empty(shape, _BF16, dev, stream)
    qos = _head_rows("q_out", q_out, shape, dev)[0]
    if k is not None:
        ks = _head_rows("k", k, None, dev)[0]
        k_shape = k.shape
        kv_heads = k_shape[1]
        if k_shape[0] != rows or k_shape[2] != d:
            raise ValueError("shapes do not fit: k must be [rows, kv_heads, head_dim]")
        if k_out is None:
            k_out = _empty(k_shape, _BF16, dev, stream)
        kos = _head_rows("k_out", k_out, k_shape, dev)[0]
        k_ptr, k_out_ptr = k.data_ptr(), k_out.data_ptr()
    elif k_out is not None:
        raise ValueError("k_out needs k")
    _call("polyspec_rotate_heads", load_library().polyspec_rotate_heads, dev, q.data_ptr(), qs, heads, k_ptr, ks, kv_heads, rows, d, rotary,
          1 if interleaved else 0, _flat("positions", positions, _I32T, (rows,), dev) if rotary else None,
          _flat("frequencies", frequencies, _F32T, (rotary // 2,), dev) if rotary else None, _flat("q_weight", q_weight, _BF16, (d,), dev),
          _flat("k_weight", k_weight, _BF16, (d,), dev), eps, q_out.data_ptr(), qos, k_out_ptr, kos, _handle(stream, dev))
    return q_out, k_out


def polyspec_prompt_attention(q, k, v, rows_at, scale=None, out=None, lse=None, device_status=None, stream=None):
    """Causal attention over packed prompts: prompt b is the rows rows_at[b] .. rows_at[b + 1] - 1 of q [rows, q_heads, d], k and v
    [rows, kv_heads, d] (bf16; rows may lie apart).  scale: d ** -0.5 where None.  out [rows, q_heads, d] bf16 and, where given, lse
    [rows, q_heads] fp32 are contiguous.  Returns (out, lse, status word)."""
    qs, dev = _head_rows("q", q, None, -1)
    shape = rows, heads, d = q.shape
    ks = _head_rows("k", k, None, dev)[0]
    k_shape = k.shape
    kv_heads = k_shape[1]
    if k_shape[0] != rows or k_shape[2] != d:
        raise ValueError("shapes do not fit: k must be [rows, kv_heads, head_dim]")
    vs = _head_rows("v", v, k_shape, dev)[0]
    if rows_at.dim() != 1 or rows_at.shape[0] < 2:
        raise ValueError("rows_at must be [n_seqs + 1]")
    if out is None:
        out = _empty(shape, _BF16, dev, stream)
    n_seqs = rows_at.shape[0] - 1
    device_status = _status_word(device_status, dev, stream)
    _call("polyspec_prompt_attention", load_library().polyspec_prompt_attention, dev, q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs,
          _flat("rows_at", rows_at, _I32T, (n_seqs + 1,), dev), n_seqs, rows, heads, kv_heads, d, d ** -0.5 if scale is None else scale,
          _flat("out", out, _BF16, shape, dev), _flat("lse", lse, _F32T, (rows, heads), dev), _flat("device_status", device_status, _I32T, (1,), dev),
          _handle(stream, dev))
    return out, lse, device_status


def cache_page_bytes(kv_heads: int, d: int, page_tokens: int) -> int:
    """Bytes of one page of one layer's keys (or values) in 4 bits."""
    return kv_heads * (page_tokens // 8) * (4 * d + 32)


def _block_rows(pages, rows, rows_at, base, extra, n_rows):
    n, dev = pages.n_seqs, pages.dev
    per_seq = (n,)
    return BlockRows(_flat("rows_at", rows_at, _I32T, (n + 1,), dev), _flat("n_rows", n_rows, _I32T, per_seq, dev), _flat("base", base, _I32T, per_seq, dev),
                     _flat("extra", extra, _I32T, per_seq, dev), rows)


def _layer_pool(pages, pool, kv_heads, d, layers=False):
    """pool: [planes, n_pages, ...] of any type; the planes of one layer (keys, values) or of all.  Returns its address."""
    size = pool.shape
    if len(size) < 3 or size[1] != pages.n_pages or (size[0] < 2 or size[0] % 2 if layers else size[0] != 2):
        raise ValueError("a pool must be [2 * layers, n_pages, ...]" if layers else "a layer's pool must be [2, n_pages, ...]: keys, values")
    if pool.numel() * pool.element_size() != size[0] * size[1] * cache_page_bytes(kv_heads, d, pages.page_tokens):
        raise ValueError("a page must have kv_heads * (page_tokens / 8) * (4 * head_dim + 32) bytes")
    if pool.get_device() != pages.dev or not pool.is_contiguous():
        raise ValueError("pool must be a contiguous tensor on the device of the pages")
    return pool.data_ptr()


def polyspec_cache_append(pages, k, v, pool, rows_at, base, extra=None, n_rows=None, k_held=None, v_held=None, weights=None, device_status=None, stream=None):
    """Keys and values of a block's rows, k and v [rows, kv_heads, d] bf16, into the 4-bit pages of one layer: pool [2, n_pages, ...].

    Sequence b has the rows rows_at[b] .. (rows_at[b+1] - rows_at[b] of them, or the first n_rows[b]); its row i goes to slot base[b] +
    extra[b] + i, which must have been reserved.  k_held, v_held [rows, kv_heads, d] bf16 take the values the pages now stand for; weights
    [n_seqs, max_pages * page_tokens] fp32 become 0 at the new slots.  Returns the status word."""
    dev = pages.dev
    ks = _head_rows("k", k, None, dev)[0]
    shape = rows, kv_heads, d = k.shape
    vs = _head_rows("v", v, shape, dev)[0]
    r = _block_rows(pages, rows, rows_at, base, extra, n_rows)
    device_status = _status_word(device_status, dev, stream)
    _call("polyspec_cache_append", load_library().polyspec_cache_append, dev, pages.c, r, k.data_ptr(), ks, v.data_ptr(), vs, kv_heads, d,
          _layer_pool(pages, pool, kv_heads, d), _flat("k_held", k_held, _BF16, shape, dev), _flat("v_held", v_held, _BF16, shape, dev),
          _flat("weights", weights, _F32T, (pages.n_seqs, pages.max_pages * pages.page_tokens), dev),
          _flat("device_status", device_status, _I32T, (1,), dev), _handle(stream, dev))
    return device_status


@functools.lru_cache(maxsize=256)       # (a function of the sizes alone)
def polyspec_cache_attention_workspace(q_heads: int, kv_heads: int, d: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().polyspec_cache_attention_workspace(q_heads, kv_heads, d, n), "polyspec_cache_attention_workspace")
    return n.value


def polyspec_cache_attention(pages, q, pool, kv_heads, rows_at, base, extra=None, n_rows=None, scale=None, out=None, lse=None, device_status=None,
                             workspace=None, stream=None):
    """Attention of a block's rows q [rows, q_heads, d] bf16 over one layer's 4-bit pages (pool [2, n_pages, ...]): row i of sequence b over the
    slots up to its own, base[b] + extra[b] + i.  Rows as in polyspec_cache_append; scale: d ** -0.5 where None.

    out [rows, q_heads, d] bf16; lse, where given, [rows, q_heads] fp32.  The workspace is the caller's or a fresh one of the call's stream.
    Returns (out, lse, status word)."""
    dev = pages.dev
    qs = _head_rows("q", q, None, dev)[0]
    shape = rows, heads, d = q.shape
    r = _block_rows(pages, rows, rows_at, base, extra, n_rows)
    pool_ptr = _layer_pool(pages, pool, kv_heads, d)
    if out is None:
        out = _empty(shape, _BF16, dev, stream)
    if workspace is None:
        workspace = _empty((polyspec_cache_attention_workspace(heads, kv_heads, d),), torch.uint8, dev, stream)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the device of the pages")
    device_status = _status_word(device_status, dev, stream)
    _call("polyspec_cache_attention", load_library().polyspec_cache_attention, dev, pages.c, r, q.data_ptr(), qs, heads, kv_heads, d,
          d ** -0.5 if scale is None else scale, pool_ptr, _flat("out", out, _BF16, shape, dev), _flat("lse", lse, _F32T, (rows, heads), dev),
          _flat("device_status", device_status, _I32T, (1,), dev), workspace.data_ptr(), workspace.nbytes, _handle(stream, dev))
    return out, lse, device_status


def polyspec_cache_weigh(pages, q, pool, kv_heads, rows_at, base, lse, weights, extra=None, n_rows=None, scale=None, keep=1.0, device_status=None, stream=None):
    """weights [n_seqs, max_pages * page_tokens] fp32 = keep * weights + the attention weight that the rows gave each cached token, over all heads;
    lse [rows, q_heads] of polyspec_cache_attention on the same rows, n_rows how many of a sequence's rows count.  Returns the status word."""
    dev = pages.dev
    qs = _head_rows("q", q, None, dev)[0]
    rows, heads, d = q.shape
    r = _block_rows(pages, rows, rows_at, base, extra, n_rows)
    device_status = _status_word(device_status, dev, stream)
    _call("polyspec_cache_weigh", load_library().polyspec_cache_weigh, dev, pages.c, r, q.data_ptr(), qs, heads, kv_heads, d,
          d ** -0.5 if scale is None else scale, _layer_pool(pages, pool, kv_heads, d), _flat("lse", lse, _F32T, (rows, heads), dev), keep,
          _flat("weights", weights, _F32T, (pages.n_seqs, pages.max_pages * pages.page_tokens), dev),
          _flat("device_status", device_status, _I32T, (1,), dev), _handle(stream, dev))
    return device_status


@functools.lru_cache(maxsize=256)
def polyspec_cache_evict_workspace(n_seqs: int, max_pages: int, page_tokens: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().polyspec_cache_evict_workspace(n_seqs, max_pages, page_tokens, n), "polyspec_cache_evict_workspace")
    return n.value


def polyspec_cache_evict(pages, budget, weights, pool, kv_heads, d, first=0, recent=0, kept_from=None, device_status=None, workspace=None, stream=None):
    """Cut sequences of more than budget[b] tokens (budget [n_seqs] int32; negative: left alone) to budget[b]: the first `first`, the last `recent` and the
    heaviest between stay and move together in every plane of pool [2 * layers, n_pages, ...] and in weights [n_seqs, max_pages * page_tokens].
    pages.len tells what is left, kept_from (int32, like weights) the slots the kept tokens had.  Returns the status word."""
    dev, shape = pages.dev, (pages.n_seqs, pages.max_pages * pages.page_tokens)
    pool_ptr = _layer_pool(pages, pool, kv_heads, d, layers=True)
    if workspace is None:
        workspace = _empty((polyspec_cache_evict_workspace(pages.n_seqs, pages.max_pages, pages.page_tokens),), torch.uint8, dev, stream)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the device of the pages")
    device_status = _status_word(device_status, dev, stream)
    _call("polyspec_cache_evict", load_library().polyspec_cache_evict, dev, pages.c, _flat("budget", budget, _I32T, (pages.n_seqs,), dev), first, recent,
          _flat("weights", weights, _F32T, shape, dev), pool_ptr, pool.shape[0], kv_heads, d, _flat("kept_from", kept_from, _I32T, shape, dev),
          _flat("device_status", device_status, _I32T, (1,), dev), workspace.data_ptr(), workspace.nbytes, _handle(stream, dev))
    return device_status
