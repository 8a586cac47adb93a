"""Python binding of libtwinkv (include/twinkv.h): argument marshalling only.

Each function has the name of the C entry point it calls.  Tensors are torch CUDA
tensors (torch supplies device memory and streams); every computation runs in the
library's CUDA kernels.  There is no CPU fallback: if the library is missing or the
device is not an sm_103 GPU, calls raise.

Paper: TwinKV (arXiv 2608.27128) Sec. 3.2 (Eq. 1, twin window, protected regions) and
Sec. 3.4 (Eq. 4, orphans, donors, the budget-exact swap).
"""
from __future__ import annotations

import ctypes
import functools
import math
import operator
import os
import threading

import torch

from . import build as _build

(OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_BUDGET, ERR_CUDA, ERR_TIMEOUT, ERR_WORKSPACE,
 ERR_TOO_LARGE) = range(8)
NOALLOC_MAX_POSITIONS = 262144
BF16, F32 = 0, 1
(OP_REDUNDANCY, OP_REPAIR, OP_REPAIR_SELECT, OP_POLICY, OP_REPAIR_SELECT_DEDUP,
 OP_REDUNDANCY_SYMMETRIC) = range(6)
KERNEL_PREP, KERNEL_AUDIT, KERNEL_REPAIR, KERNEL_REFINE = 0, 1, 2, 3
KERNEL_NAMES = ("prep", "audit", "repair", "refine")

EXPORTED = (
    "twinkv_abi_version", "twinkv_default_params", "twinkv_swaps_capacity",
    "twinkv_workspace_size", "twinkv_redundancy", "twinkv_repair", "twinkv_repair_select",
    "twinkv_status_string", "twinkv_get_last_error", "twinkv_set_wait_timeout_ns",
    "twinkv_wait_probe", "twinkv_profile_begin", "twinkv_profile_end",
    "twinkv_repair_select_noalloc", "twinkv_host_arena_size", "twinkv_host_default_chunk",
    "twinkv_repair_host",
    "twinkv_policy", "twinkv_repair_dedup", "twinkv_repair_select_dedup",
    "twinkv_redundancy_symmetric",
    "twinkv_cache_page_bytes", "twinkv_cache_move_workspace", "twinkv_cache_attend_workspace",
    "twinkv_qk_norm_rope", "twinkv_cache_pack", "twinkv_cache_append", "twinkv_cache_compact",
    "twinkv_cache_read", "twinkv_cache_attend",
)
PAGE_SLOTS = 64                                 # slots of a page (TWINKV_PAGE_SLOTS)
PAGE_BYTES = {64: 4864, 128: 9472}              # twinkv_cache_page_bytes by head dimension
_PAGE_DIM = {v: k for k, v in PAGE_BYTES.items()}


class Shape(ctypes.Structure):
    _fields_ = [("L", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32),
                ("d", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class Params(ctypes.Structure):
    _fields_ = [("threshold", ctypes.c_float), ("window", ctypes.c_int32),
                ("n_sink", ctypes.c_int32), ("n_recent", ctypes.c_int32)]


class Pool(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("n_pages", ctypes.c_int32), ("d", ctypes.c_int32)]


class Heads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("tokens", "heads_q", "heads_k", "d", "dtype",
                                              "rows")] + \
               [(n, ctypes.c_int64) for n in ("q_token", "q_head", "k_token", "k_head",
                                              "out_q_token", "out_q_head", "out_k_token",
                                              "out_k_head")]


class Rows(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "H", "n", "dtype")] + \
               [(n, ctypes.c_int64) for n in ("k_batch", "k_token", "k_head", "v_batch",
                                              "v_token", "v_head")]


class Queries(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "H", "Hq", "n")] + \
               [(n, ctypes.c_int64) for n in ("q_batch", "q_token", "q_head")]


class TwinKVError(RuntimeError):
    def __init__(self, status: int, what: str = ""):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})")


_P = ctypes.c_void_p
_lock = threading.Lock()
_lib = None


def library_path() -> str:
    return _build.LIB


def load(build_if_missing: bool = True):
    """Load libtwinkv.so (building it with nvcc first when it is missing or stale)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        path = _build.LIB
        if build_if_missing:
            path = _build.build()
        if not os.path.exists(path):
            raise RuntimeError(f"libtwinkv.so not found at {path}; run "
                               "`python -m paper_2608_27128_gb300.build`")
        lib = ctypes.CDLL(path)
        lib.twinkv_abi_version.restype = ctypes.c_int32
        lib.twinkv_default_params.restype = Params
        lib.twinkv_swaps_capacity.argtypes = [Shape]
        lib.twinkv_swaps_capacity.restype = ctypes.c_size_t
        lib.twinkv_workspace_size.argtypes = [Shape, ctypes.c_int32]
        lib.twinkv_workspace_size.restype = ctypes.c_size_t
        lib.twinkv_redundancy.argtypes = [_P, Shape, ctypes.c_int32, _P, _P, _P,
                                          ctypes.c_size_t, _P]
        lib.twinkv_redundancy_symmetric.argtypes = lib.twinkv_redundancy.argtypes
        lib.twinkv_repair.argtypes = [_P, Shape, _P, _P, ctypes.c_float,
                                      ctypes.POINTER(Params), _P, _P, _P, _P, _P, _P, _P, _P,
                                      _P, ctypes.c_size_t, _P]
        lib.twinkv_repair_select.argtypes = [_P, Shape, _P, _P, ctypes.c_float,
                                             ctypes.POINTER(Params), _P, _P, _P, _P, _P,
                                             ctypes.c_size_t, _P]
        lib.twinkv_repair_select_noalloc.argtypes = [_P, Shape, _P, _P, ctypes.c_float,
                                                     ctypes.POINTER(Params), _P, _P, _P, _P,
                                                     _P]
        lib.twinkv_host_arena_size.argtypes = [Shape, ctypes.c_int32]
        lib.twinkv_host_arena_size.restype = ctypes.c_size_t
        lib.twinkv_host_default_chunk.argtypes = [Shape]
        lib.twinkv_host_default_chunk.restype = ctypes.c_int32
        lib.twinkv_repair_host.argtypes = [_P, Shape, _P, _P, ctypes.c_float,
                                           ctypes.POINTER(Params), _P, _P, _P, _P, _P, _P, _P,
                                           _P, ctypes.c_int32, _P, ctypes.c_size_t, _P]
        lib.twinkv_repair_dedup.argtypes = lib.twinkv_repair.argtypes
        lib.twinkv_repair_select_dedup.argtypes = [_P, _P, Shape, _P, _P, ctypes.c_float,
                                                   ctypes.POINTER(Params), _P, _P, _P, _P, _P,
                                                   ctypes.c_size_t, _P]
        lib.twinkv_policy.argtypes = [_P, Shape, _P, ctypes.c_float, ctypes.POINTER(Params),
                                      _P, _P, _P, _P, ctypes.c_size_t, _P]
        i32 = ctypes.c_int32
        lib.twinkv_cache_page_bytes.argtypes = [i32]
        lib.twinkv_cache_page_bytes.restype = ctypes.c_size_t
        lib.twinkv_cache_move_workspace.argtypes = [i32, i32]
        lib.twinkv_cache_move_workspace.restype = ctypes.c_size_t
        lib.twinkv_cache_attend_workspace.argtypes = [Queries, i32]
        lib.twinkv_cache_attend_workspace.restype = ctypes.c_size_t
        lib.twinkv_qk_norm_rope.argtypes = [_P, _P, Heads, _P, _P, ctypes.c_float, _P, _P, _P,
                                            _P, _P, _P]
        lib.twinkv_cache_pack.argtypes = [_P, _P, Shape, _P, Pool, _P, i32, _P, _P, _P,
                                          ctypes.c_size_t, _P]
        lib.twinkv_cache_append.argtypes = [_P, _P, Rows, _P, Pool, _P, i32, _P, _P, _P, _P]
        lib.twinkv_cache_compact.argtypes = [Pool, _P, i32, _P, i32, _P, i32, _P, i32, _P, _P,
                                             _P, ctypes.c_size_t, _P]
        lib.twinkv_cache_read.argtypes = [Pool, _P, i32, _P, i32, i32, i32, _P, _P, _P, _P, _P]
        lib.twinkv_cache_attend.argtypes = [_P, Queries, ctypes.c_float, i32, i32, Pool, _P, i32,
                                            _P, _P, _P, _P, _P, ctypes.c_size_t, _P]
        for name in ("twinkv_qk_norm_rope", "twinkv_cache_pack", "twinkv_cache_append",
                     "twinkv_cache_compact", "twinkv_cache_read", "twinkv_cache_attend"):
            getattr(lib, name).restype = ctypes.c_int
        lib.twinkv_status_string.argtypes = [ctypes.c_int]
        lib.twinkv_status_string.restype = ctypes.c_char_p
        lib.twinkv_set_wait_timeout_ns.argtypes = [ctypes.c_uint64]
        lib.twinkv_wait_probe.argtypes = [ctypes.c_uint64, ctypes.POINTER(ctypes.c_int32), _P]
        lib.twinkv_profile_end.argtypes = [ctypes.POINTER(ctypes.c_int32),
                                           ctypes.POINTER(ctypes.c_double)]
        for name in ("twinkv_redundancy", "twinkv_redundancy_symmetric", "twinkv_repair",
                     "twinkv_repair_select",
                     "twinkv_repair_select_noalloc", "twinkv_repair_host", "twinkv_policy",
                     "twinkv_repair_dedup", "twinkv_repair_select_dedup",
                     "twinkv_get_last_error", "twinkv_set_wait_timeout_ns",
                     "twinkv_wait_probe", "twinkv_profile_begin", "twinkv_profile_end"):
            getattr(lib, name).restype = ctypes.c_int
        _lib = lib
        return lib


def status_string(status: int) -> str:
    try:
        return load().twinkv_status_string(int(status)).decode()
    except Exception:  # the library itself failed to load
        return f"status {status}"


def _check(status: int, what: str):
    if status != OK:
        raise TwinKVError(status, what)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _current_calls():
    """Functions for the current device's number and for the handle of a device's current stream."""
    # torch.cuda's own make objects on the way (1.5 us a call); what lies beneath them is not public,
    # so a torch that lacks it gets the public ones
    device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return device, raw or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


_current_device, _current_stream = _current_calls()


def _stream(stream):
    return _current_stream(_current_device()) if stream is None else stream.cuda_stream


def _need(t, name, dtype, shape, device):
    # what a call with valid tensors passes, before the checks that name what is wrong
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.shape == shape
            and t.device == device and t.is_contiguous()):
        return t
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.device != device or not t.is_cuda:
        raise ValueError(f"{name} must live on {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _out(t, name, dtype, shape, device):
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    return _need(t, name, dtype, shape, device)


def shape_of(keys) -> Shape:
    if keys.dim() != 4:
        raise ValueError("keys must be [L, H, N, d]")
    if keys.dtype == torch.bfloat16:
        dt = BF16
    elif keys.dtype == torch.float32:
        dt = F32
    else:
        raise ValueError("keys must be bfloat16 or float32")
    L, H, N, d = (int(x) for x in keys.shape)
    return Shape(L, H, N, d, dt)


def twinkv_default_params() -> Params:
    return load().twinkv_default_params()


def twinkv_swaps_capacity(shape: Shape) -> int:
    return int(load().twinkv_swaps_capacity(shape))


@functools.lru_cache(maxsize=1024)
def _workspace_size(L, H, N, d, dtype, op) -> int:
    return int(load().twinkv_workspace_size(Shape(L, H, N, d, dtype), op))


def twinkv_workspace_size(shape: Shape, op: int) -> int:
    return _workspace_size(shape.L, shape.H, shape.N, shape.d, shape.dtype, int(op))


def workspace(shape: Shape, op: int, device) -> torch.Tensor:
    """A device workspace of the size `op` needs (torch's allocator: 512-byte aligned)."""
    n = twinkv_workspace_size(shape, op)
    return torch.empty(max(n, 1), dtype=torch.uint8, device=device)


def _ws(ws, shape, op, device):
    need = twinkv_workspace_size(shape, op)
    if ws is None:
        ws = workspace(shape, op, device)
    if ws.numel() < need:
        raise ValueError(f"workspace needs {need} bytes, got {ws.numel()}")
    if ws.device != device or not ws.is_contiguous():
        raise ValueError(f"workspace must be contiguous and live on {device}")
    return ws


def twinkv_redundancy(keys, window: int = 32, out_score=None, out_twin=None, ws=None,
                      stream=None):
    """Best twin of every key over all other keys outside the +-window band.

    keys: [L,H,N,d] bf16/float32 CUDA tensor.  Returns (score float64 [L,H,N],
    twin int32 [L,H,N]); score = -1 and twin = -1 where no position lies beyond w.
    """
    s = shape_of(keys)
    dev = keys.device
    _need(keys, "keys", keys.dtype, keys.shape, dev)
    out_score = _out(out_score, "out_score", torch.float64, keys.shape[:3], dev)
    out_twin = _out(out_twin, "out_twin", torch.int32, keys.shape[:3], dev)
    ws = _ws(ws, s, OP_REDUNDANCY, dev)
    st = load().twinkv_redundancy(_ptr(keys), s, int(window), _ptr(out_score), _ptr(out_twin),
                                  _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "twinkv_redundancy")
    return out_score, out_twin


def twinkv_redundancy_symmetric(keys, window: int = 32, out_score=None, out_twin=None,
                                ws=None, stream=None):
    """twinkv_redundancy from the upper-triangle similarity tiles only (each tile serves
    its rows and its columns); same arguments and results."""
    s = shape_of(keys)
    dev = keys.device
    _need(keys, "keys", keys.dtype, keys.shape, dev)
    out_score = _out(out_score, "out_score", torch.float64, keys.shape[:3], dev)
    out_twin = _out(out_twin, "out_twin", torch.int32, keys.shape[:3], dev)
    ws = _ws(ws, s, OP_REDUNDANCY_SYMMETRIC, dev)
    st = load().twinkv_redundancy_symmetric(_ptr(keys), s, int(window), _ptr(out_score),
                                            _ptr(out_twin), _ptr(ws), ws.numel(),
                                            _stream(stream))
    _check(st, "twinkv_redundancy_symmetric")
    return out_score, out_twin


@functools.lru_cache(maxsize=1)
def _defaults():
    p = twinkv_default_params()
    return p.threshold, p.window, p.n_sink, p.n_recent


def _params(params, threshold, window, n_sink, n_recent):
    p = Params(*(_defaults() if params is None else
                 (params.threshold, params.window, params.n_sink, params.n_recent)))
    if threshold is not None:
        p.threshold = float(threshold)
    if window is not None:
        p.window = int(window)
    if n_sink is not None:
        p.n_sink = int(n_sink)
    if n_recent is not None:
        p.n_recent = int(n_recent)
    return p


def twinkv_repair_dedup(keys, retained_mask, budget=None, threshold=None, params=None,
                        **kw) -> dict:
    """twinkv_repair, but a donor is never evicted together with its twin (see the C
    header); same arguments and outputs."""
    return twinkv_repair(keys, retained_mask, budget, threshold, params, _fn="twinkv_repair_dedup",
                         **kw)


def twinkv_repair(keys, retained_mask, budget=None, threshold=None, params=None, *,
                  window=None, n_sink=None, n_recent=None, want_ret=True, want_all=False,
                  out=None, ws=None, stream=None, _fn="twinkv_repair") -> dict:
    """Audit of the retained set S0 and the budget-exact orphan/donor swap.

    keys [L,H,N,d] bf16/float32; retained_mask [L,H,N] uint8; budget [L*H] int32 or None.
    Returns a dict of CUDA tensors: mask (S1), swaps [L*H, N//2, 2], nswaps, status,
    and score_ret/twin_ret (b_i(S0)) if want_ret, score_all/twin_all if want_all.
    ``out`` may hold preallocated tensors under the same keys.
    """
    s = shape_of(keys)
    dev = keys.device
    _need(keys, "keys", keys.dtype, keys.shape, dev)
    L, H, N = s.L, s.H, s.N
    _need(retained_mask, "retained_mask", torch.uint8, (L, H, N), dev)
    if budget is not None:
        _need(budget, "budget", torch.int32, (L * H,), dev)
    p = _params(params, threshold, window, n_sink, n_recent)
    out = dict(out or {})
    o = {
        "mask": _out(out.get("mask"), "mask", torch.uint8, (L, H, N), dev),
        "swaps": _out(out.get("swaps"), "swaps", torch.int32, (L * H, N // 2, 2), dev),
        "nswaps": _out(out.get("nswaps"), "nswaps", torch.int32, (L * H,), dev),
        "status": _out(out.get("status"), "status", torch.int32, (L * H,), dev),
    }
    if want_ret:
        o["score_ret"] = _out(out.get("score_ret"), "score_ret", torch.float64, (L, H, N), dev)
        o["twin_ret"] = _out(out.get("twin_ret"), "twin_ret", torch.int32, (L, H, N), dev)
    if want_all:
        o["score_all"] = _out(out.get("score_all"), "score_all", torch.float64, (L, H, N), dev)
        o["twin_all"] = _out(out.get("twin_all"), "twin_all", torch.int32, (L, H, N), dev)
    ws = _ws(ws, s, OP_REPAIR, dev)
    st = getattr(load(), _fn)(
        _ptr(keys), s, _ptr(retained_mask), _ptr(budget), p.threshold,
        ctypes.byref(p), _ptr(o["mask"]), _ptr(o["swaps"]), _ptr(o["nswaps"]),
        _ptr(o.get("score_ret")), _ptr(o.get("twin_ret")), _ptr(o.get("score_all")),
        _ptr(o.get("twin_all")), _ptr(o["status"]), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, _fn)
    return o


def twinkv_repair_select_dedup(score_ret, twin_ret, retained_mask, budget=None, threshold=None,
                               params=None, *, n_sink=None, n_recent=None, out=None, ws=None,
                               stream=None) -> dict:
    """The dedup selection alone, on given float64 b_i(S0) and int32 twins [L,H,N]."""
    if score_ret.dim() != 3:
        raise ValueError("score_ret must be [L, H, N]")
    L, H, N = (int(x) for x in score_ret.shape)
    dev = score_ret.device
    _need(score_ret, "score_ret", torch.float64, (L, H, N), dev)
    _need(twin_ret, "twin_ret", torch.int32, (L, H, N), dev)
    _need(retained_mask, "retained_mask", torch.uint8, (L, H, N), dev)
    if budget is not None:
        _need(budget, "budget", torch.int32, (L * H,), dev)
    s = Shape(L, H, N, 64, BF16)
    p = _params(params, threshold, None, n_sink, n_recent)
    out = dict(out or {})
    o = {
        "mask": _out(out.get("mask"), "mask", torch.uint8, (L, H, N), dev),
        "swaps": _out(out.get("swaps"), "swaps", torch.int32, (L * H, N // 2, 2), dev),
        "nswaps": _out(out.get("nswaps"), "nswaps", torch.int32, (L * H,), dev),
        "status": _out(out.get("status"), "status", torch.int32, (L * H,), dev),
    }
    ws = _ws(ws, s, OP_REPAIR_SELECT_DEDUP, dev)
    st = load().twinkv_repair_select_dedup(
        _ptr(score_ret), _ptr(twin_ret), s, _ptr(retained_mask), _ptr(budget),
        p.threshold, ctypes.byref(p), _ptr(o["mask"]), _ptr(o["swaps"]),
        _ptr(o["nswaps"]), _ptr(o["status"]), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "twinkv_repair_select_dedup")
    return o


def twinkv_repair_select(score_ret, retained_mask, budget=None, threshold=None, params=None,
                         *, n_sink=None, n_recent=None, out=None, ws=None,
                         stream=None) -> dict:
    """The classification, ranking and swap alone, on given float64 b_i(S0) [L,H,N]."""
    if score_ret.dim() != 3:
        raise ValueError("score_ret must be [L, H, N]")
    L, H, N = (int(x) for x in score_ret.shape)
    dev = score_ret.device
    _need(score_ret, "score_ret", torch.float64, (L, H, N), dev)
    _need(retained_mask, "retained_mask", torch.uint8, (L, H, N), dev)
    if budget is not None:
        _need(budget, "budget", torch.int32, (L * H,), dev)
    s = Shape(L, H, N, 64, BF16)
    p = _params(params, threshold, None, n_sink, n_recent)
    out = dict(out or {})
    o = {
        "mask": _out(out.get("mask"), "mask", torch.uint8, (L, H, N), dev),
        "swaps": _out(out.get("swaps"), "swaps", torch.int32, (L * H, N // 2, 2), dev),
        "nswaps": _out(out.get("nswaps"), "nswaps", torch.int32, (L * H,), dev),
        "status": _out(out.get("status"), "status", torch.int32, (L * H,), dev),
    }
    ws = _ws(ws, s, OP_REPAIR_SELECT, dev)
    st = load().twinkv_repair_select(
        _ptr(score_ret), s, _ptr(retained_mask), _ptr(budget), p.threshold,
        ctypes.byref(p), _ptr(o["mask"]), _ptr(o["swaps"]), _ptr(o["nswaps"]),
        _ptr(o["status"]), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "twinkv_repair_select")
    return o


def twinkv_repair_select_noalloc(score_ret, retained_mask, budget=None, threshold=None,
                                 params=None, *, n_sink=None, n_recent=None, out=None,
                                 stream=None) -> dict:
    """twinkv_repair_select without a workspace, for callers that may not allocate
    device memory: the library's own fixed scratch array holds the sort buffers, so at
    most NOALLOC_MAX_POSITIONS positions (L*H*N) per call, and calls that may run
    concurrently on the GPU must be ordered on one stream.  Output tensors are created
    here when ``out`` does not supply them; pass them in ``out`` to allocate nothing."""
    if score_ret.dim() != 3:
        raise ValueError("score_ret must be [L, H, N]")
    L, H, N = (int(x) for x in score_ret.shape)
    dev = score_ret.device
    _need(score_ret, "score_ret", torch.float64, (L, H, N), dev)
    _need(retained_mask, "retained_mask", torch.uint8, (L, H, N), dev)
    if budget is not None:
        _need(budget, "budget", torch.int32, (L * H,), dev)
    s = Shape(L, H, N, 64, BF16)
    p = _params(params, threshold, None, n_sink, n_recent)
    out = dict(out or {})
    o = {
        "mask": _out(out.get("mask"), "mask", torch.uint8, (L, H, N), dev),
        "swaps": _out(out.get("swaps"), "swaps", torch.int32, (L * H, N // 2, 2), dev),
        "nswaps": _out(out.get("nswaps"), "nswaps", torch.int32, (L * H,), dev),
        "status": _out(out.get("status"), "status", torch.int32, (L * H,), dev),
    }
    st = load().twinkv_repair_select_noalloc(
        _ptr(score_ret), s, _ptr(retained_mask), _ptr(budget), p.threshold,
        ctypes.byref(p), _ptr(o["mask"]), _ptr(o["swaps"]), _ptr(o["nswaps"]),
        _ptr(o["status"]), _stream(stream))
    _check(st, "twinkv_repair_select_noalloc")
    return o


def budget_for_ratio(N: int, ratio: float) -> int:
    """Retained count of Sec. 3.1: |S| = ceil((1 - rho) n)."""
    return int(math.ceil((1.0 - float(ratio)) * N - 1e-9))


def twinkv_policy(keys, budget, threshold=None, params=None, *, window=None, n_sink=None,
                  n_recent=None, want_count=True, out=None, ws=None, stream=None) -> dict:
    """The standalone TwinKV policy (Sec. 3.2, Eq. 2-3) on keys [L,H,N,d].

    budget: int32 CUDA tensor [L*H], or an int used for every unit.  Returns a dict of
    CUDA tensors: mask [L,H,N] uint8 (kept positions), status [L*H] int32 and, with
    want_count, count [L,H,N] int32 (r_i of Eq. 2).
    """
    s = shape_of(keys)
    dev = keys.device
    _need(keys, "keys", keys.dtype, keys.shape, dev)
    L, H, N = s.L, s.H, s.N
    if not isinstance(budget, torch.Tensor):
        budget = torch.full((L * H,), int(budget), dtype=torch.int32, device=dev)
    _need(budget, "budget", torch.int32, (L * H,), dev)
    p = _params(params, threshold, window, n_sink, n_recent)
    out = dict(out or {})
    o = {
        "mask": _out(out.get("mask"), "mask", torch.uint8, (L, H, N), dev),
        "status": _out(out.get("status"), "status", torch.int32, (L * H,), dev),
    }
    if want_count:
        o["count"] = _out(out.get("count"), "count", torch.int32, (L, H, N), dev)
    ws = _ws(ws, s, OP_POLICY, dev)
    st = load().twinkv_policy(
        _ptr(keys), s, _ptr(budget), p.threshold, ctypes.byref(p),
        _ptr(o["mask"]), _ptr(o.get("count")), _ptr(o["status"]), _ptr(ws), ws.numel(),
        _stream(stream))
    _check(st, "twinkv_policy")
    return o


def _need_host(t, name, dtype, shape):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.device.type != "cpu":
        raise ValueError(f"{name} must be a host tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _out_host(t, name, dtype, shape, pin):
    if t is None:
        return torch.empty(shape, dtype=dtype, pin_memory=pin)
    return _need_host(t, name, dtype, shape)


def twinkv_host_default_chunk(shape: Shape) -> int:
    """Units per chunk twinkv_repair_host uses when chunk_units is 0."""
    return int(load().twinkv_host_default_chunk(shape))


def twinkv_host_arena_size(shape: Shape, chunk_units: int = 0) -> int:
    return int(load().twinkv_host_arena_size(shape, int(chunk_units)))


def host_arena(shape: Shape, chunk_units: int = 0, device=None) -> torch.Tensor:
    """A device arena for twinkv_repair_host (torch's allocator: 512-byte aligned)."""
    n = twinkv_host_arena_size(shape, chunk_units)
    if n == 0:
        raise ValueError("invalid shape or chunk size")
    return torch.empty(n, dtype=torch.uint8, device=device or torch.cuda.current_device())


_arenas = {}


def _cached_arena(shape: Shape, chunk_units: int) -> torch.Tensor:
    """The binding's own arena for the current device, grown on demand.  It stays alive
    between calls because the library's copy streams may still be using it when a call
    returns; the library orders successive calls' use of it."""
    dev = torch.cuda.current_device()
    n = twinkv_host_arena_size(shape, chunk_units)
    if n == 0:
        raise ValueError("invalid shape or chunk size")
    a = _arenas.get(dev)
    if a is None or a.numel() < n:
        if a is not None:
            torch.cuda.synchronize(dev)   # the old arena may still be in use
        a = _arenas[dev] = torch.empty(n, dtype=torch.uint8, device=dev)
    return a


def twinkv_repair_host(keys, retained_mask, budget=None, threshold=None, params=None, *,
                       window=None, n_sink=None, n_recent=None, want_ret=True, want_all=False,
                       chunk_units=0, out=None, arena=None, stream=None) -> dict:
    """twinkv_repair on HOST tensors (a cache held in host memory): the units go to the
    device in chunks whose copies overlap the computation of other chunks.  Inputs and
    the returned outputs are CPU tensors (pinned ones copy asynchronously); the outputs
    are valid once ``stream`` (default: the current stream) has completed.  ``arena`` is
    a device uint8 tensor of twinkv_host_arena_size bytes that the caller keeps alive
    until the stream has completed (a cached one of the binding's when not given)."""
    s = shape_of(keys)
    _need_host(keys, "keys", keys.dtype, keys.shape)
    L, H, N = s.L, s.H, s.N
    _need_host(retained_mask, "retained_mask", torch.uint8, (L, H, N))
    if budget is not None:
        _need_host(budget, "budget", torch.int32, (L * H,))
    p = _params(params, threshold, window, n_sink, n_recent)
    pin = keys.is_pinned()
    out = dict(out or {})
    o = {
        "mask": _out_host(out.get("mask"), "mask", torch.uint8, (L, H, N), pin),
        "swaps": _out_host(out.get("swaps"), "swaps", torch.int32, (L * H, N // 2, 2), pin),
        "nswaps": _out_host(out.get("nswaps"), "nswaps", torch.int32, (L * H,), pin),
        "status": _out_host(out.get("status"), "status", torch.int32, (L * H,), pin),
    }
    if want_ret:
        o["score_ret"] = _out_host(out.get("score_ret"), "score_ret", torch.float64,
                                   (L, H, N), pin)
        o["twin_ret"] = _out_host(out.get("twin_ret"), "twin_ret", torch.int32, (L, H, N), pin)
    if want_all:
        o["score_all"] = _out_host(out.get("score_all"), "score_all", torch.float64,
                                   (L, H, N), pin)
        o["twin_all"] = _out_host(out.get("twin_all"), "twin_all", torch.int32, (L, H, N), pin)
    if arena is None:
        arena = _cached_arena(s, chunk_units)
    if not arena.is_cuda or arena.dtype != torch.uint8:
        raise ValueError("arena must be a CUDA uint8 tensor")
    st = load().twinkv_repair_host(
        _ptr(keys), s, _ptr(retained_mask), _ptr(budget), p.threshold,
        ctypes.byref(p), _ptr(o["mask"]), _ptr(o["swaps"]), _ptr(o["nswaps"]),
        _ptr(o.get("score_ret")), _ptr(o.get("twin_ret")), _ptr(o.get("score_all")),
        _ptr(o.get("twin_all")), _ptr(o["status"]), int(chunk_units), _ptr(arena),
        arena.numel(), _stream(stream))
    _check(st, "twinkv_repair_host")
    return o


# ---- the cache in pages of 4-bit codes --------------------------------------------------
#
# What the calls make themselves (outputs that ``out`` does not hold, workspaces) is allocated on
# the stream they run on.  Tensors that the caller passes must stay alive until that stream is done.

def cache_pool(n_pages: int, d: int, device="cuda") -> torch.Tensor:
    """A pool of pages for head dimension d: uint8 [n_pages, PAGE_BYTES[d]]."""
    if d not in PAGE_BYTES:
        raise ValueError("d must be 64 or 128")
    return torch.zeros((int(n_pages), PAGE_BYTES[d]), dtype=torch.uint8, device=device)


def cache_move_workspace(units: int, N: int, device) -> torch.Tensor:
    """A workspace for twinkv_cache_pack and twinkv_cache_compact with a mask [units, N]."""
    n = int(load().twinkv_cache_move_workspace(int(units), int(N)))
    if n == 0:
        raise ValueError("invalid number of units or positions")
    return torch.empty(n, dtype=torch.uint8, device=device)


@functools.lru_cache(maxsize=1024)
def _attend_workspace_size(B, n, Hq, H, d) -> int:
    return int(load().twinkv_cache_attend_workspace(Queries(B, H, Hq, n, 0, 0, 0), d))


def cache_attend_workspace(q_shape, H: int, device) -> torch.Tensor:
    """A workspace for twinkv_cache_attend with queries of q_shape [B, n, Hq, d], H KV heads."""
    B, n, Hq, d = (int(x) for x in q_shape)
    size = _attend_workspace_size(B, n, Hq, int(H), d)
    if size == 0:
        raise ValueError("unsupported queries")
    return torch.empty(size, dtype=torch.uint8, device=device)


# The checks of a call with small tensors cost as much as its kernels, so what depends on types,
# shapes and strides alone is checked once per combination (the cached functions below), and the
# rest in as few steps as it takes.

def _same(t, name, dtype, shape, dev: int):
    """A contiguous tensor of the given type and shape on CUDA device number `dev`."""
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape
            and t.get_device() == dev and t.is_contiguous()):
        return t
    return _need(t, name, dtype, shape, torch.device("cuda", dev))


def _made(t, name, dtype, shape, dev: int, stream):
    """An output: the caller's, or a new one, allocated on the stream the call runs on."""
    if t is not None:
        return _same(t, name, dtype, shape, dev)
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=dev)


def _bytes(ws, need, dev: int, stream):
    """A workspace: the caller's, or a new one, allocated on the stream the call runs on."""
    if ws is None:
        return _made(None, "workspace", torch.uint8, (max(need, 1),), dev, stream)
    if (ws.get_device() != dev or ws.dtype is not torch.uint8 or ws.numel() < need
            or not ws.is_contiguous()):
        raise ValueError(f"workspace must be a contiguous uint8 tensor of {need} bytes on CUDA "
                         f"device {dev}")
    return ws


def _pool(pool):
    """(Pool, head dimension, CUDA device number) of a pool on the current device."""
    if not isinstance(pool, torch.Tensor):
        raise TypeError("pool must be a torch tensor")
    shape, dev = pool.shape, pool.get_device()
    d = _PAGE_DIM.get(shape[-1]) if len(shape) == 2 else None
    if d is None:
        raise ValueError("pool must be [n_pages, PAGE_BYTES[d]]")
    if dev < 0 or dev != _current_device():
        raise ValueError(f"pool must live on the current CUDA device, not on {pool.device}")
    if pool.dtype is not torch.uint8 or not pool.is_contiguous():
        raise ValueError("pool must be contiguous uint8")
    return Pool(pool.data_ptr(), shape[0], d), d, dev


def _table(table, name, units, dev: int):
    """A page table [*units, max_pages]; its last size."""
    if not isinstance(table, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    shape = table.shape
    if (shape[:-1] != units or table.dtype is not torch.int32 or table.get_device() != dev
            or not table.is_contiguous()):
        raise ValueError(f"{name} must be contiguous int32 [{', '.join(map(str, units))}, "
                         f"max_pages] on CUDA device {dev}")
    return shape[-1]


def _kind(t, name):
    """Type, shape, strides of a tensor of rows."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    return t.dtype, t.shape, t.stride()


def _row_strides(kind, name, dtype, shape):
    """Strides of a tensor of rows: any but the last, each row on a 16-byte boundary."""
    if kind[0] is not dtype or tuple(kind[1]) != tuple(shape):
        raise ValueError(f"{name} must be {dtype} {tuple(shape)}, got {kind[0]} {tuple(kind[1])}")
    # a dimension of one has no stride
    strides = [x if n > 1 else 0 for x, n in zip(kind[2], shape)][:-1]
    step = 4 if dtype is torch.float32 else 8
    if kind[2][-1] != 1 or any(x % step for x in strides):
        raise ValueError(f"{name}'s rows must be contiguous and start on 16-byte boundaries")
    return strides


def _rows_dtype(dtype, name):
    if dtype is torch.bfloat16:
        return BF16
    if dtype is torch.float32:
        return F32
    raise ValueError(f"{name} must be bfloat16 or float32")


def _int32(x, name):
    """An int that int32 holds: ctypes takes others modulo 2^32 without a word."""
    i = operator.index(x)
    if not -0x80000000 <= i <= 0x7fffffff:
        raise ValueError(f"{name} must fit 32 bits, got {i}")
    return i


def _elsewhere(name, t, dev):
    return ValueError(f"{name} must live on CUDA device {dev}, not on {t.device}")


@functools.lru_cache(maxsize=1024)
def _rope_plan(q, k, out_q, out_k, cs):
    dtype, shape = (k if q is None else q)[:2]
    code = _rows_dtype(dtype, "q and k")
    if len(shape) != 3 or (k is not None and len(k[1]) != 3):
        raise ValueError("q and k must be [T, heads, d]")
    T, _, d = shape
    if cs[0] is not torch.float32 or len(cs[1]) != 2 or cs[1][1] != d or cs[2] != (d, 1):
        raise ValueError("cos_sin must be contiguous float32 [rows, d]")
    heads, strides = [0, 0], [0] * 8
    for i, (x, y, name) in enumerate(((q, out_q, "q"), (k, out_k, "k"))):
        if x is None:
            continue
        heads[i] = x[1][1]
        want = (T, heads[i], d)
        strides[2 * i:2 * i + 2] = _row_strides(x, name, dtype, want)
        strides[4 + 2 * i:6 + 2 * i] = _row_strides(y, f"out {name}", dtype, want)
    return Heads(T, heads[0], heads[1], d, code, cs[1][0], *strides), dtype, T, d


def twinkv_qk_norm_rope(q, k, wq, wk, cos_sin, positions, eps=1e-6, *, out=None,
                        stream=None) -> dict:
    """Norms of queries and keys per head and their rotation by position, in one pass.

    q [T,Hq,d] and k [T,H,d], bf16 or float32, any strides that keep rows on 16-byte boundaries
    (views into a fused projection); either may be None.  wq, wk [d] of the same dtype, or None
    (no norm).  cos_sin [rows,d] float32, cosines then sines; positions [T] int32.  Returns a
    dict: q, k (dense unless ``out`` holds tensors with other strides; ``out`` may hold q and k
    themselves) and status [T] int32 (1 where a position is outside the table; that token is 0).
    """
    x = k if q is None else q
    if not isinstance(x, torch.Tensor):
        raise TypeError("q and k must be torch tensors")
    dev = x.get_device()
    if dev < 0 or dev != _current_device():
        raise _elsewhere("q and k", x, "current")
    given = out or {}
    oq = ok = qk = kk = oqk = okk = None
    if q is not None:
        oq = given.get("q")
        if oq is None:
            oq = _made(None, "q", q.dtype, q.shape, dev, stream)
        qk, oqk = _kind(q, "q"), _kind(oq, "out q")
        if oq.get_device() != dev:
            raise _elsewhere("out q", oq, dev)
    if k is not None:
        ok = given.get("k")
        if ok is None:
            ok = _made(None, "k", k.dtype, k.shape, dev, stream)
        kk, okk = _kind(k, "k"), _kind(ok, "out k")
        if k.get_device() != dev or ok.get_device() != dev:
            raise _elsewhere("k and out k", k if k.get_device() != dev else ok, dev)
    s, dtype, T, d = _rope_plan(qk, kk, oqk, okk, _kind(cos_sin, "cos_sin"))
    if cos_sin.get_device() != dev:
        raise _elsewhere("cos_sin", cos_sin, dev)
    if wq is not None:
        _same(wq, "wq", dtype, (d,), dev)
    if wk is not None:
        _same(wk, "wk", dtype, (d,), dev)
    _same(positions, "positions", torch.int32, (T,), dev)
    status = _made(given.get("status"), "status", torch.int32, (T,), dev, stream)
    st = load().twinkv_qk_norm_rope(_ptr(q), _ptr(k), s, _ptr(wq), _ptr(wk), eps,
                                    cos_sin.data_ptr(), positions.data_ptr(), _ptr(oq), _ptr(ok),
                                    status.data_ptr(), _stream(stream))
    _check(st, "twinkv_qk_norm_rope")
    o = {"status": status}
    if q is not None:
        o["q"] = oq
    if k is not None:
        o["k"] = ok
    return o


def _lens_status(out, units, dev, stream):
    given = out or {}
    return (_made(given.get("lens"), "lens", torch.int32, units, dev, stream),
            _made(given.get("status"), "status", torch.int32, units, dev, stream))


@functools.lru_cache(maxsize=1024)
def _move_workspace_size(units, N) -> int:
    return int(load().twinkv_cache_move_workspace(units, N))


@functools.lru_cache(maxsize=1024)
def _pack_plan(dtype, shape):
    if len(shape) != 4:
        raise ValueError("keys must be [L, H, N, d]")
    return Shape(*shape, _rows_dtype(dtype, "keys"))


def twinkv_cache_pack(keys, values, retained_mask, pool, table, *, out=None, ws=None,
                      stream=None) -> dict:
    """The retained rows of a dense cache into pages, rounded to 4 bits.

    keys, values [L,H,N,d] bf16 or float32; retained_mask [L,H,N] uint8 or None (every row);
    pool as cache_pool makes it; table [L,H,max_pages] int32, the pages of each unit.  Returns a
    dict: lens [L,H] int32 and status [L,H] int32.
    """
    if not isinstance(keys, torch.Tensor):
        raise TypeError("keys must be a torch tensor")
    shape = keys.shape
    s = _pack_plan(keys.dtype, shape)
    p, d, dev = _pool(pool)
    _same(keys, "keys", keys.dtype, shape, dev)
    _same(values, "values", keys.dtype, shape, dev)
    if s.d != d:
        raise ValueError(f"the pool's pages hold rows of {d} values, the keys have {s.d}")
    units = shape[:2]
    pages = _table(table, "table", units, dev)
    wp, wn = None, 0
    if retained_mask is not None:
        _same(retained_mask, "retained_mask", torch.uint8, shape[:3], dev)
        ws = _bytes(ws, _move_workspace_size(s.L * s.H, s.N), dev, stream)
        wp, wn = ws.data_ptr(), ws.numel()
    lens, status = _lens_status(out, units, dev, stream)
    st = load().twinkv_cache_pack(
        keys.data_ptr(), values.data_ptr(), s, _ptr(retained_mask), p, table.data_ptr(), pages,
        lens.data_ptr(), status.data_ptr(), wp, wn, _stream(stream))
    _check(st, "twinkv_cache_pack")
    return {"lens": lens, "status": status}


@functools.lru_cache(maxsize=1024)
def _append_plan(k, v):
    code = _rows_dtype(k[0], "k")
    if len(k[1]) != 4:
        raise ValueError("k must be [B, n, H, d]")
    B, n, H, d = k[1]
    return Rows(B, H, n, code, *_row_strides(k, "k", k[0], k[1]),
                *_row_strides(v, "v", k[0], k[1])), B, n, H, d


def twinkv_cache_append(k, v, positions, pool, table, lens, *, out=None, stream=None) -> dict:
    """The rows of new tokens behind each unit's last slot.

    k, v [B,n,H,d] bf16 or float32, any strides that keep rows on 16-byte boundaries; positions
    [B,n] int32; table [B,H,max_pages]; lens [B,H] int32.  Returns a dict: lens [B,H], the new
    lengths (``out`` may hold ``lens`` itself), and status [B,H].
    """
    p, d, dev = _pool(pool)
    s, B, n, H, dk = _append_plan(_kind(k, "k"), _kind(v, "v"))
    if dk != d:
        raise ValueError(f"the pool's pages hold rows of {d} values, k has {dk}")
    if k.get_device() != dev or v.get_device() != dev:
        raise _elsewhere("k and v", k if k.get_device() != dev else v, dev)
    units = (B, H)
    _same(positions, "positions", torch.int32, (B, n), dev)
    pages = _table(table, "table", units, dev)
    _same(lens, "lens", torch.int32, units, dev)
    new, status = _lens_status(out, units, dev, stream)
    st = load().twinkv_cache_append(
        k.data_ptr(), v.data_ptr(), s, positions.data_ptr(), p, table.data_ptr(), pages,
        lens.data_ptr(), new.data_ptr(), status.data_ptr(), _stream(stream))
    _check(st, "twinkv_cache_append")
    return {"lens": new, "status": status}


def twinkv_cache_compact(pool, table, lens, keep, new_table, *, out=None, ws=None,
                         stream=None) -> dict:
    """The kept slots of each unit into other pages, in order.

    table [...,max_pages] and lens [...] of the units; keep [...,N] uint8 over their slots, N at
    least the longest, or None (a copy); new_table [...,new_max_pages], pages that no table uses.
    Returns a dict: lens and status, shaped as ``lens``.
    """
    p, _, dev = _pool(pool)
    if not isinstance(lens, torch.Tensor):
        raise TypeError("lens must be a torch tensor")
    units = lens.shape
    _same(lens, "lens", torch.int32, units, dev)
    pages, new_pages = (_table(table, "table", units, dev),
                        _table(new_table, "new_table", units, dev))
    U, N, wp, wn = lens.numel(), pages * PAGE_SLOTS, None, 0
    if keep is not None:
        if not isinstance(keep, torch.Tensor) or keep.dim() != len(units) + 1:
            raise ValueError("keep must be [units, N]")
        N = keep.shape[-1]
        _same(keep, "keep", torch.uint8, (*units, N), dev)
        ws = _bytes(ws, _move_workspace_size(U, N), dev, stream)
        wp, wn = ws.data_ptr(), ws.numel()
    new, status = _lens_status(out, units, dev, stream)
    st = load().twinkv_cache_compact(
        p, table.data_ptr(), pages, lens.data_ptr(), U, _ptr(keep), N, new_table.data_ptr(),
        new_pages, new.data_ptr(), status.data_ptr(), wp, wn, _stream(stream))
    _check(st, "twinkv_cache_compact")
    return {"lens": new, "status": status}


def twinkv_cache_read(pool, table, lens, rows: int, *, last=False, out=None,
                      stream=None) -> dict:
    """The first (or last) ``rows`` slots of each unit as bf16 rows.

    table [...,max_pages] and lens [...] of the units.  Returns a dict: keys and values
    [...,rows,d] bf16, positions [...,rows] int32 (-1, and rows of 0, where there is no slot) and
    status [...] int32.
    """
    p, d, dev = _pool(pool)
    if not isinstance(lens, torch.Tensor):
        raise TypeError("lens must be a torch tensor")
    units, rows, given = lens.shape, int(rows), out or {}
    _same(lens, "lens", torch.int32, units, dev)
    pages = _table(table, "table", units, dev)
    shape = (*units, rows, d)
    keys = _made(given.get("keys"), "keys", torch.bfloat16, shape, dev, stream)
    values = _made(given.get("values"), "values", torch.bfloat16, shape, dev, stream)
    positions = _made(given.get("positions"), "positions", torch.int32, (*units, rows), dev, stream)
    status = _made(given.get("status"), "status", torch.int32, units, dev, stream)
    st = load().twinkv_cache_read(
        p, table.data_ptr(), pages, lens.data_ptr(), lens.numel(), rows, 1 if last else 0,
        keys.data_ptr(), values.data_ptr(), positions.data_ptr(), status.data_ptr(),
        _stream(stream))
    _check(st, "twinkv_cache_read")
    return {"keys": keys, "values": values, "positions": positions, "status": status}


@functools.lru_cache(maxsize=1024)
def _attend_plan(q, H, d):
    if len(q[1]) != 4:
        raise ValueError("q must be [B, n, Hq, d]")
    B, n, Hq, _ = q[1]
    strides = _row_strides(q, "q", torch.bfloat16, (B, n, Hq, d))
    need = _attend_workspace_size(B, n, Hq, H, d) if H > 0 else 0
    return Queries(B, H, Hq, n, *strides), B, (B, n, Hq, d), need


def twinkv_cache_attend(q, pool, table, lens, *, scale=None, window=0, n_sink=0, want_lse=False,
                        out=None, ws=None, stream=None) -> dict:
    """Attention of each sequence's newest n tokens over its pages (append them first).

    q [B,n,Hq,d] bf16, any strides that keep rows on 16-byte boundaries; table [B,H,max_pages];
    lens [B,H] int32; scale: d ** -0.5 by default; window > 0: a token sees only the slots whose
    position is above its own minus ``window``, and those below ``n_sink``.  Returns a dict: out
    [B,n,Hq,d] bf16, status [B,H] int32 and, with want_lse, lse [B,n,Hq] float32.
    """
    p, d, dev = _pool(pool)
    if not isinstance(lens, torch.Tensor) or lens.dim() != 2:
        raise ValueError("lens must be [B, H]")
    units = lens.shape
    s, B, shape, need = _attend_plan(_kind(q, "q"), units[1], d)
    if q.get_device() != dev:
        raise _elsewhere("q", q, dev)
    if units[0] != B:
        raise ValueError(f"lens must be [{B}, H]")
    _same(lens, "lens", torch.int32, units, dev)
    pages = _table(table, "table", units, dev)
    given = out or {}
    o = {"out": _made(given.get("out"), "out", torch.bfloat16, shape, dev, stream),
         "status": _made(given.get("status"), "status", torch.int32, units, dev, stream)}
    lse = None
    if want_lse:
        o["lse"] = _made(given.get("lse"), "lse", torch.float32, shape[:3], dev, stream)
        lse = o["lse"].data_ptr()
    ws = _bytes(ws, need, dev, stream)
    st = load().twinkv_cache_attend(
        q.data_ptr(), s, d ** -0.5 if scale is None else scale, _int32(window, "window"),
        _int32(n_sink, "n_sink"), p,
        table.data_ptr(), pages, lens.data_ptr(), o["out"].data_ptr(), lse,
        o["status"].data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream))
    _check(st, "twinkv_cache_attend")
    return o


def twinkv_get_last_error() -> int:
    return int(load().twinkv_get_last_error())


def twinkv_set_wait_timeout_ns(ns: int):
    _check(load().twinkv_set_wait_timeout_ns(int(ns)), "twinkv_set_wait_timeout_ns")


def twinkv_wait_probe(timeout_ns: int, stream=None) -> int:
    out = ctypes.c_int32(-1)
    _check(load().twinkv_wait_probe(int(timeout_ns), ctypes.byref(out), _stream(stream)),
           "twinkv_wait_probe")
    return int(out.value)


def twinkv_profile_begin():
    _check(load().twinkv_profile_begin(), "twinkv_profile_begin")


def twinkv_profile_end() -> dict:
    k = len(KERNEL_NAMES)
    n = (ctypes.c_int32 * k)()
    ms = (ctypes.c_double * k)()
    _check(load().twinkv_profile_end(n, ms), "twinkv_profile_end")
    return {KERNEL_NAMES[i]: (int(n[i]), float(ms[i])) for i in range(k)}
