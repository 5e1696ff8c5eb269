"""Thin ctypes binding of libobcache.so (C ABI in include/obcache.h).

Argument marshalling only: tensors in, device pointers and sizes out.  Every step of
the path runs in the HIP kernels; torch supplies device memory and the current
stream.  There is no CPU fallback: a missing library is built once with hipcc, and a
failure to build or load it raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libobcache.so")

OBC_VALUE, OBC_KEY, OBC_JOINT, OBC_ALL, OBC_ATTN, OBC_VATP = 0, 1, 2, 3, 4, 5
OBC_F32, OBC_BF16, OBC_E4M3 = 0, 1, 2
OBC_OK, OBC_EINVAL, OBC_EUNSUPPORTED, OBC_EWORKSPACE, OBC_ELAUNCH = 0, -1, -2, -3, -4
VARIANT_CODES = {"value": OBC_VALUE, "key": OBC_KEY, "joint": OBC_JOINT, "all": OBC_ALL, "attn": OBC_ATTN,
                 "vatp": OBC_VATP}

_lib = None
_F32, _BF16, _I32 = torch.float32, torch.bfloat16, torch.int32
_E4M3, _U8 = torch.float8_e4m3fn, torch.uint8


class _CacheArg(ctypes.Structure):
    """obc_cache_t"""
    _fields_ = ([(x, ctypes.c_void_p) for x in ("k", "v", "k_scale", "v_scale", "page_table")]
                + [(x, ctypes.c_int32) for x in ("batch", "num_pages", "pages_per_seq", "page_size", "Hkv", "d", "dtype")])


class _RowsArg(ctypes.Structure):
    """obc_rows_t"""
    _fields_ = [("data", ctypes.c_void_p)] + [(x, ctypes.c_int64) for x in ("batch_stride", "token_stride", "head_stride")]


class ObcError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s" % (where, obc_status_string(status)))


def load_library():
    """Loads (building first if absent) the HIP library and declares the ABI signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from . import build as _build
        _build.build_library()
    lib = ctypes.CDLL(LIB_PATH)
    c_int, c_void_p, c_size_t = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    i32p = ctypes.POINTER(ctypes.c_int32)
    lib.obc_version.restype = c_int
    lib.obc_status_string.restype = ctypes.c_char_p
    lib.obc_status_string.argtypes = [c_int]
    lib.obc_score_workspace_bytes.restype = c_int
    lib.obc_score_workspace_bytes.argtypes = [c_int] * 8 + [ctypes.POINTER(c_size_t)]
    lib.obc_score.restype = c_int
    lib.obc_score.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, c_int, c_void_p,
                              c_int, c_int, i32p, c_void_p, c_size_t, c_void_p]
    lib.obc_score_accumulate.restype = c_int
    lib.obc_score_accumulate.argtypes = lib.obc_score.argtypes
    lib.obc_score_stages.restype = c_int
    lib.obc_score_stages.argtypes = lib.obc_score.argtypes + [c_int]
    lib.obc_select.restype = c_int
    lib.obc_select.argtypes = [c_void_p, c_int, c_void_p, c_int, c_int, c_int, i32p, c_void_p, c_size_t, c_void_p]
    lib.obc_select_workspace_bytes.restype = c_int
    lib.obc_select_workspace_bytes.argtypes = [c_int, c_int, c_int, ctypes.POINTER(c_size_t)]
    lib.obc_select_protected.restype = c_int
    lib.obc_select_protected.argtypes = [c_void_p, c_int, c_int, c_int, c_int, c_void_p, c_int, c_int, c_int, i32p,
                                         c_void_p, c_size_t, c_void_p]
    lib.obc_select_pooled.restype = c_int
    lib.obc_select_pooled.argtypes = [c_void_p, c_int, c_int, c_int, c_int, c_int, c_void_p, c_int, c_int, c_int, i32p,
                                      c_void_p, c_size_t, c_void_p]
    lib.obc_select_adaptive_workspace_bytes.restype = c_int
    lib.obc_select_adaptive_workspace_bytes.argtypes = [c_int, c_int, c_int, c_int, c_int, ctypes.POINTER(c_size_t)]
    lib.obc_select_adaptive.restype = c_int
    lib.obc_select_adaptive.argtypes = [c_void_p, c_int, c_int, c_void_p, c_void_p, c_int, c_int, c_int, c_int, i32p,
                                        c_void_p, c_size_t, c_void_p]
    lib.obc_compact.restype = c_int
    lib.obc_compact.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int,
                                c_int, c_void_p]
    lib.obc_compact_inplace.restype = c_int
    lib.obc_compact_inplace.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, c_int,
                                        c_void_p]
    lib.obc_compact_scores.restype = c_int
    lib.obc_compact_scores.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, c_void_p]
    lib.obc_probe_read_bandwidth.restype = c_int
    lib.obc_probe_read_bandwidth.argtypes = [c_void_p, c_size_t, c_void_p, c_void_p]
    lib.obc_init.restype = c_int
    lib.obc_score_static.restype = c_int
    lib.obc_score_static.argtypes = [c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int, c_int, c_void_p,
                                     c_int, c_int, i32p, c_int, c_void_p]
    lib.obc_decode_step_workspace_bytes.restype = c_int
    lib.obc_decode_step_workspace_bytes.argtypes = [c_int] * 7 + [ctypes.POINTER(c_size_t)]
    lib.obc_decode_step.restype = c_int
    lib.obc_decode_step.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_int, c_int,
                                    c_int, c_int, i32p, c_int, c_int, c_void_p, c_size_t, c_void_p]
    lib.obc_set_score_path.restype = c_int
    lib.obc_set_score_path.argtypes = [c_int]
    lib.obc_set_score_tuning.restype = c_int
    lib.obc_set_score_tuning.argtypes = [c_int, c_int]
    lib.obc_set_sweep2_form.restype = c_int
    lib.obc_set_sweep2_form.argtypes = [c_int]
    cache_p, rows_p, c_float = ctypes.POINTER(_CacheArg), ctypes.POINTER(_RowsArg), ctypes.c_float
    lib.obc_cache_append.restype = c_int
    lib.obc_cache_append.argtypes = [rows_p, rows_p, rows_p, cache_p, c_void_p, c_void_p, c_int, c_void_p, c_int, c_void_p, c_void_p,
                                     c_int, c_float, c_int, c_void_p, c_void_p, c_float, c_int, c_int, c_int, c_int, c_void_p]
    lib.obc_attend_workspace_bytes.restype = c_int
    lib.obc_attend_workspace_bytes.argtypes = [c_int, c_int, c_int, cache_p, c_int, ctypes.POINTER(c_size_t)]
    lib.obc_attend.restype = c_int
    lib.obc_attend.argtypes = [c_void_p, cache_p, c_void_p, c_void_p, c_int, c_void_p, c_int, c_int, c_int, c_int, c_int, c_float,
                               c_void_p, c_size_t, c_void_p]
    lib.obc_cache_read.restype = c_int
    lib.obc_cache_read.argtypes = [cache_p, c_void_p, c_void_p, c_void_p, c_int, c_int, c_int, c_void_p]
    _lib = lib
    return lib


def obc_version() -> int:
    return int(load_library().obc_version())


def obc_status_string(status: int) -> str:
    return load_library().obc_status_string(int(status)).decode()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return OBC_F32
    if t.dtype == torch.bfloat16:
        return OBC_BF16
    raise TypeError("q, k, v must be float32 or bfloat16, got %s" % t.dtype)


def _variant_code(variant) -> int:
    return VARIANT_CODES[variant] if isinstance(variant, str) else int(variant)


def _lens_arg(seq_lens: Optional[Sequence[int]], B: int):
    if seq_lens is None:
        return None
    if len(seq_lens) != B:
        raise ValueError("seq_lens needs one entry per sequence")
    return (ctypes.c_int32 * B)(*[int(x) for x in seq_lens])


# The current stream's handle without the Stream object torch.cuda.current_stream builds (2 us, as much as a launch).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(t: torch.Tensor) -> int:
    if _raw_stream is not None:
        return _raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream


def _require_cuda(*tensors):
    for t in tensors:
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("tensors must be contiguous and on the GPU")


def obc_score_workspace_bytes(B, N, W, Hq, Hkv, d, dtype, variant) -> int:
    out = ctypes.c_size_t(0)
    rc = load_library().obc_score_workspace_bytes(B, N, W, Hq, Hkv, d, dtype, variant, ctypes.byref(out))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_score_workspace_bytes")
    return int(out.value)


OBC_STAGE_SWEEP1, OBC_STAGE_COMBINE, OBC_STAGE_SWEEP2, OBC_STAGE_ALL = 1, 2, 4, 7
PATH_CODES = {"auto": 0, "plain": 1, "mfma": 2, "decode": 3}


def obc_set_score_path(path="auto") -> None:
    """Test hook: pins the scoring kernels process-wide ("auto" | "plain" | "mfma" | "decode")."""
    rc = load_library().obc_set_score_path(PATH_CODES[path] if isinstance(path, str) else int(path))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_set_score_path")


def obc_set_sweep2_form(form: int = 0) -> None:
    """Test hook: 0 = second sweep chosen by shape, 1 = 32 rows per wave, 2 = 64 rows per wave where the variant has a
    cross term; 1 and 2 also where the few-row kernel would run."""
    rc = load_library().obc_set_sweep2_form(int(form))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_set_sweep2_form")


def obc_set_score_tuning(splits: int = 0, range_len: int = 0) -> None:
    """Tuning hook: sweep-1 split count and sweep-2 token range of the matrix-core path (0 = automatic)."""
    rc = load_library().obc_set_score_tuning(int(splits), int(range_len))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_set_score_tuning")


def obc_score(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, variant="joint", seq_lens=None,
              scores: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
              stage_mask: Optional[int] = None, accumulate: bool = False) -> torch.Tensor:
    """q [B,Hq,W,d], k,v [B,Hkv,N,d] -> scores [B,Hkv,N] fp32 ([3,B,Hkv,N] for variant "all").

    stage_mask (measurement hook) routes the call through obc_score_stages; accumulate=True through
    obc_score_accumulate (adds to the `scores` passed in, which is then required)."""
    _require_cuda(q, k, v)
    B, Hq, W, d = q.shape
    Bk, Hkv, N, dk = k.shape
    if (Bk, dk) != (B, d) or v.shape != k.shape or k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q, k, v shapes or dtypes disagree")
    var = VARIANT_CODES[variant] if isinstance(variant, str) else int(variant)
    dt = _dtype_code(q)
    if workspace is None:
        workspace = torch.empty(obc_score_workspace_bytes(B, N, W, Hq, Hkv, d, dt, var), dtype=torch.uint8,
                                device=q.device)
    shape = (3, B, Hkv, N) if var == OBC_ALL else (B, Hkv, N)
    if scores is None:
        if accumulate:
            raise ValueError("accumulate=True needs the running scores tensor")
        scores = torch.empty(shape, dtype=torch.float32, device=q.device)
    elif tuple(scores.shape) != shape or scores.dtype != torch.float32 or not scores.is_contiguous():
        raise ValueError("scores must be a contiguous float32 tensor of shape %s" % (shape,))
    _require_cuda(scores, workspace)
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), N, W, Hq, Hkv, d, var, scores.data_ptr(), B, dt,
            _lens_arg(seq_lens, B), workspace.data_ptr(), workspace.numel(), _stream_ptr(q))
    if accumulate:
        if stage_mask is not None:
            raise ValueError("stage_mask and accumulate exclude each other")
        rc = load_library().obc_score_accumulate(*args)
    elif stage_mask is None:
        rc = load_library().obc_score(*args)
    else:
        rc = load_library().obc_score_stages(*args, int(stage_mask))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_score")
    return scores


OBC_STATIC_SCRATCH_BYTES = 48 << 20


def obc_init() -> None:
    rc = load_library().obc_init()
    if rc != OBC_OK:
        raise ObcError(rc, "obc_init")


def obc_score_static(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, variant, scores: torch.Tensor, seq_lens=None,
                     accumulate: bool = False) -> torch.Tensor:
    """obc_score / obc_score_accumulate on the library's static scratch: the caller passes inputs and the output
    tensor, and nothing is allocated (not by torch either)."""
    if not (q.is_cuda and k.is_cuda and v.is_cuda and scores.is_cuda and q.is_contiguous() and k.is_contiguous()
            and v.is_contiguous() and scores.is_contiguous()):
        raise ValueError("tensors must be contiguous and on the GPU")
    B, Hq, W, d = q.shape
    Bk, Hkv, N, dk = kv_shape = k.shape
    if Bk != B or dk != d or v.shape != kv_shape or k.dtype is not q.dtype or v.dtype is not q.dtype:
        raise ValueError("q, k, v shapes or dtypes disagree")
    var = VARIANT_CODES[variant] if isinstance(variant, str) else int(variant)
    shape = (3, B, Hkv, N) if var == OBC_ALL else (B, Hkv, N)
    if tuple(scores.shape) != shape or scores.dtype != torch.float32:
        raise ValueError("scores must be a contiguous float32 tensor of shape %s" % (shape,))
    rc = load_library().obc_score_static(q.data_ptr(), k.data_ptr(), v.data_ptr(), N, W, Hq, Hkv, d, var,
                                         scores.data_ptr(), B, _dtype_code(q), None if seq_lens is None else _lens_arg(seq_lens, B),
                                         1 if accumulate else 0, _stream_ptr(q))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_score_static")
    return scores


def obc_select_workspace_bytes(B: int, Hkv: int, N: int) -> int:
    out = ctypes.c_size_t(0)
    rc = load_library().obc_select_workspace_bytes(B, Hkv, N, ctypes.byref(out))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_select_workspace_bytes")
    return int(out.value)


def _select_ws(scores: torch.Tensor, workspace):
    """(pointer, bytes, tensor) of the optional selection scratch; allocates it when the shape profits and none was
    given.  The caller keeps the tensor alive until its C call has enqueued the kernels: torch's allocator hands a
    freed block to the next allocation on the same stream, which is only safe after the launches that use it.
    workspace=False asks for the one-block-per-head path."""
    if workspace is False:
        return None, 0, None
    B, Hkv, N = scores.shape
    if workspace is None:
        need = obc_select_workspace_bytes(B, Hkv, N)
        if need == 0:
            return None, 0, None
        workspace = torch.empty(need, dtype=torch.uint8, device=scores.device)
    _require_cuda(workspace)
    return workspace.data_ptr(), workspace.numel(), workspace


def obc_select(scores: torch.Tensor, budget: int, seq_lens=None,
               keep_idx: Optional[torch.Tensor] = None, workspace=None) -> torch.Tensor:
    """scores [B,Hkv,N] fp32 -> keep_idx [B,Hkv,budget] int32 ascending."""
    _require_cuda(scores)
    if scores.dtype != torch.float32 or scores.dim() != 3:
        raise ValueError("scores must be [B,Hkv,N] float32")
    B, Hkv, N = scores.shape
    if keep_idx is None:
        keep_idx = torch.empty((B, Hkv, max(int(budget), 0)), dtype=torch.int32, device=scores.device)
    elif keep_idx.dtype != torch.int32 or tuple(keep_idx.shape) != (B, Hkv, int(budget)) or not keep_idx.is_contiguous():
        raise ValueError("keep_idx must be a contiguous [B,Hkv,%d] int32 tensor" % int(budget))
    ws_ptr, ws_bytes, ws_hold = _select_ws(scores, workspace)
    rc = load_library().obc_select(scores.data_ptr(), int(budget), keep_idx.data_ptr(), B, Hkv, N,
                                   _lens_arg(seq_lens, B), ws_ptr, ws_bytes, _stream_ptr(scores))
    del ws_hold          # (released only now, after the kernels that use it were enqueued)
    if rc != OBC_OK:
        raise ObcError(rc, "obc_select")
    return keep_idx


def obc_select_protected(scores: torch.Tensor, num_hh: int, num_sinks: int = 0, num_recent: int = 0,
                         num_coming: int = 0, seq_lens=None, keep_idx: Optional[torch.Tensor] = None,
                         workspace=None) -> torch.Tensor:
    """scores [B,Hkv,N] fp32 -> keep_idx [B,Hkv,num_sinks+num_hh+num_recent-num_coming] int32 ascending."""
    _require_cuda(scores)
    if scores.dtype != torch.float32 or scores.dim() != 3:
        raise ValueError("scores must be [B,Hkv,N] float32")
    B, Hkv, N = scores.shape
    total = int(num_sinks) + int(num_hh) + int(num_recent) - int(num_coming)
    if keep_idx is None:
        keep_idx = torch.empty((B, Hkv, max(total, 0)), dtype=torch.int32, device=scores.device)
    elif keep_idx.dtype != torch.int32 or tuple(keep_idx.shape) != (B, Hkv, total) or not keep_idx.is_contiguous():
        raise ValueError("keep_idx must be a contiguous [B,Hkv,%d] int32 tensor" % total)
    ws_ptr, ws_bytes, ws_hold = _select_ws(scores, workspace)
    rc = load_library().obc_select_protected(scores.data_ptr(), int(num_hh), int(num_sinks), int(num_recent),
                                             int(num_coming), keep_idx.data_ptr(), B, Hkv, N,
                                             _lens_arg(seq_lens, B), ws_ptr, ws_bytes, _stream_ptr(scores))
    del ws_hold
    if rc != OBC_OK:
        raise ObcError(rc, "obc_select_protected")
    return keep_idx


def obc_select_pooled(scores: torch.Tensor, num_hh: int, pool: int = 5, num_sinks: int = 0, num_recent: int = 0,
                      num_coming: int = 0, seq_lens=None, keep_idx: Optional[torch.Tensor] = None,
                      workspace=None) -> torch.Tensor:
    """Like obc_select_protected, competitors ranked by their centred window sum of `pool` scores."""
    _require_cuda(scores)
    if scores.dtype != torch.float32 or scores.dim() != 3:
        raise ValueError("scores must be [B,Hkv,N] float32")
    B, Hkv, N = scores.shape
    total = int(num_sinks) + int(num_hh) + int(num_recent) - int(num_coming)
    if keep_idx is None:
        keep_idx = torch.empty((B, Hkv, max(total, 0)), dtype=torch.int32, device=scores.device)
    elif keep_idx.dtype != torch.int32 or tuple(keep_idx.shape) != (B, Hkv, total) or not keep_idx.is_contiguous():
        raise ValueError("keep_idx must be a contiguous [B,Hkv,%d] int32 tensor" % total)
    ws_ptr, ws_bytes, ws_hold = _select_ws(scores, workspace)
    rc = load_library().obc_select_pooled(scores.data_ptr(), int(num_hh), int(num_sinks), int(num_recent),
                                          int(num_coming), int(pool), keep_idx.data_ptr(), B, Hkv, N,
                                          _lens_arg(seq_lens, B), ws_ptr, ws_bytes, _stream_ptr(scores))
    del ws_hold
    if rc != OBC_OK:
        raise ObcError(rc, "obc_select_pooled")
    return keep_idx


def obc_select_adaptive(scores: torch.Tensor, budget: int, n_safe: int, cap: Optional[int] = None, seq_lens=None,
                        workspace: Optional[torch.Tensor] = None):
    """Head-adaptive budgets: (keep_idx [B,Hkv,cap] int32 ascending then -1, counts [B,Hkv] int32)."""
    _require_cuda(scores)
    if scores.dtype != torch.float32 or scores.dim() != 3:
        raise ValueError("scores must be [B,Hkv,N] float32")
    B, Hkv, N = scores.shape
    if cap is None:
        longest = N if seq_lens is None else max(int(x) for x in seq_lens)
        cap = min(longest, Hkv * int(budget) - (Hkv - 1) * int(n_safe))
    if workspace is None:
        need = ctypes.c_size_t(0)
        rc = load_library().obc_select_adaptive_workspace_bytes(B, Hkv, N, int(budget), int(n_safe), ctypes.byref(need))
        if rc != OBC_OK:
            raise ObcError(rc, "obc_select_adaptive_workspace_bytes")
        workspace = torch.empty(max(int(need.value), 256), dtype=torch.uint8, device=scores.device)
    keep_idx = torch.empty((B, Hkv, max(int(cap), 0)), dtype=torch.int32, device=scores.device)
    counts = torch.empty((B, Hkv), dtype=torch.int32, device=scores.device)
    rc = load_library().obc_select_adaptive(scores.data_ptr(), int(budget), int(n_safe), keep_idx.data_ptr(),
                                            counts.data_ptr(), int(cap), B, Hkv, N, _lens_arg(seq_lens, B),
                                            workspace.data_ptr(), workspace.numel(), _stream_ptr(scores))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_select_adaptive")
    return keep_idx, counts


def _require_room(out: torch.Tensor, nbytes: int):
    _require_cuda(out)
    if out.numel() * out.element_size() < nbytes:
        raise ValueError("k_out, v_out need room for [B,Hkv,budget,d]")


def _kept(k: torch.Tensor, v: torch.Tensor, keep_idx: torch.Tensor):
    """Shape and type of caches and the rows kept per head, where they fit together (rows are moved by k's bytes)."""
    if not (k.is_cuda and v.is_cuda and keep_idx.is_cuda and k.is_contiguous() and v.is_contiguous() and keep_idx.is_contiguous()):
        raise ValueError("tensors must be contiguous and on the GPU")
    shape, kept, dtype = k.shape, keep_idx.shape, k.dtype
    if (len(kept) < 3 and kept[1:] != (1,) or kept[0] != shape[0] or kept[1] != shape[1] or keep_idx.dtype is not _I32 or v.shape != shape
            or v.dtype is not dtype and v.element_size() != k.element_size()):
        raise ValueError("keep_idx must be [B,Hkv,budget] int32 matching k, v")
    return shape, dtype, kept[-1]


def obc_compact(k: torch.Tensor, v: torch.Tensor, keep_idx: torch.Tensor, k_out=None, v_out=None):
    """k,v [B,Hkv,N,d], keep_idx [B,Hkv,budget] int32 -> (k_out, v_out) [B,Hkv,budget,d]."""
    (B, Hkv, N, d), dtype, budget = _kept(k, v, keep_idx)
    rows = B * Hkv * budget * d
    if k_out is None:
        k_out = torch.empty((B, Hkv, budget, d), dtype=dtype, device=k.device)
    elif not (k_out.dtype is dtype and k_out.numel() >= rows and k_out.is_cuda and k_out.is_contiguous()):
        _require_room(k_out, rows * k.element_size())
    if v_out is None:
        v_out = torch.empty((B, Hkv, budget, d), dtype=v.dtype, device=v.device)
    elif not (v_out.dtype is dtype and v_out.numel() >= rows and v_out.is_cuda and v_out.is_contiguous()):
        _require_room(v_out, rows * k.element_size())
    rc = (_lib or load_library()).obc_compact(
        k.data_ptr(), v.data_ptr(), keep_idx.data_ptr(), k_out.data_ptr(), v_out.data_ptr(), B, Hkv, N, budget, d,
        OBC_BF16 if dtype is _BF16 else _dtype_code(k), _raw_stream(k.get_device()) if _raw_stream is not None else _stream_ptr(k))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_compact")
    return k_out, v_out


def obc_compact_inplace(k: torch.Tensor, v: torch.Tensor, keep_idx: torch.Tensor,
                        scores: Optional[torch.Tensor] = None) -> None:
    """Moves rows keep_idx[b,g,j] of k, v (and entries of scores, whose tail is zeroed) to position j, in place."""
    (B, Hkv, N, d), dtype, budget = _kept(k, v, keep_idx)
    sp = None
    if scores is not None:
        _require_cuda(scores)
        if tuple(scores.shape) != (B, Hkv, N) or scores.dtype != torch.float32 or not scores.is_contiguous():
            raise ValueError("scores must be a contiguous [B,Hkv,N] float32 tensor")
        sp = scores.data_ptr()
    rc = load_library().obc_compact_inplace(k.data_ptr(), v.data_ptr(), sp, keep_idx.data_ptr(), B, Hkv, N, budget, d,
                                            OBC_BF16 if dtype is _BF16 else _dtype_code(k), _stream_ptr(k))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_compact_inplace")


def obc_decode_step_workspace_bytes(B, N, Hq, Hkv, d, dtype, variant) -> int:
    out = ctypes.c_size_t(0)
    rc = load_library().obc_decode_step_workspace_bytes(B, N, Hq, Hkv, d, dtype, variant, ctypes.byref(out))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_decode_step_workspace_bytes")
    return int(out.value)


def obc_decode_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scores: torch.Tensor, variant="joint",
                    num_sinks: int = 0, num_recent: int = 0, seq_lens=None, evicted: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Accumulates the new row's scores, drops the lowest-scored unprotected token of every head and closes the gap in
    k, v and scores, all in place.  Returns the dropped positions [B,Hkv] int32."""
    # (A call per layer and token, as long on the host as on the GPU: no loop over the tensors, nothing asked twice.)
    if not (q.is_cuda and k.is_cuda and v.is_cuda and scores.is_cuda and q.is_contiguous() and k.is_contiguous()
            and v.is_contiguous() and scores.is_contiguous()):
        raise ValueError("tensors must be contiguous and on the GPU")
    B, Hq, W, d = q.shape
    kv_shape, dtype = k.shape, q.dtype
    Bk, Hkv, N, dk = kv_shape
    if not (W == 1 and Bk == B and dk == d and v.shape == kv_shape and k.dtype is dtype and v.dtype is dtype
            and scores.shape == (B, Hkv, N) and scores.dtype is _F32):
        raise ValueError("q must be [B,Hq,1,d], k, v [B,Hkv,N,d] of its type, scores [B,Hkv,N] float32")
    var = VARIANT_CODES[variant] if type(variant) is str else _variant_code(variant)
    dt = OBC_BF16 if dtype is _BF16 else _dtype_code(q)
    if workspace is None:
        workspace = torch.empty(obc_decode_step_workspace_bytes(B, N, Hq, Hkv, d, dt, var), dtype=torch.uint8, device=q.device)
    if evicted is None:
        evicted = torch.empty((B, Hkv), dtype=torch.int32, device=q.device)
    if not (evicted.is_cuda and workspace.is_cuda and evicted.is_contiguous() and workspace.is_contiguous()):
        raise ValueError("tensors must be contiguous and on the GPU")
    if evicted.dtype is not _I32 or evicted.numel() < B * Hkv:
        raise ValueError("evicted must be int32 with room for [B,Hkv]")
    rc = (_lib or load_library()).obc_decode_step(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), scores.data_ptr(), evicted.data_ptr(), N, Hq, Hkv, d, var, B, dt,
        None if seq_lens is None else _lens_arg(seq_lens, B), num_sinks if type(num_sinks) is int else int(num_sinks),
        num_recent if type(num_recent) is int else int(num_recent), workspace.data_ptr(), workspace.numel(),
        _raw_stream(q.get_device()) if _raw_stream is not None else _stream_ptr(q))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_decode_step")
    return evicted


def obc_compact_scores(scores: torch.Tensor, keep_idx: torch.Tensor, n_out: Optional[int] = None,
                       scores_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scores [B,Hkv,N] fp32, keep_idx [B,Hkv,budget] -> [B,Hkv,n_out]: gathered scores, then zeros."""
    _require_cuda(scores, keep_idx)
    B, Hkv, N = scores.shape
    budget = keep_idx.shape[-1]
    if scores.dtype != torch.float32 or keep_idx.dtype != torch.int32 or tuple(keep_idx.shape[:2]) != (B, Hkv):
        raise ValueError("scores must be [B,Hkv,N] float32 and keep_idx [B,Hkv,budget] int32")
    n_out = budget if n_out is None else int(n_out)
    if scores_out is None:
        scores_out = torch.empty((B, Hkv, n_out), dtype=torch.float32, device=scores.device)
    elif tuple(scores_out.shape) != (B, Hkv, n_out) or scores_out.dtype != torch.float32 or not scores_out.is_contiguous():
        raise ValueError("scores_out must be a contiguous [B,Hkv,%d] float32 tensor" % n_out)
    rc = load_library().obc_compact_scores(scores.data_ptr(), keep_idx.data_ptr(), scores_out.data_ptr(), B, Hkv, N,
                                           budget, n_out, _stream_ptr(scores))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_compact_scores")
    return scores_out


class KvCache:
    """The cache of one layer that obc_cache_append, obc_attend and obc_cache_read work on.

    k, v [P,Hkv,S,d] float32, bfloat16 or float8_e4m3fn, the latter with k_scale, v_scale [P,Hkv,S,d/32] uint8; page_table [B,M]
    int32, or None: page b is all of sequence b, so that the library's [B,Hkv,N,d] caches serve as they are.  Tensors are
    checked here, once; the handle keeps them and their addresses, so they are written to but not exchanged: other tensors, a
    table of more pages for one, take a handle of their own."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: Optional[torch.Tensor] = None,
                 k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None):
        _require_cuda(k, v)
        if k.dim() != 4 or v.shape != k.shape or v.dtype is not k.dtype or v.device != k.device:
            raise ValueError("k, v must be [P,Hkv,S,d] of one type")
        codes = {_F32: OBC_F32, _BF16: OBC_BF16, _E4M3: OBC_E4M3}
        if k.dtype not in codes:
            raise TypeError("a cache is float32, bfloat16 or float8_e4m3fn, got %s" % k.dtype)
        P, Hkv, S, d = k.shape
        if 0 in k.shape or d not in (64, 128):
            raise ValueError("a cache has pages, heads and rows of 64 or 128 channels")
        if k.dtype is _E4M3:
            for x in (k_scale, v_scale):
                if x is None or x.dtype is not _U8 or tuple(x.shape) != (P, Hkv, S, d // 32) or x.device != k.device:
                    raise ValueError("an 8-bit cache needs k_scale, v_scale [P,Hkv,S,%d] uint8" % (d // 32))
                _require_cuda(x)
        elif k_scale is not None or v_scale is not None:
            raise ValueError("scales belong to an 8-bit cache")
        if page_table is not None:
            _require_cuda(page_table)
            if page_table.dim() != 2 or page_table.dtype is not _I32 or page_table.device != k.device or 0 in page_table.shape:
                raise ValueError("page_table must be [B,M] int32")
            if S & (S - 1):
                raise ValueError("pages of a table hold a power of two of rows")
        batch, pages = (P, 1) if page_table is None else tuple(page_table.shape)
        if pages * S > 1 << 30 or batch * Hkv > 65535:
            raise ValueError("at most 2^30 rows per sequence and 65535 KV heads over the batch")
        ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        self.__dict__.update(
            k=k, v=v, k_scale=k_scale, v_scale=v_scale, page_table=page_table, batch=batch, Hkv=Hkv, d=d, dtype=k.dtype, device=k.device,
            capacity=pages * S, _index=k.get_device(),
            _arg=_CacheArg(ptr(k), ptr(v), ptr(k_scale), ptr(v_scale), ptr(page_table), batch, P, pages, S, Hkv, d, codes[k.dtype]))

    _FIXED = frozenset(("k", "v", "k_scale", "v_scale", "page_table", "batch", "Hkv", "d", "dtype", "device", "capacity", "_index", "_arg"))

    def __setattr__(self, name, value):
        if name in self._FIXED:
            raise AttributeError("a cache's tensors are not exchanged: make another KvCache")
        object.__setattr__(self, name, value)

    def __delattr__(self, name):
        if name in self._FIXED:
            raise AttributeError("a cache's tensors are not exchanged: make another KvCache")
        object.__delattr__(self, name)

    @classmethod
    def empty(cls, num_pages: int, Hkv: int, page_size: int, d: int, dtype=torch.bfloat16, page_table=None, device="cuda"):
        """A cache of its own memory, not initialised."""
        k, v = (torch.empty((num_pages, Hkv, page_size, d), dtype=dtype, device=device) for _ in range(2))
        ks = vs = None
        if dtype is _E4M3:
            ks, vs = (torch.empty((num_pages, Hkv, page_size, d // 32), dtype=_U8, device=device) for _ in range(2))
        return cls(k, v, page_table, ks, vs)

    def _ints(self, t: torch.Tensor, what: str, per_head: bool = True) -> int:
        """1 for lengths [B,Hkv], 0 for [B]."""
        if t.dtype is _I32 and t.get_device() == self._index and t.is_contiguous():
            shape = t.shape
            if shape == (self.batch,):
                return 0
            if per_head and shape == (self.batch, self.Hkv):
                return 1
        raise ValueError("%s must be contiguous int32 [B]%s on the cache's GPU" % (what, " or [B,Hkv]" if per_head else ""))

    def _launch(self, call, args):
        """call(*args, stream) on the current stream of the cache's GPU, with that one current."""
        index = self._index
        if index == torch.cuda.current_device():
            return call(*args, _raw_stream(index) if _raw_stream is not None else _stream_ptr(self.k))
        with torch.cuda.device(index):
            return call(*args, _stream_ptr(self.k))


def obc_cache_append(cache: KvCache, k: torch.Tensor, v: torch.Tensor, lens: torch.Tensor, q: Optional[torch.Tensor] = None,
                     q_out: Optional[torch.Tensor] = None, new_lens: Optional[torch.Tensor] = None,
                     positions: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None, rot_scale: float = 1.0,
                     interleaved: bool = False, q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None,
                     eps: float = 1e-6) -> Optional[torch.Tensor]:
    """k, v [B,T,Hkv,d] (and q [B,T,Hq,d]), any strides over whole rows, normed, rotated and written: k, v to rows lens - n .. lens - 1
    of the cache, q to q_out [B,Hq,T,d], which is returned.  lens [B] or [B,Hkv] int32 counts the new rows in; new_lens [B] int32
    (without q also [B,Hkv]): the first n of the T are new; positions [B,T] int32 and inv_freq [pairs] float32 turn on the rotation."""
    # (A call per layer and token, like obc_decode_step: nothing is asked twice.)
    index, dtype, shape = cache._index, k.dtype, k.shape
    if len(shape) != 4 or shape[0] != cache.batch or shape[2] != cache.Hkv or shape[3] != cache.d or k.get_device() != index:
        raise ValueError("k must be [B,T,Hkv,d] on the cache's GPU")
    if dtype is not cache.dtype and cache.dtype is not _E4M3:
        raise ValueError("rows and cache must be of one type, or the cache of 8 bits")
    if v.shape != shape or v.dtype is not dtype or v.get_device() != index:
        raise ValueError("v must be like k")
    B, T, _, d = shape
    kb, kt, kh, kc = k.stride()
    vb, vt, vh, vc = v.stride()
    if kc != 1 or vc != 1:
        raise ValueError("the channels of a row must be contiguous")
    per_head = cache._ints(lens, "lens")
    new_ptr, new_per_head = (None, 0) if new_lens is None else (new_lens.data_ptr(), cache._ints(new_lens, "new_lens", q is None))
    q_arg, q_ptr, Hq = None, None, 0
    if q is not None:
        q_shape = q.shape
        if len(q_shape) != 4 or q_shape[0] != B or q_shape[1] != T or q_shape[3] != d or q.dtype is not dtype or q.get_device() != index:
            raise ValueError("q must be [B,T,Hq,d] and fit k")
        Hq = q_shape[2]
        if Hq < 1 or Hq % cache.Hkv:
            raise ValueError("q needs a multiple of Hkv heads")
        qb, qt, qh, qc = q.stride()
        if qc != 1:
            raise ValueError("the channels of a row must be contiguous")
        q_arg = _RowsArg(q.data_ptr(), qb, qt, qh)
        if q_out is None:
            q_out = torch.empty((B, Hq, T, d), dtype=dtype, device=k.device)
        elif q_out.shape != (B, Hq, T, d) or q_out.dtype is not dtype or q_out.get_device() != index or not q_out.is_contiguous():
            raise ValueError("q_out must be contiguous [B,Hq,T,d] of q's type")
        q_ptr = q_out.data_ptr()
    elif q_out is not None or q_norm is not None:
        raise ValueError("q_out and q_norm belong to q")
    pos_ptr, freq_ptr, pairs = None, None, 0
    if inv_freq is not None and positions is not None:
        pairs = inv_freq.numel()
        if (inv_freq.dtype is not _F32 or inv_freq.get_device() != index or not inv_freq.is_contiguous() or positions.dtype is not _I32
                or positions.shape != (B, T) or positions.get_device() != index or not positions.is_contiguous() or pairs < 1):
            raise ValueError("positions must be contiguous [B,T] int32, inv_freq [pairs] float32, on the cache's GPU")
        pos_ptr, freq_ptr = positions.data_ptr(), inv_freq.data_ptr()
    elif inv_freq is not None or positions is not None:
        raise ValueError("positions and inv_freq belong together")
    norms = [None, None]
    if q_norm is not None or k_norm is not None:
        for i, w in enumerate((q_norm, k_norm)):
            if w is not None:
                if w.shape != (d,) or w.dtype is not dtype or w.get_device() != index or not w.is_contiguous():
                    raise ValueError("q_norm, k_norm must be contiguous [d] of the rows' type")
                norms[i] = w.data_ptr()
    rc = cache._launch((_lib or load_library()).obc_cache_append, (
        q_arg, _RowsArg(k.data_ptr(), kb, kt, kh), _RowsArg(v.data_ptr(), vb, vt, vh), cache._arg, q_ptr, lens.data_ptr(), per_head, new_ptr,
        new_per_head, pos_ptr, freq_ptr, pairs, rot_scale, 1 if interleaved else 0, norms[0], norms[1], eps, B, T, Hq,
        OBC_BF16 if dtype is _BF16 else _dtype_code(k)))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_cache_append")
    return q_out


def obc_attend_workspace_bytes(B: int, T: int, Hq: int, cache: KvCache, dtype) -> int:
    """dtype: the queries', a torch type or its code."""
    out = ctypes.c_size_t(0)
    code = {_F32: OBC_F32, _BF16: OBC_BF16}.get(dtype, dtype)
    if not isinstance(code, int):
        raise TypeError("queries are float32 or bfloat16, got %s" % dtype)
    rc = load_library().obc_attend_workspace_bytes(B, T, Hq, cache._arg, code, ctypes.byref(out))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_attend_workspace_bytes")
    return int(out.value)


def obc_attend(q: torch.Tensor, cache: KvCache, lens: torch.Tensor, new_lens: Optional[torch.Tensor] = None, causal: bool = True,
               scale: Optional[float] = None, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """q [B,Hq,T,d] over the first lens rows of the cache, the last n of which are the new rows themselves -> out [B,T,Hq,d].
    lens [B] or [B,Hkv] int32, new_lens [B] int32 (None: T); scale defaults to 1/sqrt(d)."""
    if not (q.is_cuda and q.is_contiguous() and q.dim() == 4):
        raise ValueError("tensors must be contiguous and on the GPU")
    B, Hq, T, d = q.shape
    if B != cache.batch or d != cache.d or q.get_device() != cache._index or 0 in q.shape or Hq % cache.Hkv:
        raise ValueError("q must be [B,Hq,T,d] and fit the cache")
    dtype = q.dtype
    if dtype is not cache.dtype and cache.dtype is not _E4M3:
        raise ValueError("queries and cache must be of one type, or the cache of 8 bits")
    code = OBC_BF16 if dtype is _BF16 else _dtype_code(q)
    per_head = cache._ints(lens, "lens")
    if new_lens is not None:
        cache._ints(new_lens, "new_lens", False)
    if out is None:
        out = torch.empty((B, T, Hq, d), dtype=dtype, device=q.device)
    elif out.shape != (B, T, Hq, d) or out.dtype is not dtype or out.get_device() != cache._index or not out.is_contiguous():
        raise ValueError("out must be contiguous [B,T,Hq,d] of q's type")
    if workspace is None:
        workspace = torch.empty(obc_attend_workspace_bytes(B, T, Hq, cache, code), dtype=_U8, device=q.device)
    elif not (workspace.is_cuda and workspace.is_contiguous() and workspace.get_device() == cache._index):
        raise ValueError("workspace must be contiguous and on the cache's GPU")
    rc = cache._launch((_lib or load_library()).obc_attend, (
        q.data_ptr(), cache._arg, out.data_ptr(), lens.data_ptr(), per_head, None if new_lens is None else new_lens.data_ptr(), B, T, Hq, code,
        1 if causal else 0, d ** -0.5 if scale is None else scale, workspace.data_ptr(), workspace.numel() * workspace.element_size()))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_attend")
    return out


def obc_cache_read(cache: KvCache, n: Optional[int] = None, keep_idx: Optional[torch.Tensor] = None, dtype=None,
                   k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None):
    """Rows keep_idx [B,Hkv,n] int32 (None: the first n) of the cache -> (k_out, v_out) [B,Hkv,n,d] of the cache's type, or of an
    8-bit cache as `dtype` (bfloat16 if neither that nor outputs are given)."""
    if keep_idx is not None:
        if (keep_idx.dim() != 3 or keep_idx.shape[:2] != (cache.batch, cache.Hkv) or keep_idx.dtype is not _I32
                or not keep_idx.is_contiguous() or keep_idx.get_device() != cache._index):
            raise ValueError("keep_idx must be contiguous [B,Hkv,n] int32 on the cache's GPU")
        if n is not None and n != keep_idx.shape[2]:
            raise ValueError("n and keep_idx disagree")
        n = keep_idx.shape[2]
    elif n is None:
        raise ValueError("either n or keep_idx says which rows")
    n = int(n)
    if n < 1 or keep_idx is None and n > cache.capacity:
        raise ValueError("the cache has rows 0 .. %d" % (cache.capacity - 1))
    if dtype is None:
        given = k_out if k_out is not None else v_out
        dtype = given.dtype if given is not None else _BF16 if cache.dtype is _E4M3 else cache.dtype
    if dtype is not cache.dtype and cache.dtype is not _E4M3 or dtype not in (_F32, _BF16):
        raise ValueError("rows are given back in the cache's type, of an 8-bit cache in float32 or bfloat16")
    shape = (cache.batch, cache.Hkv, n, cache.d)
    outs = []
    for x in (k_out, v_out):
        if x is None:
            x = torch.empty(shape, dtype=dtype, device=cache.device)
        elif x.shape != shape or x.dtype is not dtype or x.get_device() != cache._index or not x.is_contiguous():
            raise ValueError("k_out, v_out must be contiguous [B,Hkv,n,d] of one type on the cache's GPU")
        outs.append(x)
    rc = cache._launch((_lib or load_library()).obc_cache_read, (
        cache._arg, None if keep_idx is None else keep_idx.data_ptr(), outs[0].data_ptr(), outs[1].data_ptr(), cache.batch, n,
        OBC_F32 if dtype is _F32 else OBC_BF16))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_cache_read")
    return outs[0], outs[1]


OBC_PROBE_BLOCKS = 2048


def obc_probe_read_bandwidth(buf: torch.Tensor, sink: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Measurement hook: one streaming read of `buf` (time it with events around the call)."""
    if sink is None:
        sink = torch.empty(OBC_PROBE_BLOCKS * 256, dtype=torch.int32, device=buf.device)
    nbytes = buf.numel() * buf.element_size()
    rc = load_library().obc_probe_read_bandwidth(buf.data_ptr(), nbytes, sink.data_ptr(), _stream_ptr(buf))
    if rc != OBC_OK:
        raise ObcError(rc, "obc_probe_read_bandwidth")
    return sink
