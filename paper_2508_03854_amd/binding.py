"""Thin ctypes binding of libtbe355.so: same names as the C ABI, argument marshalling only.

torch is used for device memory and streams: with stream=, results that are not given are allocated on that stream, and whoever uses them
on another one waits for it, as for any work there.  There is no fallback: if the HIP library is missing or a
call fails, an exception is raised."""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Dict, List, Optional, Sequence, Tuple

import torch  # must be imported before the library so that both share one HIP runtime

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libtbe355.so")

OK, EINVAL, ESHAPE, EDTYPE, EWORKSPACE, EINDEX, EHIP = range(7)
STATIC_SCRATCH_BYTES = 64 << 20        # TBE_STATIC_SCRATCH_BYTES
F32, F16 = 0, 1
SUM, MEAN = 0, 1
I64, I32 = 0, 1                       # tbe_index_dtype
IO_F32, IO_F16, IO_BF16 = 0, 1, 2     # tbe_io_dtype
CODE_E4M3, CODE_I8 = 0, 1             # tbe_code
_CODE = {torch.float8_e4m3fn: CODE_E4M3, torch.int8: CODE_I8}
ROTARY_SCALING = {"plain": 0, "linear": 1, "base": 2, "turns": 3}   # tbe_rotary_scaling
FWD_WAVEFRONT_PER_BAG, FWD_LANE_GROUPS, FWD_HOT_ROWS, FWD_LONG_BAGS = 1, 2, 4, 8   # TBE_FWD_*
TUNABLES = {"hot_rows_min_workgroups": 0}   # tbe_tunable
TUNE_AUTO = -(1 << 63)                 # TBE_TUNE_AUTO
_IDX = {torch.int64: I64, torch.int32: I32}
_IO = {torch.float32: IO_F32, torch.float16: IO_F16, torch.bfloat16: IO_BF16}

# every symbol include/tbe355.h declares
EXPORTS = ["tbe_create", "tbe_destroy", "tbe_workspace_bytes", "tbe_forward", "tbe_backward_rowwise_adagrad",
           "tbe_forward_ex", "tbe_backward_rowwise_adagrad_ex", "tbe_backward_rowwise_adagrad_static", "tbe_backward_prepare",
           "tbe_backward_apply_rowwise_adagrad", "tbe_backward_apply_sgd", "tbe_backward_sgd", "tbe_replica_mean", "tbe_lookup_seq",
           "tbe_backward_seq_rowwise_adagrad", "tbe_debug_sorted", "tbe_debug_hot_rows", "tbe_debug_forward_kernels", "tbe_poll_index_error", "tbe_set_tunable", "tbe_timing_enable",
           "tbe_timing_count", "tbe_timing_read", "tbe_calibration_copy", "tbe_calibration_gather", "tbe_status_string", "tbe_build_info",
           "tbe_layer_norm", "tbe_layer_norm_workspace_bytes", "tbe_layer_norm_backward", "tbe_attention_workspace_bytes", "tbe_attention", "tbe_attention_backward",
           "tbe_rotate_heads", "tbe_rotate_workspace_bytes", "tbe_rotate_heads_backward", "tbe_rotary_frequencies",
           "tbe_cache_write", "tbe_cache_read", "tbe_cache_attention_workspace_bytes", "tbe_cache_attention"]


class TbeError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: status {status} ({_status_string(status)})")
        self.status = status


class Rows(ctypes.Structure):
    """tbe_rows"""
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class AttentionArgs(ctypes.Structure):
    """tbe_attention_args"""
    _fields_ = [("sequences", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("q_rows", ctypes.c_int64), ("k_rows", ctypes.c_int64), ("dtype", ctypes.c_int), ("index_dtype", ctypes.c_int),
                ("q", Rows), ("k", Rows), ("v", Rows), ("q_offsets", ctypes.c_void_p), ("k_offsets", ctypes.c_void_p),
                ("k_lengths", ctypes.c_void_p), ("causal", ctypes.c_int32), ("scale", ctypes.c_float), ("bias", ctypes.c_void_p),
                ("bucket_map", ctypes.c_void_p), ("bias_dtype", ctypes.c_int), ("buckets", ctypes.c_int32), ("max_distance", ctypes.c_int32)]


class RotationArgs(ctypes.Structure):
    """tbe_rotation_args"""
    _fields_ = [("q_heads", ctypes.c_int32), ("k_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32),
                ("rows", ctypes.c_int64), ("dtype", ctypes.c_int), ("index_dtype", ctypes.c_int), ("positions", ctypes.c_void_p),
                ("frequencies", ctypes.c_void_p), ("interleaved", ctypes.c_int32), ("amplitude", ctypes.c_float), ("norm", ctypes.c_int32),
                ("eps", ctypes.c_float), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("weight_dtype", ctypes.c_int)]


class CacheArgs(ctypes.Structure):
    """tbe_cache"""
    _fields_ = [("rows", ctypes.c_int64), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("code", ctypes.c_int), ("k", Rows), ("v", Rows),
                ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p)]


# The same fields packed in one go: filling the structure field by field takes 6 us of a call that is otherwise over in ten.
_PACK_ATTENTION = struct.Struct("@4i2q2i" + "Pqq" * 3 + "3Pif2P3i4x").pack
_PACK_CACHE = struct.Struct("@q3i4xPqqPqq2P").pack
_PACK_ROTATION = struct.Struct("@4iq2i2Pifif2Pi4x").pack

_lib = None


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads libtbe355.so; raises if it has not been built (python -m paper_2508_03854_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(f"{_LIB_PATH} is missing: build it with `python paper_2508_03854_amd/build.py`")
    L = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    L.tbe_create.restype = ctypes.c_int
    L.tbe_create.argtypes = [i32, ctypes.POINTER(i64), ctypes.POINTER(i32), ctypes.c_int, ctypes.POINTER(vp)]
    L.tbe_destroy.restype = ctypes.c_int
    L.tbe_destroy.argtypes = [vp]
    L.tbe_workspace_bytes.restype = ctypes.c_int
    L.tbe_workspace_bytes.argtypes = [vp, i32, i64, ctypes.POINTER(ctypes.c_size_t)]
    L.tbe_forward.restype = ctypes.c_int
    L.tbe_forward.argtypes = [vp, vp, vp, vp, vp, i32, i64, ctypes.c_int, vp, vp]
    L.tbe_backward_rowwise_adagrad.restype = ctypes.c_int
    L.tbe_backward_rowwise_adagrad.argtypes = [vp, vp, vp, vp, i32, i64, ctypes.c_int, f32, f32, f32, vp, vp, vp,
                                               ctypes.c_size_t, vp]
    L.tbe_forward_ex.restype = ctypes.c_int
    L.tbe_forward_ex.argtypes = [vp, vp, vp, vp, vp, ctypes.c_int, i32, i64, ctypes.c_int, vp, ctypes.c_int, vp]
    L.tbe_backward_rowwise_adagrad_ex.restype = ctypes.c_int
    L.tbe_backward_rowwise_adagrad_ex.argtypes = [vp, vp, ctypes.c_int, vp, vp, ctypes.c_int, i32, i64, ctypes.c_int,
                                                  f32, f32, f32, vp, vp, vp, ctypes.c_size_t, vp]
    L.tbe_backward_rowwise_adagrad_static.restype = ctypes.c_int
    L.tbe_backward_rowwise_adagrad_static.argtypes = [vp, vp, ctypes.c_int, vp, vp, ctypes.c_int, i32, i64, ctypes.c_int,
                                                      f32, f32, f32, vp, vp, vp]
    L.tbe_backward_prepare.restype = ctypes.c_int
    L.tbe_backward_prepare.argtypes = [vp, vp, vp, ctypes.c_int, i32, i64, vp, ctypes.c_size_t, vp]
    L.tbe_backward_apply_rowwise_adagrad.restype = ctypes.c_int
    L.tbe_backward_apply_rowwise_adagrad.argtypes = [vp, vp, ctypes.c_int, vp, ctypes.c_int, i32, i64, ctypes.c_int,
                                                     f32, f32, f32, vp, vp, vp, ctypes.c_size_t, vp]
    L.tbe_backward_apply_sgd.restype = ctypes.c_int
    L.tbe_backward_apply_sgd.argtypes = [vp, vp, ctypes.c_int, vp, ctypes.c_int, i32, i64, ctypes.c_int, f32, vp, vp,
                                         ctypes.c_size_t, vp]
    L.tbe_backward_sgd.restype = ctypes.c_int
    L.tbe_backward_sgd.argtypes = [vp, vp, ctypes.c_int, vp, vp, ctypes.c_int, i32, i64, ctypes.c_int, f32, vp, vp,
                                   ctypes.c_size_t, vp]
    L.tbe_lookup_seq.restype = ctypes.c_int
    L.tbe_lookup_seq.argtypes = [vp, vp, vp, vp, ctypes.c_int, i64, vp, ctypes.c_int, i64, vp]
    L.tbe_backward_seq_rowwise_adagrad.restype = ctypes.c_int
    L.tbe_backward_seq_rowwise_adagrad.argtypes = [vp, vp, ctypes.c_int, i64, vp, vp, ctypes.c_int, i64, f32, f32, f32,
                                                   vp, vp, vp, ctypes.c_size_t, vp]
    L.tbe_replica_mean.restype = ctypes.c_int
    L.tbe_replica_mean.argtypes = [vp, ctypes.POINTER(vp), i32, ctypes.c_size_t, ctypes.c_int, vp]
    L.tbe_debug_sorted.restype = ctypes.c_int
    L.tbe_debug_sorted.argtypes = [vp, vp, i32, i64] + [ctypes.POINTER(vp)] * 5
    L.tbe_debug_hot_rows.restype = ctypes.c_int
    L.tbe_debug_hot_rows.argtypes = [vp, vp, i32, i64] + [ctypes.POINTER(vp)] * 5
    L.tbe_debug_forward_kernels.restype = ctypes.c_int
    L.tbe_debug_forward_kernels.argtypes = [vp, i32, i64, ctypes.POINTER(ctypes.c_uint32)]
    L.tbe_poll_index_error.restype = ctypes.c_int
    L.tbe_poll_index_error.argtypes = [vp]
    L.tbe_set_tunable.restype = ctypes.c_int
    L.tbe_set_tunable.argtypes = [vp, ctypes.c_int, i64]
    L.tbe_timing_enable.restype = ctypes.c_int
    L.tbe_timing_enable.argtypes = [vp, ctypes.c_int]
    L.tbe_timing_count.restype = ctypes.c_int
    L.tbe_timing_count.argtypes = [vp, ctypes.POINTER(i32)]
    L.tbe_timing_read.restype = ctypes.c_int
    L.tbe_timing_read.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(f32)]
    L.tbe_calibration_copy.restype = ctypes.c_int
    L.tbe_calibration_copy.argtypes = [vp, vp, vp, ctypes.c_size_t, vp]
    L.tbe_calibration_gather.restype = ctypes.c_int
    L.tbe_calibration_gather.argtypes = [vp, vp, ctypes.c_size_t, ctypes.c_size_t, i32, i32, i64, i32, vp,
                                         ctypes.c_size_t, vp]
    L.tbe_layer_norm.restype = ctypes.c_int
    L.tbe_layer_norm.argtypes = [vp, vp, i64, ctypes.c_int, i64, i32, vp, vp, ctypes.c_int, f32, vp, i64, vp, vp, vp]
    L.tbe_layer_norm_workspace_bytes.restype = ctypes.c_int
    L.tbe_layer_norm_workspace_bytes.argtypes = [vp, i64, i32, ctypes.POINTER(ctypes.c_size_t)]
    L.tbe_layer_norm_backward.restype = ctypes.c_int
    L.tbe_layer_norm_backward.argtypes = [vp, vp, i64, vp, i64, ctypes.c_int, i64, i32, vp, ctypes.c_int, vp, vp, vp, i64, vp, vp, vp,
                                          ctypes.c_size_t, vp]
    L.tbe_attention_workspace_bytes.restype = ctypes.c_int
    L.tbe_attention_workspace_bytes.argtypes = [vp, vp, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)]
    L.tbe_attention.restype = ctypes.c_int
    L.tbe_attention.argtypes = [vp, vp, Rows, vp, vp, ctypes.c_size_t, vp]
    L.tbe_attention_backward.restype = ctypes.c_int
    L.tbe_attention_backward.argtypes = [vp, vp, Rows, vp, Rows, Rows, Rows, Rows, vp, vp, ctypes.c_size_t, vp]
    L.tbe_rotate_heads.restype = ctypes.c_int
    L.tbe_rotate_heads.argtypes = [vp, vp, Rows, Rows, Rows, Rows, vp]
    L.tbe_rotate_workspace_bytes.restype = ctypes.c_int
    L.tbe_rotate_workspace_bytes.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_size_t)]
    L.tbe_rotate_heads_backward.restype = ctypes.c_int
    L.tbe_rotate_heads_backward.argtypes = [vp, vp, Rows, Rows, Rows, Rows, Rows, Rows, vp, vp, vp, ctypes.c_size_t, vp]
    f64 = ctypes.c_double
    L.tbe_rotary_frequencies.restype = ctypes.c_int
    L.tbe_rotary_frequencies.argtypes = [i32, f64, ctypes.c_int, f64, f64, f64, f64, vp]
    L.tbe_cache_write.restype = ctypes.c_int
    L.tbe_cache_write.argtypes = [vp, vp, Rows, Rows, ctypes.c_int, vp, ctypes.c_int, i64, vp]
    L.tbe_cache_read.restype = ctypes.c_int
    L.tbe_cache_read.argtypes = [vp, vp, vp, ctypes.c_int, i64, Rows, Rows, ctypes.c_int, vp]
    L.tbe_cache_attention_workspace_bytes.restype = ctypes.c_int
    L.tbe_cache_attention_workspace_bytes.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_size_t)]
    L.tbe_cache_attention.restype = ctypes.c_int
    L.tbe_cache_attention.argtypes = [vp, vp, vp, Rows, vp, vp, ctypes.c_size_t, vp]
    L.tbe_build_info.restype = ctypes.c_char_p
    L.tbe_build_info.argtypes = []
    L.tbe_status_string.restype = ctypes.c_char_p
    L.tbe_status_string.argtypes = [ctypes.c_int]
    _lib = L
    return L


def build_info() -> str:
    """tbe_build_info(): "tbe355 gfx950 <digest of the sources the loaded library was built from>"."""
    return load_library().tbe_build_info().decode()


def _status_string(s: int) -> str:
    try:
        return load_library().tbe_status_string(int(s)).decode()
    except Exception:  # pragma: no cover
        return "?"


def _check(status: int, what: str) -> None:
    if status != OK:
        raise TbeError(status, what)


def _dev_ptr(t: Optional[torch.Tensor], dtype: torch.dtype, what: str) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


def _rows_ptr(t: torch.Tensor, like: Optional[torch.Tensor], what: str) -> int:
    """A device matrix whose last axis is contiguous; same type and shape as `like`."""
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if t.dtype not in _IO:
        raise TypeError(f"{what} must be float32, float16 or bfloat16, got {t.dtype}")
    if like is not None and (t.dtype != like.dtype or t.shape != like.shape):
        raise ValueError(f"{what} must be {like.dtype} {tuple(like.shape)}, got {t.dtype} {tuple(t.shape)}")
    if t.stride(-1) != 1 and t.shape[-1] > 1 and t.numel():
        raise ValueError(f"the last axis of {what} must be contiguous")
    return t.data_ptr()


def _heads(t: torch.Tensor, like: Optional[torch.Tensor], what: str) -> Rows:
    """A device matrix [rows, heads, head_dim] whose last axis is contiguous; same type and shape as `like`."""
    if t.dim() != 3:
        raise ValueError(f"{what} must have three axes: rows, heads, head_dim")
    return Rows(_rows_ptr(t, like, what), t.stride(0), t.stride(1))


def _param_ptr(t: Optional[torch.Tensor], n: int, dtype: Optional[torch.dtype], what: str) -> Optional[int]:
    """A parameter vector or table of n elements, or None."""
    if t is None:
        return None
    if t.dtype not in _IO:
        raise TypeError(f"{what} must be float32, float16 or bfloat16, got {t.dtype}")
    if t.numel() != n:
        raise ValueError(f"{what} must have {n} elements, got {t.numel()}")
    return _dev_ptr(t, dtype or t.dtype, what)


def _index_dtype(indices: torch.Tensor, offsets: torch.Tensor) -> int:
    if indices.dtype != offsets.dtype or indices.dtype not in _IDX:
        raise TypeError(f"indices and offsets must both be int64 or both int32, got {indices.dtype} / {offsets.dtype}")
    return _IDX[indices.dtype]


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is not None:
        return stream.cuda_stream
    # torch.cuda.current_stream().cuda_stream, without the 5 us that making the stream object takes
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _empty(shape, dtype: torch.dtype, device, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """A result's tensor, allocated on the stream that writes it: its memory may still be in use by earlier work there, and by that alone."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, context: float = 0.0,
                       low_turns: float = 1.0, high_turns: float = 32.0, device="cuda") -> torch.Tensor:
    """tbe_rotary_frequencies: float64 [rotary_dim / 2] on `device`; scaling: "plain", "linear", "base" or "turns"."""
    f = torch.empty(max(0, int(rotary_dim)) // 2, dtype=torch.float64)
    _check(load_library().tbe_rotary_frequencies(int(rotary_dim), float(base), ROTARY_SCALING[scaling], float(factor), float(context),
                                                 float(low_turns), float(high_turns), f.data_ptr()), "tbe_rotary_frequencies")
    return f.to(device)


def _new_heads(like: torch.Tensor, shape, stream: Optional[torch.cuda.Stream]) -> Tuple[torch.Tensor, Rows]:
    """A result [rows, heads, head_dim] of like's type, and its rows (without the checks that a given one goes through: they take a quarter of a
    small call)."""
    out = like.new_empty(shape) if stream is None else _empty(shape, like.dtype, like.device, stream)
    return out, Rows(out.data_ptr(), shape[1] * shape[2], shape[2])


class Cache:
    """tbe_cache: keys and values as one byte an element, k and v [rows, heads, head_dim] float8_e4m3fn or int8 (last axis contiguous), and scales,
    k_scales and v_scales float32 [heads, rows]; a value is code * scale.  TBE.alloc_cache makes an empty one."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor):
        if k.dim() != 3 or v.shape != k.shape:
            raise ValueError("k and v must have three axes: rows, heads, head_dim, and one shape")
        if k.dtype not in _CODE or v.dtype != k.dtype:
            raise TypeError(f"k and v must both be float8_e4m3fn or both int8, got {k.dtype} / {v.dtype}")
        if not (k.is_cuda and v.is_cuda):
            raise ValueError("k and v must be device tensors")
        if any(t.stride(2) != 1 and t.shape[2] > 1 and t.numel() for t in (k, v)):
            raise ValueError("the last axis of k and v must be contiguous")
        for t, what in ((k_scales, "k_scales"), (v_scales, "v_scales")):
            _dev_ptr(t, torch.float32, what)
            if t.shape != (k.shape[1], k.shape[0]):
                raise ValueError(f"{what} must be [heads, rows], got {tuple(t.shape)}")
        self.k, self.v, self.k_scales, self.v_scales = k, v, k_scales, v_scales

    def _args(self) -> bytes:
        k, v = self.k, self.v
        rows, heads, dim = k.shape
        ks, vs = k.stride(), v.stride()
        return _PACK_CACHE(rows, heads, dim, _CODE[k.dtype], k.data_ptr(), ks[0], ks[1], v.data_ptr(), vs[0], vs[1], self.k_scales.data_ptr(),
                           self.v_scales.data_ptr())


class TBE:
    """One table set (tbe_handle).  Methods mirror the C entry points one to one."""

    def __init__(self, rows: Sequence[int], D: Sequence[int], weight_dtype: str = "f32"):
        self._lib = load_library()
        self.rows = [int(r) for r in rows]
        self.D = [int(d) for d in D]
        self.T = len(self.rows)
        assert len(self.D) == self.T
        self.weight_dtype = weight_dtype
        self.torch_dtype = {"f32": torch.float32, "f16": torch.float16}[weight_dtype]
        self.sum_D = sum(self.D)
        self.total_rows = sum(self.rows)
        self.total_elems = sum(r * d for r, d in zip(self.rows, self.D))
        rows_a = (ctypes.c_int64 * self.T)(*self.rows)
        D_a = (ctypes.c_int32 * self.T)(*self.D)
        h = ctypes.c_void_p()
        _check(self._lib.tbe_create(self.T, rows_a, D_a, {"f32": F32, "f16": F16}[weight_dtype], ctypes.byref(h)),
               "tbe_create")
        self._h = h

    def close(self) -> None:
        if getattr(self, "_h", None):
            self._lib.tbe_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- tbe_workspace_bytes
    def workspace_bytes(self, B: int, max_nnz: int) -> int:
        n = ctypes.c_size_t()
        _check(self._lib.tbe_workspace_bytes(self._h, int(B), int(max_nnz), ctypes.byref(n)), "tbe_workspace_bytes")
        return int(n.value)

    def alloc_workspace(self, B: int, max_nnz: int, device="cuda") -> torch.Tensor:
        return torch.empty(self.workspace_bytes(B, max_nnz), dtype=torch.uint8, device=device)

    # ---- tbe_forward
    def forward(self, tables: torch.Tensor, indices: torch.Tensor, offsets: torch.Tensor, B: int, pooling: str = "sum",
                out: Optional[torch.Tensor] = None, D_offsets: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        if out is None:
            out = _empty((B, self.sum_D), torch.float32, tables.device, stream)
        if tables.numel() != self.total_elems or out.shape != (B, self.sum_D):
            raise ValueError("tables / out shape does not match the handle")
        if offsets.numel() != self.T * B + 1:
            raise ValueError("offsets must have T*B+1 entries")
        nnz = indices.numel()
        st = self._lib.tbe_forward(self._h, _dev_ptr(tables, self.torch_dtype, "tables"),
                                   _dev_ptr(D_offsets, torch.int32, "D_offsets"),
                                   _dev_ptr(indices, torch.int64, "indices"), _dev_ptr(offsets, torch.int64, "offsets"),
                                   int(B), int(nnz), {"sum": SUM, "mean": MEAN}[pooling],
                                   _dev_ptr(out, torch.float32, "out"), _stream_ptr(stream))
        _check(st, "tbe_forward")
        return out

    # ---- tbe_forward_ex
    def forward_ex(self, tables: torch.Tensor, indices: torch.Tensor, offsets: torch.Tensor, B: int,
                   pooling: str = "sum", out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.float32,
                   D_offsets: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """int64 or int32 indices/offsets (both the same); float32, float16 or bfloat16 out."""
        if out is None:
            out = _empty((B, self.sum_D), out_dtype, tables.device, stream)
        if out.dtype not in _IO:
            raise TypeError(f"out must be float32, float16 or bfloat16, got {out.dtype}")
        if tables.numel() != self.total_elems or out.shape != (B, self.sum_D):
            raise ValueError("tables / out shape does not match the handle")
        if offsets.numel() != self.T * B + 1:
            raise ValueError("offsets must have T*B+1 entries")
        idt = _index_dtype(indices, offsets)
        st = self._lib.tbe_forward_ex(self._h, _dev_ptr(tables, self.torch_dtype, "tables"),
                                      _dev_ptr(D_offsets, torch.int32, "D_offsets"),
                                      _dev_ptr(indices, indices.dtype, "indices"),
                                      _dev_ptr(offsets, offsets.dtype, "offsets"), idt, int(B), int(indices.numel()),
                                      {"sum": SUM, "mean": MEAN}[pooling], _dev_ptr(out, out.dtype, "out"),
                                      _IO[out.dtype], _stream_ptr(stream))
        _check(st, "tbe_forward_ex")
        return out

    # ---- tbe_backward_rowwise_adagrad_ex
    def backward_rowwise_adagrad_ex(self, grad_out: torch.Tensor, indices: torch.Tensor, offsets: torch.Tensor, B: int,
                                    tables: torch.Tensor, state: torch.Tensor, workspace: torch.Tensor, *,
                                    pooling: str = "sum", lr: float, eps: float, momentum_scale: float = 1.0,
                                    stream: Optional[torch.cuda.Stream] = None) -> None:
        """int64 or int32 indices/offsets (both the same); float32, float16 or bfloat16 grad_out."""
        if tables.numel() != self.total_elems or state.numel() != self.total_rows:
            raise ValueError("tables / state shape does not match the handle")
        if grad_out.shape != (B, self.sum_D) or offsets.numel() != self.T * B + 1:
            raise ValueError("grad_out / offsets shape does not match the handle")
        if grad_out.dtype not in _IO:
            raise TypeError(f"grad_out must be float32, float16 or bfloat16, got {grad_out.dtype}")
        idt = _index_dtype(indices, offsets)
        st = self._lib.tbe_backward_rowwise_adagrad_ex(
            self._h, _dev_ptr(grad_out, grad_out.dtype, "grad_out"), _IO[grad_out.dtype],
            _dev_ptr(indices, indices.dtype, "indices"), _dev_ptr(offsets, offsets.dtype, "offsets"), idt, int(B),
            int(indices.numel()), {"sum": SUM, "mean": MEAN}[pooling], float(lr), float(eps), float(momentum_scale),
            _dev_ptr(tables, self.torch_dtype, "tables"), _dev_ptr(state, torch.float32, "state"),
            _dev_ptr(workspace, torch.uint8, "workspace"), int(workspace.numel()), _stream_ptr(stream))
        _check(st, "tbe_backward_rowwise_adagrad_ex")

    # ---- tbe_backward_rowwise_adagrad_static
    def backward_rowwise_adagrad_static(self, grad_out: torch.Tensor, indices: torch.Tensor, offsets: torch.Tensor,
                                        B: int, tables: torch.Tensor, state: torch.Tensor, *, pooling: str = "sum",
                                        lr: float, eps: float, momentum_scale: float = 1.0,
                                        stream: Optional[torch.cuda.Stream] = None) -> None:
        """The backward with the library's own fixed scratch array instead of a caller's workspace."""
        if tables.numel() != self.total_elems or state.numel() != self.total_rows:
            raise ValueError("tables / state shape does not match the handle")
        if grad_out.shape != (B, self.sum_D) or offsets.numel() != self.T * B + 1:
            raise ValueError("grad_out / offsets shape does not match the handle")
        if grad_out.dtype not in _IO:
            raise TypeError(f"grad_out must be float32, float16 or bfloat16, got {grad_out.dtype}")
        idt = _index_dtype(indices, offsets)
        st = self._lib.tbe_backward_rowwise_adagrad_static(
            self._h, _dev_ptr(grad_out, grad_out.dtype, "grad_out"), _IO[grad_out.dtype],
            _dev_ptr(indices, indices.dtype, "indices"), _dev_ptr(offsets, offsets.dtype, "offsets"), idt, int(B),
            int(indices.numel()), {"sum": SUM, "mean": MEAN}[pooling], float(lr), float(eps), float(momentum_scale),
            _dev_ptr(tables, self.torch_dtype, "tables"), _dev_ptr(state, torch.float32, "state"), _stream_ptr(stream))
        _check(st, "tbe_backward_rowwise_adagrad_static")

    # ---- tbe_backward_prepare / tbe_backward_apply_rowwise_adagrad
    def backward_prepare(self, indices: torch.Tensor, offsets: torch.Tensor, B: int, workspace: torch.Tensor,
                         stream: Optional[torch.cuda.Stream] = None) -> None:
        """Sort / dedup / segment the batch's ids into `workspace` (needs no gradient; may run on another stream)."""
        if offsets.numel() != self.T * B + 1:
            raise ValueError("offsets shape does not match the handle")
        idt = _index_dtype(indices, offsets)
        st = self._lib.tbe_backward_prepare(
            self._h, _dev_ptr(indices, indices.dtype, "indices"), _dev_ptr(offsets, offsets.dtype, "offsets"), idt,
            int(B), int(indices.numel()), _dev_ptr(workspace, torch.uint8, "workspace"), int(workspace.numel()),
            _stream_ptr(stream))
        _check(st, "tbe_backward_prepare")

    def backward_apply_rowwise_adagrad(self, grad_out: torch.Tensor, offsets: torch.Tensor, B: int, nnz: int,
                                       tables: torch.Tensor, state: torch.Tensor, workspace: torch.Tensor, *,
                                       pooling: str = "sum", lr: float, eps: float, momentum_scale: float = 1.0,
                                       stream: Optional[torch.cuda.Stream] = None) -> None:
        """Row gradients and the step from a workspace that backward_prepare filled for the same batch."""
        if tables.numel() != self.total_elems or state.numel() != self.total_rows:
            raise ValueError("tables / state shape does not match the handle")
        if grad_out.shape != (B, self.sum_D) or offsets.numel() != self.T * B + 1:
            raise ValueError("grad_out / offsets shape does not match the handle")
        if grad_out.dtype not in _IO:
            raise TypeError(f"grad_out must be float32, float16 or bfloat16, got {grad_out.dtype}")
        if offsets.dtype not in _IDX:
            raise TypeError(f"offsets must be int64 or int32, got {offsets.dtype}")
        st = self._lib.tbe_backward_apply_rowwise_adagrad(
            self._h, _dev_ptr(grad_out, grad_out.dtype, "grad_out"), _IO[grad_out.dtype],
            _dev_ptr(offsets, offsets.dtype, "offsets"), _IDX[offsets.dtype], int(B), int(nnz),
            {"sum": SUM, "mean": MEAN}[pooling], float(lr), float(eps), float(momentum_scale),
            _dev_ptr(tables, self.torch_dtype, "tables"), _dev_ptr(state, torch.float32, "state"),
            _dev_ptr(workspace, torch.uint8, "workspace"), int(workspace.numel()), _stream_ptr(stream))
        _check(st, "tbe_backward_apply_rowwise_adagrad")

    def backward_apply_sgd(self, grad_out: torch.Tensor, offsets: torch.Tensor, B: int, nnz: int, tables: torch.Tensor,
                           workspace: torch.Tensor, *, pooling: str = "sum", lr: float,
                           stream: Optional[torch.cuda.Stream] = None) -> None:
        """Row gradients and the plain SGD step from a workspace that backward_prepare filled for the same batch."""
        if tables.numel() != self.total_elems:
            raise ValueError("tables shape does not match the handle")
        if grad_out.shape != (B, self.sum_D) or offsets.numel() != self.T * B + 1:
            raise ValueError("grad_out / offsets shape does not match the handle")
        if grad_out.dtype not in _IO:
            raise TypeError(f"grad_out must be float32, float16 or bfloat16, got {grad_out.dtype}")
        if offsets.dtype not in _IDX:
            raise TypeError(f"offsets must be int64 or int32, got {offsets.dtype}")
        st = self._lib.tbe_backward_apply_sgd(
            self._h, _dev_ptr(grad_out, grad_out.dtype, "grad_out"), _IO[grad_out.dtype],
            _dev_ptr(offsets, offsets.dtype, "offsets"), _IDX[offsets.dtype], int(B), int(nnz),
            {"sum": SUM, "mean": MEAN}[pooling], float(lr), _dev_ptr(tables, self.torch_dtype, "tables"),
            _dev_ptr(workspace, torch.uint8, "workspace"), int(workspace.numel()), _stream_ptr(stream))
        _check(st, "tbe_backward_apply_sgd")

    # ---- tbe_backward_sgd
    def backward_sgd(self, grad_out: torch.Tensor, indices: torch.Tensor, offsets: torch.Tensor, B: int,
                     tables: torch.Tensor, workspace: torch.Tensor, *, pooling: str = "sum", lr: float,
                     stream: Optional[torch.cuda.Stream] = None) -> None:
        if tables.numel() != self.total_elems:
            raise ValueError("tables shape does not match the handle")
        if grad_out.shape != (B, self.sum_D) or offsets.numel() != self.T * B + 1:
            raise ValueError("grad_out / offsets shape does not match the handle")
        if grad_out.dtype not in _IO:
            raise TypeError(f"grad_out must be float32, float16 or bfloat16, got {grad_out.dtype}")
        idt = _index_dtype(indices, offsets)
        st = self._lib.tbe_backward_sgd(
            self._h, _dev_ptr(grad_out, grad_out.dtype, "grad_out"), _IO[grad_out.dtype],
            _dev_ptr(indices, indices.dtype, "indices"), _dev_ptr(offsets, offsets.dtype, "offsets"), idt, int(B),
            int(indices.numel()), {"sum": SUM, "mean": MEAN}[pooling], float(lr),
            _dev_ptr(tables, self.torch_dtype, "tables"), _dev_ptr(workspace, torch.uint8, "workspace"),
            int(workspace.numel()), _stream_ptr(stream))
        _check(st, "tbe_backward_sgd")

    # ---- tbe_backward_rowwise_adagrad
    def backward_rowwise_adagrad(self, grad_out: torch.Tensor, indices: torch.Tensor, offsets: torch.Tensor, B: int,
                                 tables: torch.Tensor, state: torch.Tensor, workspace: torch.Tensor, *,
                                 pooling: str = "sum", lr: float, eps: float, momentum_scale: float = 1.0,
                                 stream: Optional[torch.cuda.Stream] = None) -> None:
        if tables.numel() != self.total_elems or state.numel() != self.total_rows:
            raise ValueError("tables / state shape does not match the handle")
        if grad_out.shape != (B, self.sum_D) or offsets.numel() != self.T * B + 1:
            raise ValueError("grad_out / offsets shape does not match the handle")
        nnz = indices.numel()
        st = self._lib.tbe_backward_rowwise_adagrad(
            self._h, _dev_ptr(grad_out, torch.float32, "grad_out"), _dev_ptr(indices, torch.int64, "indices"),
            _dev_ptr(offsets, torch.int64, "offsets"), int(B), int(nnz), {"sum": SUM, "mean": MEAN}[pooling],
            float(lr), float(eps), float(momentum_scale), _dev_ptr(tables, self.torch_dtype, "tables"),
            _dev_ptr(state, torch.float32, "state"), _dev_ptr(workspace, torch.uint8, "workspace"),
            int(workspace.numel()), _stream_ptr(stream))
        _check(st, "tbe_backward_rowwise_adagrad")

    # ---- tbe_lookup_seq
    def lookup_seq(self, tables: torch.Tensor, indices: torch.Tensor, offsets: torch.Tensor, out: torch.Tensor,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """offsets: [T+1]; out: flat tensor of >= sum_t n_t * D_t elements (float32, float16 or bfloat16)."""
        if tables.numel() != self.total_elems or offsets.numel() != self.T + 1:
            raise ValueError("tables / offsets shape does not match the handle")
        if out.dtype not in _IO:
            raise TypeError(f"out must be float32, float16 or bfloat16, got {out.dtype}")
        idt = _index_dtype(indices, offsets)
        st = self._lib.tbe_lookup_seq(self._h, _dev_ptr(tables, self.torch_dtype, "tables"),
                                      _dev_ptr(indices, indices.dtype, "indices"),
                                      _dev_ptr(offsets, offsets.dtype, "offsets"), idt, int(indices.numel()),
                                      _dev_ptr(out, out.dtype, "out"), _IO[out.dtype], int(out.numel()),
                                      _stream_ptr(stream))
        _check(st, "tbe_lookup_seq")
        return out

    # ---- tbe_backward_seq_rowwise_adagrad
    def backward_seq_rowwise_adagrad(self, grad_seq: torch.Tensor, indices: torch.Tensor, offsets: torch.Tensor,
                                     tables: torch.Tensor, state: torch.Tensor, workspace: torch.Tensor, *, lr: float,
                                     eps: float, momentum_scale: float = 1.0,
                                     stream: Optional[torch.cuda.Stream] = None) -> None:
        if tables.numel() != self.total_elems or state.numel() != self.total_rows or offsets.numel() != self.T + 1:
            raise ValueError("tables / state / offsets shape does not match the handle")
        if grad_seq.dtype not in _IO:
            raise TypeError(f"grad_seq must be float32, float16 or bfloat16, got {grad_seq.dtype}")
        idt = _index_dtype(indices, offsets)
        st = self._lib.tbe_backward_seq_rowwise_adagrad(
            self._h, _dev_ptr(grad_seq, grad_seq.dtype, "grad_seq"), _IO[grad_seq.dtype], int(grad_seq.numel()),
            _dev_ptr(indices, indices.dtype, "indices"), _dev_ptr(offsets, offsets.dtype, "offsets"), idt,
            int(indices.numel()), float(lr), float(eps), float(momentum_scale),
            _dev_ptr(tables, self.torch_dtype, "tables"), _dev_ptr(state, torch.float32, "state"),
            _dev_ptr(workspace, torch.uint8, "workspace"), int(workspace.numel()), _stream_ptr(stream))
        _check(st, "tbe_backward_seq_rowwise_adagrad")

    # ---- tbe_replica_mean
    def replica_mean(self, replicas: Sequence[torch.Tensor], stream: Optional[torch.cuda.Stream] = None) -> None:
        """Every tensor (one per replica, same shape; float32 or float16) becomes the element-wise mean."""
        first = replicas[0]
        if first.dtype not in (torch.float32, torch.float16):
            raise TypeError(f"replicas must be float32 or float16, got {first.dtype}")
        for r in replicas:
            if r.dtype != first.dtype or r.numel() != first.numel():
                raise ValueError("replicas must agree in dtype and size")
        ptrs = (ctypes.c_void_p * len(replicas))(*[_dev_ptr(r, first.dtype, "replica") for r in replicas])
        st = self._lib.tbe_replica_mean(self._h, ptrs, len(replicas), first.numel(),
                                        F32 if first.dtype == torch.float32 else F16, _stream_ptr(stream))
        _check(st, "tbe_replica_mean")

    # ---- tbe_layer_norm
    def layer_norm(self, x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *,
                   eps: float = 1e-5, out: Optional[torch.Tensor] = None, mean: Optional[torch.Tensor] = None,
                   rstd: Optional[torch.Tensor] = None, stats: bool = True, stream: Optional[torch.cuda.Stream] = None
                   ) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
        """x: [rows, cols] (float32, float16 or bfloat16; rows may be apart); weight, bias: [cols] of one type.  Returns (out, mean,
        rstd); mean and rstd, float32 [rows], are what the backward needs - stats=False leaves out those that are not given."""
        if x.dim() != 2:
            raise ValueError("x must have two axes")
        rows, cols = x.shape
        params = weight if weight is not None else bias
        if weight is not None and bias is not None and weight.dtype != bias.dtype:
            raise TypeError(f"weight and bias must be of one type, got {weight.dtype} / {bias.dtype}")
        out = _empty((rows, cols), x.dtype, x.device, stream) if out is None else out
        if stats and mean is None:
            mean = _empty(rows, torch.float32, x.device, stream)
        if stats and rstd is None:
            rstd = _empty(rows, torch.float32, x.device, stream)
        st = self._lib.tbe_layer_norm(self._h, _rows_ptr(x, None, "x"), x.stride(0), _IO[x.dtype], rows, cols,
                                      _param_ptr(weight, cols, None, "weight"), _param_ptr(bias, cols, None, "bias"),
                                      IO_F32 if params is None else _IO[params.dtype], float(eps), _rows_ptr(out, x, "out"), out.stride(0),
                                      _param_ptr(mean, rows, torch.float32, "mean"), _param_ptr(rstd, rows, torch.float32, "rstd"),
                                      _stream_ptr(stream))
        _check(st, "tbe_layer_norm")
        return out, mean, rstd

    # ---- tbe_layer_norm_workspace_bytes
    def layer_norm_workspace_bytes(self, rows: int, cols: int) -> int:
        n = ctypes.c_size_t()
        _check(self._lib.tbe_layer_norm_workspace_bytes(self._h, int(rows), int(cols), ctypes.byref(n)), "tbe_layer_norm_workspace_bytes")
        return int(n.value)

    def alloc_layer_norm_workspace(self, rows: int, cols: int, device="cuda") -> torch.Tensor:
        return torch.empty(self.layer_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device=device)

    # ---- tbe_layer_norm_backward
    def layer_norm_backward(self, grad_out: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor,
                            rstd: torch.Tensor, workspace: Optional[torch.Tensor], *, grad_x: Optional[torch.Tensor] = None,
                            grad_weight: Optional[torch.Tensor] = None, grad_bias: Optional[torch.Tensor] = None, params: bool = True,
                            param_dtype: Optional[torch.dtype] = None, stream: Optional[torch.cuda.Stream] = None
                            ) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
        """Returns (grad_x, grad_weight, grad_bias); the last two, of the weight's type (param_dtype, or float32, where there is no
        weight), are made unless params=False leaves out those that are not given."""
        if x.dim() != 2:
            raise ValueError("x must have two axes")
        rows, cols = x.shape
        given = [t.dtype for t in (weight, grad_weight, grad_bias) if t is not None]
        pt = given[0] if given else (param_dtype or torch.float32)
        if pt not in _IO or any(t != pt for t in given) or (param_dtype or pt) != pt:
            raise TypeError(f"weight and its gradients must be of one type, got {given}")
        grad_x = _empty((rows, cols), x.dtype, x.device, stream) if grad_x is None else grad_x
        if params and grad_weight is None:
            grad_weight = _empty(cols, pt, x.device, stream)
        if params and grad_bias is None:
            grad_bias = _empty(cols, pt, x.device, stream)
        st = self._lib.tbe_layer_norm_backward(
            self._h, _rows_ptr(grad_out, x, "grad_out"), grad_out.stride(0), _rows_ptr(x, None, "x"), x.stride(0), _IO[x.dtype], rows, cols,
            _param_ptr(weight, cols, None, "weight"), _IO[pt], _param_ptr(mean, rows, torch.float32, "mean"),
            _param_ptr(rstd, rows, torch.float32, "rstd"), _rows_ptr(grad_x, x, "grad_x"), grad_x.stride(0),
            _param_ptr(grad_weight, cols, pt, "grad_weight"), _param_ptr(grad_bias, cols, pt, "grad_bias"),
            _dev_ptr(workspace, torch.uint8, "workspace"), 0 if workspace is None else int(workspace.numel()), _stream_ptr(stream))
        _check(st, "tbe_layer_norm_backward")
        return grad_x, grad_weight, grad_bias

    # ---- tbe_attention_workspace_bytes
    def attention_workspace_bytes(self, sequences: int, q_rows: int, k_rows: int, heads: int, kv_heads: int, head_dim: int, *,
                                  buckets: int = 0, backward: bool = False) -> int:
        """For calls of these sizes, with a bias of `buckets` buckets (0: without), of any element type."""
        dtype = IO_F32 if head_dim % 8 else IO_BF16
        a = AttentionArgs(sequences=int(sequences), heads=int(heads), kv_heads=int(kv_heads), head_dim=int(head_dim), q_rows=int(q_rows),
                          k_rows=int(k_rows), dtype=dtype, buckets=int(buckets))
        n = ctypes.c_size_t()
        _check(self._lib.tbe_attention_workspace_bytes(self._h, ctypes.addressof(a), int(backward), ctypes.byref(n)),
               "tbe_attention_workspace_bytes")
        return int(n.value)

    def alloc_attention_workspace(self, sequences: int, q_rows: int, k_rows: int, heads: int, kv_heads: int, head_dim: int, *,
                                  buckets: int = 0, backward: bool = False, device="cuda") -> torch.Tensor:
        return torch.empty(self.attention_workspace_bytes(sequences, q_rows, k_rows, heads, kv_heads, head_dim, buckets=buckets,
                                                          backward=backward), dtype=torch.uint8, device=device)

    def _attention_args(self, q, k, v, q_offsets, k_offsets, k_lengths, causal, scale, bias, bucket_map) -> bytes:
        """tbe_attention_args"""
        if q.dim() != 3 or k.dim() != 3:
            raise ValueError("q, k and v must have three axes: rows, heads, head_dim")
        if q.dtype not in _IO:
            raise TypeError(f"q must be float32, float16 or bfloat16, got {q.dtype}")
        dtype = q.dtype
        if k.dtype != dtype or v.dtype != dtype or v.shape != k.shape or k.shape[2] != q.shape[2]:
            raise ValueError("q, k and v must agree in type and head_dim, k and v in shape")
        kp, vp = _rows_ptr(k, None, "k"), _rows_ptr(v, None, "v")
        ks, vs = k.stride(), v.stride()
        return self._pack_attention(q, k.shape, (kp, ks[0], ks[1], vp, vs[0], vs[1]), q_offsets, k_offsets, k_lengths, causal, scale, bias, bucket_map)

    def _pack_attention(self, q, k_shape, kv, q_offsets, k_offsets, k_lengths, causal, scale, bias, bucket_map) -> bytes:
        """... from the matrices of k and v as they stand in it"""
        q_rows, heads, dim = q.shape
        k_rows, kv_heads, _ = k_shape
        n = q_offsets.numel() - 1
        if k_offsets.numel() != n + 1 or (k_lengths is not None and k_lengths.numel() != n):
            raise ValueError("q_offsets and k_offsets must have one entry more than k_lengths")
        it = q_offsets.dtype
        table = map_ = 0
        bias_io = buckets = far = 0
        if bias is not None or bucket_map is not None:
            if bias is None or bucket_map is None:
                raise ValueError("bias and bucket_map belong together")
            if bias.dim() != 2 or bias.shape[0] != heads or bucket_map.dim() != 1 or bucket_map.numel() % 2 != 1:
                raise ValueError("bias must be [heads, buckets] and bucket_map [2 * max_distance + 1]")
            table, map_ = _param_ptr(bias, bias.numel(), None, "bias"), _dev_ptr(bucket_map, torch.int32, "bucket_map")
            bias_io, buckets, far = _IO[bias.dtype], bias.shape[1], bucket_map.numel() // 2
        qp, qs = _rows_ptr(q, None, "q"), q.stride()
        return _PACK_ATTENTION(n, heads, kv_heads, dim, q_rows, k_rows, _IO[q.dtype], _index_dtype(q_offsets, k_offsets), qp, qs[0], qs[1], *kv,
                               _dev_ptr(q_offsets, it, "q_offsets"), _dev_ptr(k_offsets, it, "k_offsets"),
                               _dev_ptr(k_lengths, it, "k_lengths") or 0, bool(causal), dim ** -0.5 if scale is None else float(scale), table, map_,
                               bias_io, buckets, far)

    # ---- tbe_attention
    def attention(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_offsets: torch.Tensor, k_offsets: torch.Tensor,
                  workspace: Optional[torch.Tensor], *, causal: bool = True, scale: Optional[float] = None,
                  k_lengths: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, bucket_map: Optional[torch.Tensor] = None,
                  out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, stats: bool = True,
                  stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        """q: [q_rows, heads, head_dim], k and v: [k_rows, kv_heads, head_dim] (float32, float16 or bfloat16; last axis contiguous,
        column blocks of one matrix are fine); offsets: [sequences + 1], k_lengths: [sequences], int64 or int32; scale: head_dim ** -0.5
        unless given; bias: [heads, buckets], bucket_map: int32 [2 * max_distance + 1].  Returns (out, lse), lse float32
        [heads, q_rows]; stats=False: no lse unless it is given."""
        a = self._attention_args(q, k, v, q_offsets, k_offsets, k_lengths, causal, scale, bias, bucket_map)
        out = _empty(q.shape, q.dtype, q.device, stream) if out is None else out
        if stats and lse is None:
            lse = _empty((q.shape[1], q.shape[0]), torch.float32, q.device, stream)
        st = self._lib.tbe_attention(self._h, a, _heads(out, q, "out"),
                                     _param_ptr(lse, q.shape[0] * q.shape[1], torch.float32, "lse"),
                                     _dev_ptr(workspace, torch.uint8, "workspace"), 0 if workspace is None else int(workspace.numel()),
                                     _stream_ptr(stream))
        _check(st, "tbe_attention")
        return out, lse

    # ---- tbe_attention_backward
    def attention_backward(self, grad_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                           lse: torch.Tensor, q_offsets: torch.Tensor, k_offsets: torch.Tensor, workspace: torch.Tensor, *,
                           causal: bool = True, scale: Optional[float] = None, k_lengths: Optional[torch.Tensor] = None,
                           bias: Optional[torch.Tensor] = None, bucket_map: Optional[torch.Tensor] = None,
                           grad_q: Optional[torch.Tensor] = None, grad_k: Optional[torch.Tensor] = None,
                           grad_v: Optional[torch.Tensor] = None, grad_bias: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None
                           ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
        """Arguments as of attention(), its out and lse, and the upstream gradient.  Returns (grad_q, grad_k, grad_v, grad_bias)."""
        a = self._attention_args(q, k, v, q_offsets, k_offsets, k_lengths, causal, scale, bias, bucket_map)
        grad_q = _empty(q.shape, q.dtype, q.device, stream) if grad_q is None else grad_q
        grad_k = _empty(k.shape, q.dtype, q.device, stream) if grad_k is None else grad_k
        grad_v = _empty(v.shape, q.dtype, q.device, stream) if grad_v is None else grad_v
        if bias is None and grad_bias is not None:
            raise ValueError("grad_bias without bias")
        if bias is not None and grad_bias is None:
            grad_bias = _empty(bias.shape, bias.dtype, bias.device, stream)
        st = self._lib.tbe_attention_backward(
            self._h, a, _heads(out, q, "out"), _param_ptr(lse, q.shape[0] * q.shape[1], torch.float32, "lse"),
            _heads(grad_out, q, "grad_out"), _heads(grad_q, q, "grad_q"), _heads(grad_k, k, "grad_k"), _heads(grad_v, v, "grad_v"),
            None if bias is None else _param_ptr(grad_bias, bias.numel(), bias.dtype, "grad_bias"),
            _dev_ptr(workspace, torch.uint8, "workspace"), 0 if workspace is None else int(workspace.numel()), _stream_ptr(stream))
        _check(st, "tbe_attention_backward")
        return grad_q, grad_k, grad_v, grad_bias

    # ---- tbe_rotate_heads
    def _rotation_args(self, q, k, like, positions, frequencies, interleaved, amplitude, norm, eps, q_weight, k_weight, weight_dtype) -> bytes:
        """tbe_rotation_args; q and k (or their gradients) of like's type"""
        rows, dim = like.shape[0], like.shape[2]
        if q is not None and k is not None and (k.dim() != 3 or k.dtype != q.dtype or k.shape[0] != rows or k.shape[2] != dim):
            raise ValueError("q and k must agree in type, rows and head_dim")
        if positions.dtype not in _IDX:
            raise TypeError(f"positions must be int64 or int32, got {positions.dtype}")
        if positions.numel() != rows:
            raise ValueError(f"positions must have {rows} entries, got {positions.numel()}")
        turned = 0 if frequencies is None else 2 * frequencies.numel()
        if not norm and (q_weight is not None or k_weight is not None):
            raise ValueError("weights without norm")
        if q_weight is not None and k_weight is not None and q_weight.dtype != k_weight.dtype:
            raise TypeError(f"q_weight and k_weight must be of one type, got {q_weight.dtype} / {k_weight.dtype}")
        return _PACK_ROTATION(0 if q is None else q.shape[1], 0 if k is None else k.shape[1], dim, turned, rows, _IO[like.dtype], _IDX[positions.dtype],
                              _dev_ptr(positions, positions.dtype, "positions"), _dev_ptr(frequencies, torch.float64, "frequencies") or 0,
                              bool(interleaved), float(amplitude), bool(norm), float(eps), _param_ptr(q_weight, dim, None, "q_weight") or 0,
                              _param_ptr(k_weight, dim, None, "k_weight") or 0, _IO[weight_dtype])

    @staticmethod
    def _heads_or_none(t: Optional[torch.Tensor], like: Optional[torch.Tensor], what: str) -> Rows:
        return Rows() if t is None else _heads(t, like, what)

    def rotate_heads(self, q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: torch.Tensor, frequencies: Optional[torch.Tensor], *,
                     interleaved: bool = False, amplitude: float = 1.0, norm: bool = False, eps: float = 1e-6,
                     q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                     k_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                     ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
        """q: [rows, q_heads, head_dim], k: [rows, k_heads, head_dim] (float32, float16 or bfloat16; last axis contiguous, column blocks of one
        matrix are fine; one of them may be None); positions: [rows], int64 or int32; frequencies: float64 [rotary_dim / 2] (see
        rotary_frequencies), None: no rotation; weights: [head_dim].  Returns (q_out, k_out); they may be q and k."""
        like = q if q is not None else k
        if like is None or like.dim() != 3:
            raise ValueError("q and k must have three axes: rows, heads, head_dim; one of them may be None")
        qp, kp = self._heads_or_none(q, None, "q"), self._heads_or_none(k, None, "k")
        weight = q_weight if q_weight is not None else k_weight
        a = self._rotation_args(q, k, like, positions, frequencies, interleaved, amplitude, norm, eps, q_weight, k_weight,
                                torch.float32 if weight is None else weight.dtype)
        if (q is None and q_out is not None) or (k is None and k_out is not None):
            raise ValueError("q_out without q, or k_out without k")
        q_out, qo = _new_heads(q, q.shape, stream) if q is not None and q_out is None else (q_out, self._heads_or_none(q_out, q, "q_out"))
        k_out, ko = _new_heads(k, k.shape, stream) if k is not None and k_out is None else (k_out, self._heads_or_none(k_out, k, "k_out"))
        st = self._lib.tbe_rotate_heads(self._h, a, qp, kp, qo, ko, _stream_ptr(stream))
        _check(st, "tbe_rotate_heads")
        return q_out, k_out

    # ---- tbe_rotate_workspace_bytes
    def rotate_workspace_bytes(self, rows: int, q_heads: int, k_heads: int, head_dim: int) -> int:
        """For rotate_heads_backward with norm, of any element type."""
        a = RotationArgs(q_heads=int(q_heads), k_heads=int(k_heads), head_dim=int(head_dim), rows=int(rows))
        n = ctypes.c_size_t()
        _check(self._lib.tbe_rotate_workspace_bytes(self._h, ctypes.addressof(a), ctypes.byref(n)), "tbe_rotate_workspace_bytes")
        return int(n.value)

    def alloc_rotate_workspace(self, rows: int, q_heads: int, k_heads: int, head_dim: int, device="cuda") -> torch.Tensor:
        return torch.empty(self.rotate_workspace_bytes(rows, q_heads, k_heads, head_dim), dtype=torch.uint8, device=device)

    # ---- tbe_rotate_heads_backward
    def rotate_heads_backward(self, grad_q_out: Optional[torch.Tensor], grad_k_out: Optional[torch.Tensor], positions: torch.Tensor,
                              frequencies: Optional[torch.Tensor], workspace: Optional[torch.Tensor] = None, *, q: Optional[torch.Tensor] = None,
                              k: Optional[torch.Tensor] = None, interleaved: bool = False, amplitude: float = 1.0, norm: bool = False,
                              eps: float = 1e-6, q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                              grad_q: Optional[torch.Tensor] = None, grad_k: Optional[torch.Tensor] = None,
                              grad_q_weight: Optional[torch.Tensor] = None, grad_k_weight: Optional[torch.Tensor] = None, params: bool = True,
                              param_dtype: Optional[torch.dtype] = None, stream: Optional[torch.cuda.Stream] = None
                              ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor], Optional[torch.Tensor], Optional[torch.Tensor]]:
        """From the upstream gradients, and with norm the q and k that rotate_heads was given.  Returns (grad_q, grad_k, grad_q_weight, grad_k_weight);
        the last two, of the weights' type (param_dtype, or float32, where there is no weight), are made with norm, unless params=False leaves out
        those that are not given."""
        like = grad_q_out if grad_q_out is not None else grad_k_out
        if like is None or like.dim() != 3:
            raise ValueError("grad_q_out and grad_k_out must have three axes: rows, heads, head_dim; one of them may be None")
        dim = like.shape[2]
        given = [t.dtype for t in (q_weight, k_weight, grad_q_weight, grad_k_weight) if t is not None]
        pt = given[0] if given else (param_dtype or torch.float32)
        if pt not in _IO or any(t != pt for t in given) or (param_dtype or pt) != pt:
            raise TypeError(f"weights and their gradients must be of one type, got {given}")
        dqo, dko = self._heads_or_none(grad_q_out, None, "grad_q_out"), self._heads_or_none(grad_k_out, None, "grad_k_out")
        a = self._rotation_args(grad_q_out, grad_k_out, like, positions, frequencies, interleaved, amplitude, norm, eps, q_weight, k_weight, pt)
        for up, x, g, gw, name in ((grad_q_out, q, grad_q, grad_q_weight, "q"), (grad_k_out, k, grad_k, grad_k_weight, "k")):
            if up is None and any(t is not None for t in (x, g, gw)):
                raise ValueError(f"{name} or its gradients without grad_{name}_out")
            if norm and up is not None and x is None:
                raise ValueError(f"{name} is needed with norm")
            if not norm and gw is not None:
                raise ValueError("weights' gradients without norm")
        if grad_q is None and grad_q_out is not None:
            grad_q, gq = _new_heads(like, grad_q_out.shape, stream)
        else:
            gq = self._heads_or_none(grad_q, grad_q_out, "grad_q")
        if grad_k is None and grad_k_out is not None:
            grad_k, gk = _new_heads(like, grad_k_out.shape, stream)
        else:
            gk = self._heads_or_none(grad_k, grad_k_out, "grad_k")
        if norm and params and grad_q_weight is None and grad_q_out is not None:
            grad_q_weight = _empty(dim, pt, like.device, stream)
        if norm and params and grad_k_weight is None and grad_k_out is not None:
            grad_k_weight = _empty(dim, pt, like.device, stream)
        st = self._lib.tbe_rotate_heads_backward(
            self._h, a, dqo, dko, self._heads_or_none(q if norm else None, grad_q_out, "q"), self._heads_or_none(k if norm else None, grad_k_out, "k"),
            gq, gk,
            _param_ptr(grad_q_weight, dim, pt, "grad_q_weight"), _param_ptr(grad_k_weight, dim, pt, "grad_k_weight"),
            _dev_ptr(workspace, torch.uint8, "workspace"), 0 if workspace is None else int(workspace.numel()), _stream_ptr(stream))
        _check(st, "tbe_rotate_heads_backward")
        return grad_q, grad_k, grad_q_weight, grad_k_weight

    # ---- tbe_cache_write
    def alloc_cache(self, rows: int, heads: int, head_dim: int, code: torch.dtype = torch.float8_e4m3fn, device="cuda") -> Cache:
        """A cache of zeros; code: torch.float8_e4m3fn or torch.int8."""
        if code not in _CODE:
            raise TypeError(f"code must be float8_e4m3fn or int8, got {code}")
        k, v = (torch.zeros(rows, heads, head_dim, dtype=torch.uint8, device=device).view(code) for _ in range(2))
        return Cache(k, v, torch.ones(heads, rows, device=device), torch.ones(heads, rows, device=device))

    @staticmethod
    def _cache_rows(cache: Cache, slots: torch.Tensor) -> int:
        if slots.dtype not in _IDX:
            raise TypeError(f"slots must be int64 or int32, got {slots.dtype}")
        return slots.numel()

    def cache_write(self, cache: Cache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, *,
                    stream: Optional[torch.cuda.Stream] = None) -> None:
        """Row r of k and v ([rows, heads, head_dim], float32, float16 or bfloat16; column blocks of one matrix are fine) goes to the cache's row
        slots[r] (int64 or int32; below 0: nowhere; no two alike otherwise, or that row's contents are not specified)."""
        rows = self._cache_rows(cache, slots)
        if k.dim() != 3 or k.shape != (rows, *cache.k.shape[1:]):
            raise ValueError(f"k must be {(rows, *cache.k.shape[1:])}, got {tuple(k.shape)}")
        st = self._lib.tbe_cache_write(self._h, cache._args(), _heads(k, None, "k"), _heads(v, k, "v"), _IO[k.dtype],
                                       _dev_ptr(slots, slots.dtype, "slots"), _IDX[slots.dtype], rows, _stream_ptr(stream))
        _check(st, "tbe_cache_write")

    # ---- tbe_cache_read
    def cache_read(self, cache: Cache, slots: torch.Tensor, *, dtype: torch.dtype = torch.float32, k_out: Optional[torch.Tensor] = None,
                   v_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """The values of the cache's rows `slots` (zeros where one is below 0), [rows, heads, head_dim] of dtype, or into k_out and v_out."""
        rows = self._cache_rows(cache, slots)
        shape = (rows, *cache.k.shape[1:])
        given = k_out if k_out is not None else v_out
        dtype = dtype if given is None else given.dtype
        k_out = _empty(shape, dtype, cache.k.device, stream) if k_out is None else k_out
        v_out = _empty(shape, dtype, cache.k.device, stream) if v_out is None else v_out
        if k_out.shape != shape:
            raise ValueError(f"k_out must be {shape}, got {tuple(k_out.shape)}")
        st = self._lib.tbe_cache_read(self._h, cache._args(), _dev_ptr(slots, slots.dtype, "slots"), _IDX[slots.dtype], rows,
                                      _heads(k_out, None, "k_out"), _heads(v_out, k_out, "v_out"), _IO[k_out.dtype], _stream_ptr(stream))
        _check(st, "tbe_cache_read")
        return k_out, v_out

    # ---- tbe_cache_attention_workspace_bytes
    def cache_attention_workspace_bytes(self, sequences: int, q_rows: int, k_rows: int, heads: int, kv_heads: int, head_dim: int, *, buckets: int = 0) -> int:
        """For calls of these sizes, with a bias of `buckets` buckets (0: without), of any element type."""
        a = AttentionArgs(sequences=int(sequences), heads=int(heads), kv_heads=int(kv_heads), head_dim=int(head_dim), q_rows=int(q_rows),
                          k_rows=int(k_rows), dtype=IO_BF16, buckets=int(buckets))
        n = ctypes.c_size_t()
        _check(self._lib.tbe_cache_attention_workspace_bytes(self._h, ctypes.addressof(a), ctypes.byref(n)), "tbe_cache_attention_workspace_bytes")
        return int(n.value)

    def alloc_cache_attention_workspace(self, sequences: int, q_rows: int, k_rows: int, heads: int, kv_heads: int, head_dim: int, *, buckets: int = 0,
                                        device="cuda") -> torch.Tensor:
        return torch.empty(self.cache_attention_workspace_bytes(sequences, q_rows, k_rows, heads, kv_heads, head_dim, buckets=buckets), dtype=torch.uint8,
                           device=device)

    # ---- tbe_cache_attention
    def cache_attention(self, q: torch.Tensor, cache: Cache, q_offsets: torch.Tensor, k_offsets: torch.Tensor, workspace: Optional[torch.Tensor], *,
                        causal: bool = True, scale: Optional[float] = None, k_lengths: Optional[torch.Tensor] = None,
                        bias: Optional[torch.Tensor] = None, bucket_map: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                        lse: Optional[torch.Tensor] = None, stats: bool = True, stream: Optional[torch.cuda.Stream] = None
                        ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        """attention() with the cache's values as k and v; k_offsets are places in the cache.  Returns (out, lse)."""
        if q.dim() != 3 or q.dtype not in _IO:
            raise ValueError(f"q must be float32, float16 or bfloat16 and have three axes: rows, heads, head_dim; got {q.dtype} {tuple(q.shape)}")
        shape = cache.k.shape
        if shape[2] != q.shape[2]:
            raise ValueError(f"q and the cache must agree in head_dim, got {q.shape[2]} / {shape[2]}")
        a = self._pack_attention(q, shape, (0, 0, 0, 0, 0, 0), q_offsets, k_offsets, k_lengths, causal, scale, bias, bucket_map)
        out, rows = _new_heads(q, q.shape, stream) if out is None else (out, _heads(out, q, "out"))
        if stats and lse is None:
            lse = _empty((q.shape[1], q.shape[0]), torch.float32, q.device, stream)
        st = self._lib.tbe_cache_attention(self._h, a, cache._args(), rows,
                                           _param_ptr(lse, q.shape[0] * q.shape[1], torch.float32, "lse"),
                                           _dev_ptr(workspace, torch.uint8, "workspace"), 0 if workspace is None else int(workspace.numel()),
                                           _stream_ptr(stream))
        _check(st, "tbe_cache_attention")
        return out, lse

    # ---- tbe_debug_sorted
    def debug_sorted(self, workspace: torch.Tensor, B: int, nnz: int) -> Dict[str, torch.Tensor]:
        """Copies the integer by-products of the last backward to host tensors (int64; synchronises)."""
        ptrs = [ctypes.c_void_p() for _ in range(5)]
        _check(self._lib.tbe_debug_sorted(self._h, workspace.data_ptr(), int(B), int(nnz),
                                          *[ctypes.byref(p) for p in ptrs]), "tbe_debug_sorted")
        base = workspace.data_ptr()
        torch.cuda.synchronize()

        def view(p: ctypes.c_void_p, n: int) -> torch.Tensor:
            off = p.value - base
            return workspace[off:off + 4 * n].view(torch.int32).cpu().to(torch.int64) & 0xFFFFFFFF

        U = int(view(ptrs[4], 1).item())
        return {"keys_sorted": view(ptrs[0], nnz), "vals_sorted": view(ptrs[1], nnz),
                "unique_rows": view(ptrs[2], U), "seg_start": view(ptrs[3], U + 1), "num_unique": U}

    def debug_sorted_device(self, workspace: torch.Tensor, B: int, nnz: int) -> Dict[str, torch.Tensor]:
        """Same by-products as device tensors (int64 copies), for checks that stay on the GPU at full size."""
        ptrs = [ctypes.c_void_p() for _ in range(5)]
        _check(self._lib.tbe_debug_sorted(self._h, workspace.data_ptr(), int(B), int(nnz),
                                          *[ctypes.byref(p) for p in ptrs]), "tbe_debug_sorted")
        base = workspace.data_ptr()

        def view(p: ctypes.c_void_p, n: int) -> torch.Tensor:
            off = p.value - base
            return workspace[off:off + 4 * n].view(torch.int32).to(torch.int64) & 0xFFFFFFFF

        U = int(view(ptrs[4], 1).item())
        return {"keys_sorted": view(ptrs[0], nnz), "vals_sorted": view(ptrs[1], nnz),
                "unique_rows": view(ptrs[2], U), "seg_start": view(ptrs[3], U + 1), "num_unique": U}

    # ---- tbe_debug_hot_rows
    def debug_hot_rows(self, workspace: torch.Tensor, B: int, nnz: int) -> Tuple[List[List[int]], List[List[int]]]:
        """Per table the hinted and the dense rows (table-local ids) of the last pooled backward or prepare call (synchronises)."""
        ptrs = [ctypes.c_void_p() for _ in range(5)]
        _check(self._lib.tbe_debug_hot_rows(self._h, workspace.data_ptr(), int(B), int(nnz),
                                            *[ctypes.byref(p) for p in ptrs]), "tbe_debug_hot_rows")
        base = workspace.data_ptr()
        torch.cuda.synchronize()

        def view(p: ctypes.c_void_p, n: int) -> torch.Tensor:
            off = p.value - base
            return workspace[off:off + 4 * n].view(torch.int32).cpu().to(torch.int64) & 0xFFFFFFFF

        hot, dense, row_base = [], [], 0
        hot_n, dense_n = [view(p, self.T).tolist() if p.value else [0] * self.T for p in (ptrs[1], ptrs[3])]
        for t in range(self.T):
            hot.append(view(ptrs[0], 256 * self.T)[256 * t:256 * t + hot_n[t]].tolist() if hot_n[t] else [])
            at = view(ptrs[2], 128 * self.T)[128 * t:128 * t + dense_n[t]] if dense_n[t] else torch.zeros(0, dtype=torch.int64)
            rows = view(ptrs[4], 2 * (int(at.max()) + 1)).view(-1, 2) if dense_n[t] else None
            dense.append((rows[at, 1] - row_base).tolist() if dense_n[t] else [])
            row_base += self.rows[t]
        return hot, dense

    # ---- tbe_debug_forward_kernels
    def debug_forward_kernels(self, B: int, nnz: int) -> int:
        """FWD_* bits: the kernels that a forward of B samples and nnz ids launches."""
        m = ctypes.c_uint32()
        _check(self._lib.tbe_debug_forward_kernels(self._h, int(B), int(nnz), ctypes.byref(m)), "tbe_debug_forward_kernels")
        return int(m.value)

    # ---- tbe_poll_index_error
    def poll_index_error(self) -> bool:
        st = self._lib.tbe_poll_index_error(self._h)
        if st == EINDEX:
            return True
        _check(st, "tbe_poll_index_error")
        return False

    # ---- tbe_calibration_copy
    def calibration_copy(self, dst: torch.Tensor, src: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
        nbytes = src.numel() * src.element_size()
        if dst.numel() * dst.element_size() != nbytes or not (dst.is_cuda and src.is_cuda):
            raise ValueError("dst and src must be device tensors of the same byte size")
        _check(self._lib.tbe_calibration_copy(self._h, dst.data_ptr(), src.data_ptr(), nbytes, _stream_ptr(stream)),
               "tbe_calibration_copy")

    # ---- tbe_calibration_gather
    def calibration_gather(self, buf: torch.Tensor, window_bytes: int, slice_bytes: int, gathers: int, *,
                           per_xcd: bool = True, write_back: bool = False, sink: torch.Tensor,
                           stream: Optional[torch.cuda.Stream] = None) -> None:
        if not (buf.is_cuda and sink.is_cuda):
            raise ValueError("buf and sink must be device tensors")
        _check(self._lib.tbe_calibration_gather(self._h, buf.data_ptr(), buf.numel() * buf.element_size(),
                                                int(window_bytes), 1 if per_xcd else 0, int(slice_bytes), int(gathers),
                                                1 if write_back else 0, sink.data_ptr(),
                                                sink.numel() * sink.element_size(), _stream_ptr(stream)),
               "tbe_calibration_gather")

    # ---- tbe_set_tunable
    def set_tunable(self, which: str, value: int) -> None:
        _check(self._lib.tbe_set_tunable(self._h, TUNABLES[which], int(value)), "tbe_set_tunable")

    # ---- tbe_timing_*
    def timing_enable(self, on: bool = True) -> None:
        _check(self._lib.tbe_timing_enable(self._h, 1 if on else 0), "tbe_timing_enable")

    def timing_read(self) -> List[Tuple[str, float]]:
        n = ctypes.c_int32()
        _check(self._lib.tbe_timing_count(self._h, ctypes.byref(n)), "tbe_timing_count")
        out = []
        for i in range(n.value):
            name = ctypes.c_char_p()
            ms = ctypes.c_float()
            _check(self._lib.tbe_timing_read(self._h, i, ctypes.byref(name), ctypes.byref(ms)), "tbe_timing_read")
            out.append((name.value.decode(), float(ms.value)))
        return out
