"""ctypes binding of libsasq_b200.so.  Same names as include/sasq.h.

Every function takes torch CUDA tensors (used purely as device memory), checks
dtype / device / contiguity, and passes raw pointers and sizes to the library on
the current torch stream.  A non-zero status raises SasqError.  If the shared
library is missing or cannot be loaded, import of this module's functions fails
loudly: there is no CPU or PyTorch fallback.
"""
from __future__ import annotations

import ctypes
import os

import torch

__all__ = [
    "SasqError", "SASQ_F16", "SASQ_BF16", "library_path", "load_library", "sasq_status_string",
    "sasq_fakequant_fwd", "sasq_fakequant_bwd_workspace", "sasq_fakequant_bwd", "sasq_fakequant_fwd_bwd",
    "sasq_fakequant_multi_workspace", "sasq_fakequant_fwd_bwd_multi", "sasq_static_w8a8_linear_workspace",
    "sasq_static_w8a8_linear", "sasq_device_status", "QDesc", "sasq_absmax_scale_workspace", "sasq_absmax_scale",
    "sasq_quantize_weight", "sasq_fakequant_fwd_bwd_static", "sasq_static_w8a8_linear_tiles",
    "sasq_fakequant_per_channel_workspace", "sasq_fakequant_fwd_bwd_per_channel",
    "sasq_fakequant_fwd_bwd_ablation", "sasq_adamw_scales", "SASQ_FULL_OPERATOR", "SASQ_WITHOUT_ROUND",
    "SASQ_WITHOUT_CLAMP", "sasq_dynamic_w8a8_linear_workspace", "sasq_dynamic_w8a8_linear", "sasq_debug_set_wait_limit", "PcDesc", "sasq_fakequant_per_channel_multi_workspace",
    "sasq_fakequant_fwd_bwd_per_channel_multi", "sasq_static_w8a8_linear_per_channel_workspace",
    "sasq_static_w8a8_linear_per_channel", "sasq_static_w8a8_linear_grouped_workspace",
    "sasq_static_w8a8_linear_grouped", "sasq_fakequant_linear_fp_weights_workspace",
    "sasq_fakequant_linear_fp_weights", "sasq_absmax_scale_per_channel", "sasq_running_mean", "LinearDesc", "sasq_static_w8a8_linear_multi_workspace",
    "sasq_static_w8a8_linear_multi", "sasq_static_w8a8_linear_multi_launches", "sasq_set_gang_launch",
    "sasq_debug_int8_issue_rate", "LinearProblems", "QuantTensors",
    "SASQ_KV_16BIT", "SASQ_KV_INT8", "SASQ_KV_INT4", "KVCacheStruct", "KVBatchStruct", "KVCache", "PagedBatch", "sasq_rope_kv_append",
    "sasq_paged_attention_workspace", "sasq_paged_attention", "sasq_w4_linear", "sasq_quantize_weight_w4",
]

SASQ_F16 = 0
SASQ_BF16 = 1
SASQ_FULL_OPERATOR = 0
SASQ_WITHOUT_ROUND = 1
SASQ_WITHOUT_CLAMP = 2
SASQ_KV_16BIT = 0
SASQ_KV_INT8 = 1
SASQ_KV_INT4 = 2


_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libsasq_b200.so")
_lib = None


class SasqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__(f"{where}: {sasq_status_string(status)} (status {status})")


class QDesc(ctypes.Structure):
    """Mirror of sasq_qdesc_t."""
    _fields_ = [("x", ctypes.c_void_p), ("grad_y", ctypes.c_void_p), ("y", ctypes.c_void_p),
                ("grad_x", ctypes.c_void_p), ("numel", ctypes.c_int64), ("scale_index", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class PcDesc(ctypes.Structure):
    """Mirror of sasq_pcdesc_t."""
    _fields_ = [("x", ctypes.c_void_p), ("grad_y", ctypes.c_void_p), ("y", ctypes.c_void_p),
                ("grad_x", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("grad_scales", ctypes.c_void_p),
                ("T", ctypes.c_int64), ("K", ctypes.c_int64), ("reserved", ctypes.c_int64)]


class LinearDesc(ctypes.Structure):
    """Mirror of sasq_linear_desc_t."""
    _fields_ = [("x", ctypes.c_void_p), ("w", ctypes.c_void_p), ("w_scale", ctypes.c_void_p),
                ("x_scale", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("y", ctypes.c_void_p),
                ("T", ctypes.c_int64), ("N", ctypes.c_int64), ("K", ctypes.c_int64)]


class KVCacheStruct(ctypes.Structure):
    """Mirror of sasq_kv_cache_t."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("num_pages", ctypes.c_int64), ("page_size", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("kind", ctypes.c_int32)]


class KVBatchStruct(ctypes.Structure):
    """Mirror of sasq_kv_batch_t."""
    _fields_ = [("page_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p), ("q_starts", ctypes.c_void_p),
                ("page_table_stride", ctypes.c_int64), ("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("total_q", ctypes.c_int32), ("max_q_len", ctypes.c_int32), ("max_seq_len", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Loads the CUDA library; raises if it has not been built (python -m paper_2512_14481_b200.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2512_14481_b200.build` "
                           "(there is no fallback path)")
    L = ctypes.CDLL(_LIB_PATH)
    vp, i64, i32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
    L.sasq_status_string.restype = ctypes.c_char_p
    L.sasq_status_string.argtypes = [i32]
    L.sasq_fakequant_fwd.restype = i32
    L.sasq_fakequant_fwd.argtypes = [vp, vp, i64, i32, vp, i32, vp]
    L.sasq_fakequant_bwd_workspace.restype = sz
    L.sasq_fakequant_bwd_workspace.argtypes = [i64]
    L.sasq_fakequant_bwd.restype = i32
    L.sasq_fakequant_bwd.argtypes = [vp, vp, vp, vp, i32, i64, i32, vp, i32, vp, sz, vp]
    L.sasq_fakequant_fwd_bwd.restype = i32
    L.sasq_fakequant_fwd_bwd.argtypes = [vp, vp, vp, vp, vp, i32, i64, i32, vp, i32, vp, sz, vp]
    L.sasq_fakequant_fwd_bwd_static.restype = i32
    L.sasq_fakequant_fwd_bwd_static.argtypes = [vp, vp, vp, vp, vp, i32, i64, i32, vp, i32, vp]
    L.sasq_fakequant_multi_workspace.restype = sz
    L.sasq_fakequant_multi_workspace.argtypes = [i32]
    L.sasq_fakequant_fwd_bwd_multi.restype = i32
    L.sasq_fakequant_fwd_bwd_multi.argtypes = [ctypes.POINTER(QDesc), i32, vp, vp, i32, i32, i32, i32, vp, sz, vp]
    L.sasq_static_w8a8_linear_workspace.restype = sz
    L.sasq_static_w8a8_linear_workspace.argtypes = [i64, i64, i64]
    L.sasq_static_w8a8_linear.restype = i32
    L.sasq_static_w8a8_linear.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, i32, vp, sz, vp]
    L.sasq_fakequant_fwd_bwd_ablation.restype = i32
    L.sasq_fakequant_fwd_bwd_ablation.argtypes = [vp, vp, vp, vp, vp, i32, i64, i32, vp, i32, i32, vp, sz, vp]
    f32 = ctypes.c_float
    L.sasq_adamw_scales.restype = i32
    L.sasq_adamw_scales.argtypes = [vp, vp, vp, vp, i32, i32, f32, f32, f32, f32, f32, vp]
    L.sasq_fakequant_per_channel_workspace.restype = sz
    L.sasq_fakequant_per_channel_workspace.argtypes = [i64, i64]
    L.sasq_fakequant_fwd_bwd_per_channel.restype = i32
    L.sasq_fakequant_fwd_bwd_per_channel.argtypes = [vp, vp, vp, vp, vp, i32, i64, i64, i32, vp, i32, vp, sz, vp]
    L.sasq_static_w8a8_linear_per_channel_workspace.restype = sz
    L.sasq_static_w8a8_linear_per_channel_workspace.argtypes = [i64, i64, i64]
    L.sasq_static_w8a8_linear_per_channel.restype = i32
    L.sasq_static_w8a8_linear_per_channel.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, i32, vp, sz, vp]
    L.sasq_w4_linear.restype = i32
    L.sasq_w4_linear.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i64, i32, vp]
    L.sasq_quantize_weight_w4.restype = i32
    L.sasq_quantize_weight_w4.argtypes = [vp, vp, vp, i64, i64, i64, i32, vp]
    L.sasq_dynamic_w8a8_linear_workspace.restype = sz
    L.sasq_dynamic_w8a8_linear_workspace.argtypes = [i64, i64, i64]
    L.sasq_dynamic_w8a8_linear.restype = i32
    L.sasq_dynamic_w8a8_linear.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, i32, vp, sz, vp]
    L.sasq_fakequant_per_channel_multi_workspace.restype = sz
    L.sasq_fakequant_per_channel_multi_workspace.argtypes = [i64]
    L.sasq_fakequant_fwd_bwd_per_channel_multi.restype = i32
    L.sasq_fakequant_fwd_bwd_per_channel_multi.argtypes = [ctypes.POINTER(PcDesc), i32, i32, i32, i32, vp, sz, vp]
    L.sasq_debug_set_wait_limit.restype = ctypes.c_longlong
    L.sasq_debug_set_wait_limit.argtypes = [ctypes.c_longlong]
    L.sasq_fakequant_linear_fp_weights_workspace.restype = sz
    L.sasq_fakequant_linear_fp_weights_workspace.argtypes = [i64, i64, i64]
    L.sasq_fakequant_linear_fp_weights.restype = i32
    L.sasq_fakequant_linear_fp_weights.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i32, i32, vp, sz, vp]
    L.sasq_static_w8a8_linear_grouped_workspace.restype = sz
    L.sasq_static_w8a8_linear_grouped_workspace.argtypes = [i64, i64, i64]
    L.sasq_static_w8a8_linear_grouped.restype = i32
    L.sasq_static_w8a8_linear_grouped.argtypes = [vp, vp, vp, vp, i64, vp, vp, i64, i64, i64, i32, i32, vp, sz, vp]
    L.sasq_static_w8a8_linear_multi_workspace.restype = sz
    L.sasq_static_w8a8_linear_multi_workspace.argtypes = [i32, ctypes.POINTER(LinearDesc)]
    L.sasq_static_w8a8_linear_multi.restype = i32
    L.sasq_static_w8a8_linear_multi.argtypes = [i32, ctypes.POINTER(LinearDesc), i32, i32, vp, sz, vp]
    L.sasq_static_w8a8_linear_multi_launches.restype = i32
    L.sasq_static_w8a8_linear_multi_launches.argtypes = [i32, ctypes.POINTER(LinearDesc), i32]
    L.sasq_static_w8a8_linear_tiles.restype = i32
    L.sasq_static_w8a8_linear_tiles.argtypes = [i64, i64, i32, i32, ctypes.POINTER(ctypes.c_int32), i32]
    L.sasq_device_status.restype = i32
    L.sasq_device_status.argtypes = [vp]
    L.sasq_absmax_scale_workspace.restype = sz
    L.sasq_absmax_scale_workspace.argtypes = [i64]
    L.sasq_absmax_scale.restype = i32
    L.sasq_absmax_scale.argtypes = [vp, i64, i32, i32, vp, vp, sz, vp]
    L.sasq_quantize_weight.restype = i32
    L.sasq_quantize_weight.argtypes = [vp, vp, vp, i64, i64, i32, vp]
    cache_p, batch_p = ctypes.POINTER(KVCacheStruct), ctypes.POINTER(KVBatchStruct)
    L.sasq_rope_kv_append.restype = i32
    L.sasq_rope_kv_append.argtypes = [cache_p, batch_p, vp, vp, vp, vp, i64, i64, i64, i64, i32, vp, i64, i32, i32, i32, vp]
    L.sasq_paged_attention_workspace.restype = sz
    L.sasq_paged_attention_workspace.argtypes = [cache_p, batch_p, i32]
    L.sasq_paged_attention.restype = i32
    L.sasq_paged_attention.argtypes = [cache_p, batch_p, vp, vp, vp, i64, i64, i32, f32, i32, i32, vp, sz, vp]
    _lib = L
    return L


def sasq_status_string(status: int) -> str:
    return load_library().sasq_status_string(int(status)).decode()


# ---------------------------------------------------------------------------
# marshalling helpers
# ---------------------------------------------------------------------------
def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float16:
        return SASQ_F16
    if t.dtype == torch.bfloat16:
        return SASQ_BF16
    raise TypeError(f"expected float16 or bfloat16, got {t.dtype}")


def _dev(t, name: str, dtype=None):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return t


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    """None: torch's current stream; a torch stream; or a raw cudaStream_t handle as an int (the cheapest to pass)."""
    if isinstance(stream, int):
        return stream
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


# SASQ_DEBUG_STATUS=1 in the environment: every call through this binding also synchronises and reads the sticky
# device status word, so that a device-detected problem (a bad factor, a bounded wait that gave up) raises at the
# call that caused it instead of waiting for the caller's next sasq_device_status().  For tests and debugging only.
_DEBUG_STATUS = os.environ.get("SASQ_DEBUG_STATUS", "0") not in ("", "0")


def _check(status: int, where: str):
    if status != 0:
        raise SasqError(status, where)
    if _DEBUG_STATUS:
        dev_status = int(load_library().sasq_device_status(_stream(None)))
        if dev_status != 0:
            raise SasqError(dev_status, where + " (device status)")


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


# ---------------------------------------------------------------------------
# the entry points
# ---------------------------------------------------------------------------
def sasq_fakequant_fwd(x: torch.Tensor, y: torch.Tensor, scale: torch.Tensor, bits: int = 8, stream=None) -> None:
    _dev(x, "x"); _dev(y, "y", x.dtype); _dev(scale, "scale", torch.float32)
    if y.numel() != x.numel():
        raise ValueError("y must have as many elements as x")
    _check(load_library().sasq_fakequant_fwd(_ptr(x), _ptr(y), x.numel(), _dt(x), _ptr(scale), int(bits),
                                             _stream(stream)), "sasq_fakequant_fwd")


def sasq_fakequant_bwd_workspace(numel: int) -> int:
    return int(load_library().sasq_fakequant_bwd_workspace(int(numel)))


def sasq_fakequant_bwd(x, grad_y, grad_x, grad_scale, scale, workspace, bits: int = 8, accumulate: bool = False,
                       stream=None) -> None:
    _dev(x, "x"); _dev(grad_y, "grad_y", x.dtype); _dev(grad_x, "grad_x", x.dtype)
    _dev(grad_scale, "grad_scale", torch.float32); _dev(scale, "scale", torch.float32); _dev(workspace, "workspace")
    if grad_y.numel() != x.numel() or grad_x.numel() != x.numel():
        raise ValueError("grad_y and grad_x must have as many elements as x")
    _check(load_library().sasq_fakequant_bwd(_ptr(x), _ptr(grad_y), _ptr(grad_x), _ptr(grad_scale), int(bool(accumulate)),
                                             x.numel(), _dt(x), _ptr(scale), int(bits), _ptr(workspace),
                                             _nbytes(workspace), _stream(stream)), "sasq_fakequant_bwd")


def sasq_fakequant_fwd_bwd(x, grad_y, y, grad_x, grad_scale, scale, workspace, bits: int = 8,
                           accumulate: bool = False, stream=None) -> None:
    _dev(x, "x"); _dev(grad_y, "grad_y", x.dtype); _dev(y, "y", x.dtype); _dev(grad_x, "grad_x", x.dtype)
    _dev(grad_scale, "grad_scale", torch.float32); _dev(scale, "scale", torch.float32); _dev(workspace, "workspace")
    if grad_y.numel() != x.numel() or grad_x.numel() != x.numel() or y.numel() != x.numel():
        raise ValueError("grad_y, y and grad_x must have as many elements as x")
    _check(load_library().sasq_fakequant_fwd_bwd(_ptr(x), _ptr(grad_y), _ptr(y), _ptr(grad_x), _ptr(grad_scale),
                                                 int(bool(accumulate)), x.numel(), _dt(x), _ptr(scale), int(bits),
                                                 _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "sasq_fakequant_fwd_bwd")


def sasq_fakequant_multi_workspace(n_tensors: int) -> int:
    return int(load_library().sasq_fakequant_multi_workspace(int(n_tensors)))


class QuantTensors:
    """The descriptor table of a sasq_fakequant_fwd_bwd_multi call, marshalled once (see LinearProblems)."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        n = len(self.tensors)
        self.descs = (QDesc * max(n, 1))()
        dt = None
        for i, (x, gy, y, gx, idx) in enumerate(self.tensors):
            _dev(x, "x")
            for name, t in (("grad_y", gy), ("y", y), ("grad_x", gx)):
                if t is not None:
                    _dev(t, name, x.dtype)
                    if t.numel() != x.numel():
                        raise ValueError(f"{name} must have as many elements as x")
            if dt is None:
                dt = _dt(x)
            elif dt != _dt(x):
                raise TypeError("all tensors of one call must share a dtype")
            self.descs[i] = QDesc(_ptr(x), _ptr(gy), _ptr(y), _ptr(gx), x.numel(), int(idx), 0)
        self.dt = SASQ_BF16 if dt is None else dt
        self.count = n


def sasq_fakequant_fwd_bwd_multi(tensors, scales, grad_scales, workspace, bits: int = 8, accumulate: bool = False,
                                 stream=None) -> None:
    """tensors: sequence of (x, grad_y | None, y | None, grad_x | None, scale_index), or a QuantTensors made from one."""
    prepared = tensors if isinstance(tensors, QuantTensors) else QuantTensors(tensors)
    _dev(scales, "scales", torch.float32)
    if grad_scales is not None:
        _dev(grad_scales, "grad_scales", torch.float32)
    if workspace is not None:
        _dev(workspace, "workspace")
    _check(load_library().sasq_fakequant_fwd_bwd_multi(prepared.descs, prepared.count, _ptr(scales), _ptr(grad_scales),
                                                       scales.numel(), int(bool(accumulate)), prepared.dt,
                                                       int(bits), _ptr(workspace), _nbytes(workspace),
                                                       _stream(stream)), "sasq_fakequant_fwd_bwd_multi")


def sasq_fakequant_fwd_bwd_ablation(x, grad_y, y, grad_x, grad_scale, scale, workspace, variant: int, bits: int = 8,
                                    accumulate: bool = False, stream=None) -> None:
    """The fused pass with Table 3's "w/o round" / "w/o clamp" ablations (variant = SASQ_WITHOUT_*)."""
    _dev(x, "x"); _dev(grad_y, "grad_y", x.dtype); _dev(y, "y", x.dtype); _dev(grad_x, "grad_x", x.dtype)
    _dev(grad_scale, "grad_scale", torch.float32); _dev(scale, "scale", torch.float32); _dev(workspace, "workspace")
    if grad_y.numel() != x.numel() or grad_x.numel() != x.numel() or y.numel() != x.numel():
        raise ValueError("grad_y, y and grad_x must have as many elements as x")
    _check(load_library().sasq_fakequant_fwd_bwd_ablation(_ptr(x), _ptr(grad_y), _ptr(y), _ptr(grad_x),
                                                          _ptr(grad_scale), int(bool(accumulate)), x.numel(), _dt(x),
                                                          _ptr(scale), int(bits), int(variant), _ptr(workspace),
                                                          _nbytes(workspace), _stream(stream)),
           "sasq_fakequant_fwd_bwd_ablation")


def sasq_adamw_scales(scales, grad_scales, exp_avg, exp_avg_sq, step: int, lr: float = 2e-4, beta1: float = 0.9,
                      beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.01, stream=None) -> None:
    """One AdamW step on the factors, in place (scales, exp_avg, exp_avg_sq: fp32 CUDA tensors of one size)."""
    for name, t in (("scales", scales), ("grad_scales", grad_scales), ("exp_avg", exp_avg), ("exp_avg_sq", exp_avg_sq)):
        _dev(t, name, torch.float32)
        if t.numel() != scales.numel():
            raise ValueError(f"{name} must have as many elements as scales")
    _check(load_library().sasq_adamw_scales(_ptr(scales), _ptr(grad_scales), _ptr(exp_avg), _ptr(exp_avg_sq),
                                            scales.numel(), int(step), float(lr), float(beta1), float(beta2),
                                            float(eps), float(weight_decay), _stream(stream)), "sasq_adamw_scales")


def sasq_fakequant_per_channel_workspace(T: int, K: int) -> int:
    return int(load_library().sasq_fakequant_per_channel_workspace(int(T), int(K)))


def sasq_fakequant_fwd_bwd_per_channel(x, grad_y, y, grad_x, grad_scales, scales, workspace, bits: int = 8,
                                       accumulate: bool = False, stream=None) -> None:
    """x [T, K] with one factor per column: scales [K], grad_scales [K]; y or (grad_y, grad_x) may be None."""
    _dev(x, "x"); _dev(scales, "scales", torch.float32)
    if x.dim() != 2 or scales.numel() != x.shape[1]:
        raise ValueError("x must be [T, K] and scales [K]")
    for name, t in (("grad_y", grad_y), ("y", y), ("grad_x", grad_x)):
        if t is not None:
            _dev(t, name, x.dtype)
            if tuple(t.shape) != tuple(x.shape):
                raise ValueError(f"{name} must have the shape of x")
    if grad_scales is not None:
        _dev(grad_scales, "grad_scales", torch.float32)
        if grad_scales.numel() != x.shape[1]:
            raise ValueError("grad_scales must be [K]")
    if workspace is not None:
        _dev(workspace, "workspace")
    _check(load_library().sasq_fakequant_fwd_bwd_per_channel(_ptr(x), _ptr(grad_y), _ptr(y), _ptr(grad_x),
                                                             _ptr(grad_scales), int(bool(accumulate)), x.shape[0],
                                                             x.shape[1], _dt(x), _ptr(scales), int(bits),
                                                             _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "sasq_fakequant_fwd_bwd_per_channel")


def sasq_fakequant_per_channel_multi_workspace(total_K: int) -> int:
    return int(load_library().sasq_fakequant_per_channel_multi_workspace(int(total_K)))


def sasq_fakequant_fwd_bwd_per_channel_multi(tensors, workspace, bits: int = 8, accumulate: bool = False,
                                             stream=None) -> None:
    """tensors: sequence of (x [T, K], grad_y | None, y | None, grad_x | None, scales [K], grad_scales [K] | None)."""
    n = len(tensors)
    descs = (PcDesc * max(n, 1))()
    dt = None
    for i, (x, gy, y, gx, sc, gs) in enumerate(tensors):
        _dev(x, "x"); _dev(sc, "scales", torch.float32)
        if x.dim() != 2 or sc.numel() != x.shape[1]:
            raise ValueError("x must be [T, K] and scales [K]")
        for name, t in (("grad_y", gy), ("y", y), ("grad_x", gx)):
            if t is not None:
                _dev(t, name, x.dtype)
                if tuple(t.shape) != tuple(x.shape):
                    raise ValueError(f"{name} must have the shape of x")
        if gs is not None:
            _dev(gs, "grad_scales", torch.float32)
        if dt is None:
            dt = _dt(x)
        elif dt != _dt(x):
            raise TypeError("all tensors of one call must share a dtype")
        descs[i] = PcDesc(_ptr(x), _ptr(gy), _ptr(y), _ptr(gx), _ptr(sc), _ptr(gs), x.shape[0], x.shape[1], 0)
    if workspace is not None:
        _dev(workspace, "workspace")
    _check(load_library().sasq_fakequant_fwd_bwd_per_channel_multi(descs, n, int(bool(accumulate)),
                                                                   SASQ_BF16 if dt is None else dt, int(bits),
                                                                   _ptr(workspace), _nbytes(workspace),
                                                                   _stream(stream)),
           "sasq_fakequant_fwd_bwd_per_channel_multi")


def sasq_static_w8a8_linear_workspace(T: int, N: int, K: int) -> int:
    return int(load_library().sasq_static_w8a8_linear_workspace(int(T), int(N), int(K)))


def sasq_static_w8a8_linear(x, w, w_scale, x_scale, y, bias=None, acc_out=None, workspace=None, bits: int = 8,
                            stream=None) -> None:
    """x [T, K] fp16/bf16, w [N, K] int8, w_scale [N] fp32, x_scale [1] fp32, y [T, N]."""
    _dev(x, "x"); _dev(w, "w", torch.int8); _dev(w_scale, "w_scale", torch.float32)
    _dev(x_scale, "x_scale", torch.float32); _dev(y, "y", x.dtype)
    if bias is not None:
        _dev(bias, "bias", x.dtype)
    if acc_out is not None:
        _dev(acc_out, "acc_out", torch.int32)
    if workspace is not None:
        _dev(workspace, "workspace")
    if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[1]:
        raise ValueError("x must be [T, K] and w [N, K]")
    T, K = x.shape
    N = w.shape[0]
    if tuple(y.shape) != (T, N) or w_scale.numel() != N or (bias is not None and bias.numel() != N):
        raise ValueError("y must be [T, N], w_scale and bias [N]")
    if acc_out is not None and tuple(acc_out.shape) != (T, N):
        raise ValueError("acc_out must be [T, N]")
    _check(load_library().sasq_static_w8a8_linear(_ptr(x), _ptr(w), _ptr(w_scale), _ptr(x_scale), _ptr(bias), _ptr(y),
                                                  _ptr(acc_out), T, N, K, _dt(x), int(bits), _ptr(workspace),
                                                  _nbytes(workspace), _stream(stream)), "sasq_static_w8a8_linear")


def sasq_fakequant_linear_fp_weights_workspace(T: int, N: int, K: int) -> int:
    return int(load_library().sasq_fakequant_linear_fp_weights_workspace(int(T), int(N), int(K)))


def sasq_fakequant_linear_fp_weights(x, w, x_scale, y, bias=None, workspace=None, bits: int = 8, stream=None) -> None:
    """Table 3's "FP weights" form: fake-quantized activations times 16-bit weights; x [T, K], w [N, K], y [T, N]."""
    _dev(x, "x"); _dev(w, "w", x.dtype); _dev(x_scale, "x_scale", torch.float32); _dev(y, "y", x.dtype)
    if bias is not None:
        _dev(bias, "bias", x.dtype)
    if workspace is not None:
        _dev(workspace, "workspace")
    if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[1]:
        raise ValueError("x must be [T, K] and w [N, K]")
    T, K = x.shape
    N = w.shape[0]
    if tuple(y.shape) != (T, N) or (bias is not None and bias.numel() != N):
        raise ValueError("y must be [T, N] and bias [N]")
    _check(load_library().sasq_fakequant_linear_fp_weights(_ptr(x), _ptr(w), _ptr(x_scale), _ptr(bias), _ptr(y), T, N, K,
                                                           _dt(x), int(bits), _ptr(workspace), _nbytes(workspace),
                                                           _stream(stream)), "sasq_fakequant_linear_fp_weights")


def sasq_static_w8a8_linear_grouped_workspace(T: int, N: int, K: int) -> int:
    return int(load_library().sasq_static_w8a8_linear_grouped_workspace(int(T), int(N), int(K)))


def sasq_static_w8a8_linear_grouped(x, w, w_scale, s_group, group: int, y, bias=None, workspace=None, bits: int = 8,
                                    stream=None) -> None:
    """Eq. 3: x [T, K], one static factor per group of `group` consecutive channels (s_group [K / group])."""
    _dev(x, "x"); _dev(w, "w", torch.int8); _dev(w_scale, "w_scale", torch.float32)
    _dev(s_group, "s_group", torch.float32); _dev(y, "y", x.dtype)
    if bias is not None:
        _dev(bias, "bias", x.dtype)
    if workspace is not None:
        _dev(workspace, "workspace")
    if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[1]:
        raise ValueError("x must be [T, K] and w [N, K]")
    T, K = x.shape
    N = w.shape[0]
    if group <= 0 or K % group != 0 or s_group.numel() != K // group:
        raise ValueError("s_group must hold one factor per group of `group` channels")
    if tuple(y.shape) != (T, N) or w_scale.numel() != N or (bias is not None and bias.numel() != N):
        raise ValueError("y must be [T, N], w_scale and bias [N]")
    _check(load_library().sasq_static_w8a8_linear_grouped(_ptr(x), _ptr(w), _ptr(w_scale), _ptr(s_group), int(group),
                                                          _ptr(bias), _ptr(y), T, N, K, _dt(x), int(bits),
                                                          _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "sasq_static_w8a8_linear_grouped")


def _linear_descs(problems):
    """problems: sequence of (x, w, w_scale, x_scale, y) or (x, w, w_scale, x_scale, y, bias)."""
    arr = (LinearDesc * max(1, len(problems)))()
    dt = None
    for i, pr in enumerate(problems):
        x, w, w_scale, x_scale, y = pr[:5]
        bias = pr[5] if len(pr) > 5 else None
        _dev(x, "x"); _dev(w, "w", torch.int8); _dev(w_scale, "w_scale", torch.float32)
        _dev(x_scale, "x_scale", torch.float32); _dev(y, "y", x.dtype)
        if bias is not None:
            _dev(bias, "bias", x.dtype)
        if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[1]:
            raise ValueError("x must be [T, K] and w [N, K]")
        T, K = x.shape
        N = w.shape[0]
        if tuple(y.shape) != (T, N) or w_scale.numel() != N or (bias is not None and bias.numel() != N):
            raise ValueError("y must be [T, N], w_scale and bias [N]")
        if dt is None:
            dt = _dt(x)
        elif dt != _dt(x):
            raise ValueError("all problems of one call share the activation dtype")
        arr[i] = LinearDesc(_ptr(x), _ptr(w), _ptr(w_scale), _ptr(x_scale), _ptr(bias), _ptr(y), T, N, K)
    return arr, dt


def sasq_static_w8a8_linear_multi_workspace(shapes) -> int:
    """shapes: sequence of (T, N, K)."""
    arr = (LinearDesc * max(1, len(shapes)))()
    for i, (T, N, K) in enumerate(shapes):
        arr[i].T, arr[i].N, arr[i].K = int(T), int(N), int(K)
    return int(load_library().sasq_static_w8a8_linear_multi_workspace(len(shapes), arr))


class LinearProblems:
    """The descriptor table of a sasq_static_w8a8_linear_multi call, marshalled once: a caller that submits the same
    tensors again and again (a layer's weights and activation buffers) passes this instead of the tuples and skips
    the per-call checks and conversions.  Holds references to the tensors so the pointers stay valid."""

    def __init__(self, problems):
        self.problems = list(problems)
        self.descs, dt = _linear_descs(self.problems)
        self.dt = SASQ_BF16 if dt is None else dt
        self.count = len(self.problems)
        self._ws = None         # (workspace tensor, pointer, bytes) of the last call: checked once per workspace


def sasq_static_w8a8_linear_multi(problems, workspace, bits: int = 8, stream=None) -> None:
    """Independent static W8A8 linears submitted together: a sequence of tuples (see _linear_descs) or a
    LinearProblems made from one."""
    prepared = problems if isinstance(problems, LinearProblems) else LinearProblems(problems)
    ws = prepared._ws
    if ws is None or ws[0] is not workspace:
        _dev(workspace, "workspace")
        ws = prepared._ws = (workspace, _ptr(workspace), _nbytes(workspace))
    _check(load_library().sasq_static_w8a8_linear_multi(prepared.count, prepared.descs, prepared.dt, int(bits),
                                                        ws[1], ws[2], _stream(stream)),
           "sasq_static_w8a8_linear_multi")


def sasq_static_w8a8_linear_multi_launches(shapes, num_pairs: int = 74) -> int:
    """Kernels one sasq_static_w8a8_linear_multi call launches for problems of these (T, N, K) on a device with
    `num_pairs` resident CTA pairs (launch counting; asks the library, touches no device)."""
    arr = (LinearDesc * max(1, len(shapes)))()
    for i, (T, N, K) in enumerate(shapes):
        arr[i].T, arr[i].N, arr[i].K = int(T), int(N), int(K)
    n = int(load_library().sasq_static_w8a8_linear_multi_launches(len(shapes), arr, int(num_pairs)))
    if n < 0:
        raise ValueError("invalid shapes")
    return n


def sasq_static_w8a8_linear_per_channel_workspace(T: int, N: int, K: int) -> int:
    return int(load_library().sasq_static_w8a8_linear_per_channel_workspace(int(T), int(N), int(K)))


def sasq_static_w8a8_linear_per_channel(x, w, w_scale, x_scales, y, bias=None, acc_out=None, workspace=None,
                                        bits: int = 8, stream=None) -> None:
    """x [T, K], x_scales [K] (one static factor per channel, already folded into w), w [N, K] int8, y [T, N]."""
    _dev(x, "x"); _dev(w, "w", torch.int8); _dev(w_scale, "w_scale", torch.float32)
    _dev(x_scales, "x_scales", torch.float32); _dev(y, "y", x.dtype)
    for name, t, dtp in (("bias", bias, x.dtype), ("acc_out", acc_out, torch.int32)):
        if t is not None:
            _dev(t, name, dtp)
    if workspace is not None:
        _dev(workspace, "workspace")
    if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[1] or x_scales.numel() != x.shape[1]:
        raise ValueError("x must be [T, K], w [N, K] and x_scales [K]")
    T, K = x.shape
    N = w.shape[0]
    if tuple(y.shape) != (T, N) or w_scale.numel() != N or (bias is not None and bias.numel() != N):
        raise ValueError("y must be [T, N], w_scale and bias [N]")
    _check(load_library().sasq_static_w8a8_linear_per_channel(_ptr(x), _ptr(w), _ptr(w_scale), _ptr(x_scales),
                                                              _ptr(bias), _ptr(y), _ptr(acc_out), T, N, K, _dt(x),
                                                              int(bits), _ptr(workspace), _nbytes(workspace),
                                                              _stream(stream)),
           "sasq_static_w8a8_linear_per_channel")


def sasq_dynamic_w8a8_linear_workspace(T: int, N: int, K: int) -> int:
    return int(load_library().sasq_dynamic_w8a8_linear_workspace(int(T), int(N), int(K)))


def sasq_dynamic_w8a8_linear(x, w, w_scale, y, bias=None, row_scale_out=None, acc_out=None, workspace=None,
                             bits: int = 8, stream=None) -> None:
    """Dynamic per-token W8A8 linear: x [T, K], w [N, K] int8, w_scale [N], y [T, N]; row_scale_out [T] fp32 or None."""
    _dev(x, "x"); _dev(w, "w", torch.int8); _dev(w_scale, "w_scale", torch.float32); _dev(y, "y", x.dtype)
    for name, t, dtp in (("bias", bias, x.dtype), ("row_scale_out", row_scale_out, torch.float32),
                         ("acc_out", acc_out, torch.int32)):
        if t is not None:
            _dev(t, name, dtp)
    if workspace is not None:
        _dev(workspace, "workspace")
    if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[1]:
        raise ValueError("x must be [T, K] and w [N, K]")
    T, K = x.shape
    N = w.shape[0]
    if tuple(y.shape) != (T, N) or w_scale.numel() != N or (bias is not None and bias.numel() != N):
        raise ValueError("y must be [T, N], w_scale and bias [N]")
    if row_scale_out is not None and row_scale_out.numel() != T:
        raise ValueError("row_scale_out must be [T]")
    if acc_out is not None and tuple(acc_out.shape) != (T, N):
        raise ValueError("acc_out must be [T, N]")
    _check(load_library().sasq_dynamic_w8a8_linear(_ptr(x), _ptr(w), _ptr(w_scale), _ptr(bias), _ptr(y),
                                                   _ptr(row_scale_out), _ptr(acc_out), T, N, K, _dt(x), int(bits),
                                                   _ptr(workspace), _nbytes(workspace), _stream(stream)),
           "sasq_dynamic_w8a8_linear")


def sasq_static_w8a8_linear_tiles(T: int, N: int, num_pairs: int, pair_id: int):
    """Tiles (first row, first column, width) that CTA pair `pair_id` of `num_pairs` walks for a [T, N] output."""
    L = load_library()
    n = L.sasq_static_w8a8_linear_tiles(int(T), int(N), int(num_pairs), int(pair_id), None, 0)
    if n < 0:
        raise ValueError("invalid arguments")
    buf = (ctypes.c_int32 * (3 * max(n, 1)))()
    L.sasq_static_w8a8_linear_tiles(int(T), int(N), int(num_pairs), int(pair_id), buf, n)
    return [(buf[3 * i], buf[3 * i + 1], buf[3 * i + 2]) for i in range(n)]


def sasq_debug_set_wait_limit(cycles: int) -> int:
    """Test hook: clock cycles after which a wait inside the GEMM kernels gives up (negative restores the default)."""
    return int(load_library().sasq_debug_set_wait_limit(int(cycles)))


def sasq_debug_int8_issue_rate(mma_per_pair: int, n_cols: int = 256, stream=None):
    """Measurement aid: back-to-back int8 tensor-core instructions of the GEMM's shape on every CTA pair.
    Returns (integer operations per second of the device, multiply-accumulates per clock per SM)."""
    L = load_library()
    L.sasq_debug_int8_issue_rate.restype = ctypes.c_int
    L.sasq_debug_int8_issue_rate.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                             ctypes.POINTER(ctypes.c_double), ctypes.c_void_p]
    ops, mac = ctypes.c_double(0.0), ctypes.c_double(0.0)
    _check(L.sasq_debug_int8_issue_rate(int(mma_per_pair), int(n_cols), ctypes.byref(ops), ctypes.byref(mac),
                                        _stream(stream)), "sasq_debug_int8_issue_rate")
    return float(ops.value), float(mac.value)


def sasq_set_gang_launch(on: bool) -> bool:
    """Launch the linears whose CTAs wait on one another as co-operative grids (the default; safe with several
    streams).  A caller that keeps all linears on one stream may pass False; returns the previous setting."""
    L = load_library()
    L.sasq_set_gang_launch.restype = ctypes.c_int
    L.sasq_set_gang_launch.argtypes = [ctypes.c_int]
    return bool(L.sasq_set_gang_launch(1 if on else 0))


def sasq_device_status(stream=None) -> int:
    """Synchronises the stream; returns and clears the sticky device status (0 = OK)."""
    return int(load_library().sasq_device_status(_stream(stream)))


def sasq_absmax_scale_per_channel(x, scales_out, bits: int = 8, stream=None) -> None:
    """scales_out[k] = max_t |x[t, k]| / Qp (Eq. 1 per channel) of one calibration batch; x [T, K]."""
    _dev(x, "x"); _dev(scales_out, "scales_out", torch.float32)
    if x.dim() != 2 or scales_out.numel() != x.shape[1]:
        raise ValueError("x must be [T, K] and scales_out [K]")
    L = load_library()
    L.sasq_absmax_scale_per_channel.restype = ctypes.c_int
    L.sasq_absmax_scale_per_channel.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_int,
                                                ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
    _check(L.sasq_absmax_scale_per_channel(_ptr(x), x.shape[0], x.shape[1], _dt(x), int(bits), _ptr(scales_out),
                                           _stream(stream)), "sasq_absmax_scale_per_channel")


def sasq_running_mean(mean, value, count: int, stream=None) -> None:
    """mean <- mean of the first `count` values, given the mean of the first count - 1 and the count-th value."""
    _dev(mean, "mean", torch.float32); _dev(value, "value", torch.float32)
    if mean.numel() != value.numel():
        raise ValueError("mean and value must have the same number of elements")
    L = load_library()
    L.sasq_running_mean.restype = ctypes.c_int
    L.sasq_running_mean.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p]
    _check(L.sasq_running_mean(_ptr(mean), _ptr(value), mean.numel(), int(count), _stream(stream)), "sasq_running_mean")


def sasq_absmax_scale_workspace(numel: int) -> int:
    return int(load_library().sasq_absmax_scale_workspace(int(numel)))


def sasq_absmax_scale(x, scale_out, workspace, bits: int = 8, stream=None) -> None:
    """scale_out[0] = max|x| / Qp (Eq. 1) of one calibration batch."""
    _dev(x, "x"); _dev(scale_out, "scale_out", torch.float32); _dev(workspace, "workspace")
    _check(load_library().sasq_absmax_scale(_ptr(x), x.numel(), _dt(x), int(bits), _ptr(scale_out), _ptr(workspace),
                                            _nbytes(workspace), _stream(stream)), "sasq_absmax_scale")


def sasq_quantize_weight(w, w_int, w_scale, bits: int = 8, stream=None) -> None:
    """w [N, K] fp32 -> w_int [N, K] int8 and w_scale [N] fp32, one factor per output channel."""
    _dev(w, "w", torch.float32); _dev(w_int, "w_int", torch.int8); _dev(w_scale, "w_scale", torch.float32)
    if w.dim() != 2 or tuple(w_int.shape) != tuple(w.shape) or w_scale.numel() != w.shape[0]:
        raise ValueError("w and w_int must be [N, K], w_scale [N]")
    _check(load_library().sasq_quantize_weight(_ptr(w), _ptr(w_int), _ptr(w_scale), w.shape[0], w.shape[1], int(bits),
                                               _stream(stream)), "sasq_quantize_weight")


def sasq_fakequant_fwd_bwd_static(x, grad_y, y, grad_x, grad_scale, scale, bits: int = 8, accumulate: bool = False,
                                  stream=None) -> None:
    """Fused forward + backward without any workspace argument: the reduction scratch is a fixed array inside the
    library, for callers that are not allowed to allocate (see include/sasq.h).  Calls on one device must not
    overlap; the first call on a device should be made outside stream capture."""
    _dev(x, "x"); _dev(grad_y, "grad_y", x.dtype); _dev(y, "y", x.dtype); _dev(grad_x, "grad_x", x.dtype)
    _dev(grad_scale, "grad_scale", torch.float32); _dev(scale, "scale", torch.float32)
    if grad_y.numel() != x.numel() or grad_x.numel() != x.numel() or y.numel() != x.numel():
        raise ValueError("grad_y, y and grad_x must have as many elements as x")
    _check(load_library().sasq_fakequant_fwd_bwd_static(_ptr(x), _ptr(grad_y), _ptr(y), _ptr(grad_x),
                                                        _ptr(grad_scale), int(bool(accumulate)), x.numel(), _dt(x),
                                                        _ptr(scale), int(bits), _stream(stream)),
           "sasq_fakequant_fwd_bwd_static")


def _on(device: int, *pairs) -> None:
    """Tensors of a call that launches on the current device: contiguous, on that device, of the given dtypes."""
    if _current_device() != device:
        raise ValueError(f"the tensors lie on cuda:{device}, the current device is cuda:{_current_device()} (enter "
                         f"torch.cuda.device({device}))")
    for t, name, dtype in pairs:
        if t is not None:
            _flat(t, name, device, dtype)


def sasq_w4_linear(x, w, w_scale, y, bias=None, stream=None) -> None:
    """y [T, N] = x [T, K] times 4-bit weights: w [N, K / 2] uint8 (column 2i in the low half of byte i), w_scale
    [N, K / group] of x's dtype with group 32, 64 or 128; bias [N] or None."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError("x must be a CUDA tensor")
    device, dt = x.get_device(), x.dtype
    if _current_device() != device:
        _on(device)
    _flat(x, "x", device)
    _flat(w, "w", device, torch.uint8)
    _flat(w_scale, "w_scale", device, dt)
    _flat(y, "y", device, dt)
    if bias is not None:
        _flat(bias, "bias", device, dt)
    xs, ws, ss, ys = x.shape, w.shape, w_scale.shape, y.shape
    if len(xs) != 2 or len(ws) != 2 or len(ss) != 2 or len(ys) != 2:
        raise ValueError("x, w, w_scale and y must be matrices")
    T, K = xs
    N, half = ws
    rows, groups = ss
    if K != 2 * half or rows != N or groups <= 0 or K % groups != 0 or ys != (T, N) or (bias is not None and bias.shape != (N,)):
        raise ValueError(f"x [{T}, K], w [N, K / 2], w_scale [N, K / group], y [{T}, N] and bias [N] do not fit together: "
                         f"{tuple(xs)}, {tuple(ws)}, {tuple(ss)}, {tuple(ys)}")
    status = (_lib or load_library()).sasq_w4_linear(x.data_ptr(), w.data_ptr(), w_scale.data_ptr(), _ptr(bias), y.data_ptr(), T, N, K,
                                                     K // groups, _dt(x), _stream_of(device, stream))
    if status != 0 or _DEBUG_STATUS:
        _check(status, "sasq_w4_linear")


def sasq_quantize_weight_w4(w, w_int, w_scale, stream=None) -> None:
    """w [N, K] fp32 -> w_int [N, K / 2] uint8 and w_scale [N, K / group] fp16 or bf16, for sasq_w4_linear."""
    if not isinstance(w, torch.Tensor) or not w.is_cuda:
        raise TypeError("w must be a CUDA tensor")
    device = w.get_device()
    _on(device, (w, "w", torch.float32), (w_int, "w_int", torch.uint8), (w_scale, "w_scale", None))
    if w.dim() != 2 or w_scale.dim() != 2 or w_int.shape != (w.shape[0], w.shape[1] // 2) or w.shape[1] % 2 or \
            w_scale.shape[0] != w.shape[0] or w_scale.shape[1] <= 0 or w.shape[1] % w_scale.shape[1] != 0:
        raise ValueError("w must be [N, K], w_int [N, K / 2] and w_scale [N, K / group]")
    N, K = w.shape
    _check(load_library().sasq_quantize_weight_w4(w.data_ptr(), w_int.data_ptr(), w_scale.data_ptr(), N, K, K // w_scale.shape[1],
                                                  _dt(w_scale), _stream_of(device, stream)), "sasq_quantize_weight_w4")


# ---------------------------------------------------------------------------
# paged key/value cache
# ---------------------------------------------------------------------------
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _elsewhere(device: int, t, name: str):
    """Says why a tensor that does not lie on `device` is refused."""
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    raise ValueError(f"{name} lies on cuda:{t.get_device()}, the other tensors of the call on cuda:{device}")


def _flat(t, name: str, device: int, dtype=None) -> None:
    """As _dev, for a tensor that goes with others of `device`."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.get_device() != device:                       # a host tensor says -1
        _elsewhere(device, t, name)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")


def _wrong_device(cache, batch):
    """Says why a call is refused whose handles do not lie on the current device, where the library launches."""
    if batch.device != cache.device:
        raise ValueError(f"the batch lies on cuda:{batch.device}, the cache on cuda:{cache.device}")
    raise ValueError(f"the cache lies on cuda:{cache.device}, the current device is cuda:{_current_device()} (enter "
                     f"torch.cuda.device({cache.device}))")


class KVCache:
    """A paged cache, marshalled once (see LinearProblems).  k, v: [num_pages, page_size, num_kv_heads, head_dim] views
    of one stride pattern, last dimension contiguous (a pool stored heads first is passed as its .transpose(1, 2));
    fp16 / bf16, or int8 with k_scale, v_scale: [num_kv_heads] fp32 factors, or uint8 for 4-bit codes, two to a byte (the
    last dimension is head_dim / 2), with k_scale, v_scale: [num_kv_heads, head_dim].  Holds references to the tensors."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        for name, t in (("k", k), ("v", v)):
            if not isinstance(t, torch.Tensor) or not t.is_cuda:
                raise TypeError(f"{name} must be a CUDA tensor")
            if t.dim() != 4 or t.stride(3) != 1:
                raise ValueError(f"{name} must be [num_pages, page_size, num_kv_heads, head_dim] with a contiguous last "
                                 "dimension")
            if t.dtype not in (torch.uint8, torch.int8, torch.float16, torch.bfloat16):
                raise TypeError(f"{name} must be uint8 (4-bit codes), int8, float16 or bfloat16, got {t.dtype}")
        if k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.get_device() != v.get_device():
            raise ValueError("k and v must share shape, strides, dtype and device")
        int8, int4 = k.dtype == torch.int8, k.dtype == torch.uint8
        self.device = k.get_device()
        self.num_kv_heads, self.head_dim = k.shape[2], k.shape[3] * 2 if int4 else k.shape[3]
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            if (int8 or int4) != (t is not None):
                raise ValueError(f"{name} goes with an int8 or 4-bit cache, and only with it")
            if t is not None:
                _flat(t, name, self.device, torch.float32)
                if int8 and t.numel() != k.shape[2]:
                    raise ValueError(f"{name} must hold one factor per KV head")
                if int4 and t.shape != (self.num_kv_heads, self.head_dim):
                    raise ValueError(f"{name} must be [num_kv_heads, head_dim]")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.dtype = k.dtype
        self.token_dtype = None if int8 or int4 else k.dtype    # of the tokens that go in and come out; None: either
        # a dimension of one entry may have any stride in torch; the library wants whole 16-byte words
        strides = [s if n > 1 else k.shape[3] for s, n in zip(k.stride()[:3], k.shape)]
        page_stride, token_stride, head_stride = (2 * s for s in strides) if int4 else strides
        self.struct = KVCacheStruct(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), page_stride, token_stride, head_stride,
                                    k.shape[0], k.shape[1], k.shape[2], self.head_dim,
                                    SASQ_KV_INT4 if int4 else SASQ_KV_INT8 if int8 else SASQ_KV_16BIT)
        self.ref = ctypes.byref(self.struct)


class PagedBatch:
    """The sequences of a call, marshalled once: page_table [batch, max_pages], seq_lens [batch], q_starts [batch + 1],
    int32 CUDA tensors whose VALUES may change between calls; total_q rows of q; upper bounds of a sequence's new tokens
    and keys, known to the host (default: total_q, and what the page table can hold)."""

    def __init__(self, page_table, seq_lens, q_starts, total_q: int, max_q_len: int | None = None,
                 max_seq_len: int | None = None):
        if not isinstance(page_table, torch.Tensor) or not page_table.is_cuda or page_table.dtype != torch.int32:
            raise TypeError("page_table must be an int32 CUDA tensor")
        if page_table.dim() != 2 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
            raise ValueError("page_table must be [batch, max_pages] with contiguous rows")
        if page_table.shape[0] > 1 and page_table.stride(0) < page_table.shape[1]:
            raise ValueError("the rows of page_table must not overlap (an expanded table needs a copy)")
        self.device = page_table.get_device()
        _flat(seq_lens, "seq_lens", self.device, torch.int32); _flat(q_starts, "q_starts", self.device, torch.int32)
        B, max_pages = page_table.shape
        if seq_lens.numel() != B or q_starts.numel() != B + 1:
            raise ValueError("seq_lens must be [batch] and q_starts [batch + 1]")
        self.page_table, self.seq_lens, self.q_starts = page_table, seq_lens, q_starts
        self.total_q = int(total_q)
        longest = 0x7FFFFFFF if max_seq_len is None else int(max_seq_len)
        self.struct = KVBatchStruct(_ptr(page_table), _ptr(seq_lens), _ptr(q_starts), page_table.stride(0) if B > 1 else max_pages,
                                    B, max_pages, self.total_q, self.total_q if max_q_len is None else int(max_q_len),
                                    longest, 0)
        self.ref = ctypes.byref(self.struct)


def _heads(t, name: str, dtype, total: int, heads: int | None, dim: int, device: int):
    """[total, heads, dim] with each row's heads contiguous; returns (heads, row stride)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.get_device() != device:
        _elsewhere(device, t, name)
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[0] != total or shape[2] != dim or (heads is not None and shape[1] != heads):
        raise ValueError(f"{name} must be [{total}, {'heads' if heads is None else heads}, {dim}]")
    if stride[2] != 1 or (shape[1] > 1 and stride[1] != dim):
        raise ValueError(f"the heads of a row of {name} must be contiguous")
    return shape[1], (stride[0] if total > 1 else shape[1] * dim)      # one row may have any stride in torch


def _stream_of(device: int, stream) -> int:
    """As _stream, for calls whose tensors are known to lie on one device: the raw handle of its current stream."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device)
    return stream if isinstance(stream, int) else stream.cuda_stream


def sasq_rope_kv_append(cache: KVCache, batch: PagedBatch, q, k, v, q_out, cos_sin, interleaved: bool = False,
                        stream=None) -> None:
    """Appends k, v [total_q, num_kv_heads, head_dim] to the cache with the rotation of cos_sin [max_positions, rot_dim]
    fp32 (None: no rotation) applied to k, and to q [total_q, num_q_heads, head_dim] -> q_out (both None: skip)."""
    T, K, D = batch.total_q, cache.num_kv_heads, cache.head_dim
    device = cache.device
    if batch.device != device or _current_device() != device:
        _wrong_device(cache, batch)
    dt = k.dtype
    if cache.token_dtype is not None and cache.token_dtype != dt:
        raise TypeError(f"k must have the cache's dtype {cache.dtype}")
    _, ks = _heads(k, "k", dt, T, K, D, device)
    _, vs = _heads(v, "v", dt, T, K, D, device)
    H = qs = qos = 0
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out go together")
    if q is not None:
        H, qs = _heads(q, "q", dt, T, None, D, device)
        _, qos = _heads(q_out, "q_out", dt, T, H, D, device)
    positions = rot = 0
    if cos_sin is not None:
        _flat(cos_sin, "cos_sin", device, torch.float32)
        if cos_sin.dim() != 2:
            raise ValueError("cos_sin must be [max_positions, rot_dim]")
        positions, rot = cos_sin.shape
    status = (_lib or load_library()).sasq_rope_kv_append(
        cache.ref, batch.ref, _ptr(q), k.data_ptr(), v.data_ptr(), _ptr(q_out), qs, ks, vs, qos, H, _ptr(cos_sin), positions,
        rot, 1 if interleaved else 0, _dt(k), _stream_of(device, stream))
    if status != 0 or _DEBUG_STATUS:
        _check(status, "sasq_rope_kv_append")


def sasq_paged_attention_workspace(cache: KVCache, batch: PagedBatch, num_q_heads: int) -> int:
    return int(load_library().sasq_paged_attention_workspace(cache.ref, batch.ref, int(num_q_heads)))


def sasq_paged_attention(cache: KVCache, batch: PagedBatch, q, out, workspace, lse=None, scale: float | None = None,
                         causal: bool = True, stream=None) -> None:
    """Attention of q [total_q, num_q_heads, head_dim] over the cache -> out of the same shape, lse [total_q, num_q_heads]
    fp32 or None; scale defaults to head_dim ** -0.5."""
    T, D = batch.total_q, cache.head_dim
    device = cache.device
    if batch.device != device or _current_device() != device:
        _wrong_device(cache, batch)
    dt = q.dtype
    if cache.token_dtype is not None and cache.token_dtype != dt:
        raise TypeError(f"q must have the cache's dtype {cache.dtype}")
    H, qs = _heads(q, "q", dt, T, None, D, device)
    _, os_ = _heads(out, "out", dt, T, H, D, device)
    if lse is not None:
        _flat(lse, "lse", device, torch.float32)
        if lse.shape != (T, H):
            raise ValueError("lse must be [total_q, num_q_heads]")
    _flat(workspace, "workspace", device)
    status = (_lib or load_library()).sasq_paged_attention(
        cache.ref, batch.ref, q.data_ptr(), out.data_ptr(), _ptr(lse), qs, os_, H, D ** -0.5 if scale is None else scale,
        1 if causal else 0, _dt(q), workspace.data_ptr(), workspace.nbytes, _stream_of(device, stream))
    if status != 0 or _DEBUG_STATUS:
        _check(status, "sasq_paged_attention")
