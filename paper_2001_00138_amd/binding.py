"""ctypes binding of ``libpatdnn.so`` - argument marshalling only.

Function names mirror the C ABI (``include/patdnn.h``).  Device buffers are passed
as ``torch`` CUDA/HIP tensors (or raw integer device pointers); every arithmetic
step runs inside the library.  There is no fallback: if the library is missing,
loading raises.
"""

from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpatdnn.so")

PATDNN_OK, PATDNN_EINVAL, PATDNN_EPATTERN, PATDNN_ENOMEM, PATDNN_EHIP, PATDNN_EUNSUPPORTED = range(6)
PATDNN_DENSE, PATDNN_STRICT, PATDNN_HOST_ONLY = 1, 2, 4
PATDNN_VARIANT_FKW = 0

EXPORTS = [
    "patdnn_mine_patterns", "patdnn_project_patterns", "patdnn_project_connectivity",
    "patdnn_encode", "patdnn_conv2d", "patdnn_conv2d_f16", "patdnn_conv2d_pool", "patdnn_conv2d_ws", "patdnn_workspace_floats",
    "patdnn_output_shape", "patdnn_decode",
    "patdnn_stack_create", "patdnn_stack_output_shape", "patdnn_stack_run", "patdnn_stack_run_static", "patdnn_stack_destroy",
    "patdnn_export_fkw", "patdnn_export_csr", "patdnn_layout_stats", "patdnn_num_variants", "patdnn_variant_name",
    "patdnn_set_config", "patdnn_get_config", "patdnn_tune", "patdnn_tune_ws", "patdnn_tiled_info",
    "patdnn_export_tiled", "patdnn_selftest", "patdnn_destroy",
    "patdnn_channels_last", "patdnn_channels_first",
    "patdnn_group_norm", "patdnn_group_norm_backward", "patdnn_group_norm_workspace_floats",
    "patdnn_mxfp4_quantize", "patdnn_mxfp4_dequantize", "patdnn_mxfp4_linear", "patdnn_mxfp4_linear_workspace_bytes",
    "patdnn_fp8_quantize", "patdnn_fp8_dequantize", "patdnn_rms_norm", "patdnn_rms_norm_backward", "patdnn_rms_norm_workspace_floats",
    "patdnn_fp8_linear", "patdnn_fp8_linear_workspace_bytes", "patdnn_fp8_gated", "patdnn_fp8_gated_workspace_bytes",
    "patdnn_fp8_gated_backward", "patdnn_fp8_gated_backward_workspace_bytes",
    "patdnn_status_string", "patdnn_last_error",
]
PATDNN_F32, PATDNN_F16, PATDNN_BF16, PATDNN_MXFP4, PATDNN_FP8 = range(5)
FP8_BLOCKS = {"rows": 0, "squares": 1}
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2}


class LayerDesc(ctypes.Structure):
    _fields_ = [("c_out", ctypes.c_int32), ("c_in", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("stride", ctypes.c_int32), ("pad", ctypes.c_int32),
                ("num_patterns", ctypes.c_int32), ("pattern_masks", ctypes.c_void_p),
                ("flags", ctypes.c_uint32)]


class Stats(ctypes.Structure):
    _fields_ = [("kept_kernels", ctypes.c_int64), ("taps", ctypes.c_int32),
                ("num_patterns", ctypes.c_int32), ("fkw_weight_bytes", ctypes.c_int64),
                ("fkw_index_bytes", ctypes.c_int64), ("tiled_bytes", ctypes.c_int64),
                ("min_filter_length", ctypes.c_int32), ("max_filter_length", ctypes.c_int32),
                ("distinct_filter_lengths", ctypes.c_int32), ("filter_groups", ctypes.c_int32),
                ("group_size", ctypes.c_int32), ("max_group_kernels", ctypes.c_int64),
                ("min_group_kernels", ctypes.c_int64)]


class Config(ctypes.Structure):
    _fields_ = [("variant", ctypes.c_int32), ("ck", ctypes.c_int32), ("waves", ctypes.c_int32),
                ("ksplit", ctypes.c_int32)]


class TiledInfo(ctypes.Structure):
    _fields_ = [("G", ctypes.c_int32), ("num_groups", ctypes.c_int32), ("ck", ctypes.c_int32),
                ("num_chunks", ctypes.c_int32), ("num_steps", ctypes.c_int64),
                ("block_bytes", ctypes.c_uint32), ("table_off", ctypes.c_uint32),
                ("ctrl_bytes", ctypes.c_uint32), ("records", ctypes.c_uint32),
                ("double_window", ctypes.c_int32), ("lds_channel_bytes", ctypes.c_int32),
                ("threaded", ctypes.c_int32), ("patch_rows", ctypes.c_int32),
                ("patch_cols", ctypes.c_int32), ("conv_stride", ctypes.c_int32),
                ("lanes_x", ctypes.c_int32), ("experimental", ctypes.c_int32),
                ("mode", ctypes.c_int32)]


class StackLayer(ctypes.Structure):
    _fields_ = [("layer", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("fuse_relu", ctypes.c_int32),
                ("pool2", ctypes.c_int32)]


class NormDesc(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("pixels", ctypes.c_int32), ("channels", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("type", ctypes.c_int32), ("act", ctypes.c_int32),
                ("eps", ctypes.c_float), ("x_image", ctypes.c_int64), ("x_pixel", ctypes.c_int64),
                ("y_image", ctypes.c_int64), ("y_pixel", ctypes.c_int64), ("dy_image", ctypes.c_int64),
                ("dy_pixel", ctypes.c_int64)]


class LinearDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("in_features", ctypes.c_int32), ("out_features", ctypes.c_int32),
                ("x_type", ctypes.c_int32), ("out_type", ctypes.c_int32), ("act", ctypes.c_int32),
                ("x_row", ctypes.c_int64), ("out_row", ctypes.c_int64)]


class RmsDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("type", ctypes.c_int32), ("y_type", ctypes.c_int32),
                ("eps", ctypes.c_float), ("x_row", ctypes.c_int64), ("residual_row", ctypes.c_int64), ("sum_row", ctypes.c_int64),
                ("y_row", ctypes.c_int64)]


class Fp8Desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("in_features", ctypes.c_int32), ("out_features", ctypes.c_int32),
                ("w_blocks", ctypes.c_int32), ("out_type", ctypes.c_int32), ("act", ctypes.c_int32), ("dh_type", ctypes.c_int32),
                ("out_row", ctypes.c_int64), ("dh_row", ctypes.c_int64)]


class PatdnnError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"patdnn status {status}: {text}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """Load the shared library (built by ``buildlib.build()``); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2001_00138_amd.buildlib`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32 = ctypes.c_void_p, ctypes.c_int32
        L.patdnn_encode.argtypes = [ctypes.POINTER(LayerDesc), vp, vp, vp, ctypes.POINTER(vp)]
        L.patdnn_conv2d.argtypes = [vp, vp, i32, i32, i32, vp, vp, i32, vp]
        L.patdnn_mine_patterns.argtypes = [vp, i32, i32, i32, vp, ctypes.POINTER(i32)]
        L.patdnn_project_patterns.argtypes = [vp, i32, i32, vp, i32, vp, vp]
        L.patdnn_project_connectivity.argtypes = [vp, i32, i32, ctypes.c_int64, vp]
        L.patdnn_conv2d_f16.argtypes = [vp, vp, i32, i32, i32, vp, vp, i32, vp]
        L.patdnn_conv2d_pool.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp]
        L.patdnn_conv2d_ws.argtypes = [vp, vp, i32, i32, i32, vp, vp, i32, i32, vp, ctypes.c_size_t, vp]
        L.patdnn_workspace_floats.argtypes = [vp, i32, i32, i32]
        L.patdnn_workspace_floats.restype = ctypes.c_size_t
        L.patdnn_stack_create.argtypes = [ctypes.POINTER(StackLayer), i32, i32, i32, i32, ctypes.POINTER(vp)]
        L.patdnn_stack_output_shape.argtypes = [vp, ctypes.POINTER(i32 * 4)]
        L.patdnn_stack_run.argtypes = [vp, vp, vp, i32, vp]
        L.patdnn_stack_run_static.argtypes = [vp, vp, vp, vp]
        L.patdnn_stack_destroy.argtypes = [vp]
        L.patdnn_stack_destroy.restype = None
        L.patdnn_output_shape.argtypes = [vp, i32, i32, i32, ctypes.POINTER(i32 * 4)]
        L.patdnn_decode.argtypes = [vp, vp, vp, vp]
        L.patdnn_export_fkw.argtypes = [vp, vp, vp, vp, vp, vp]
        L.patdnn_layout_stats.argtypes = [vp, ctypes.POINTER(Stats)]
        L.patdnn_export_csr.argtypes = [vp, ctypes.POINTER(ctypes.c_int64), vp, vp, vp]
        L.patdnn_num_variants.argtypes = []
        L.patdnn_variant_name.argtypes = [i32]
        L.patdnn_variant_name.restype = ctypes.c_char_p
        L.patdnn_set_config.argtypes = [vp, ctypes.POINTER(Config)]
        L.patdnn_get_config.argtypes = [vp, ctypes.POINTER(Config)]
        L.patdnn_tune.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, ctypes.POINTER(ctypes.c_float)]
        L.patdnn_tune_ws.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, ctypes.c_size_t, vp,
                                     ctypes.POINTER(ctypes.c_float)]
        L.patdnn_tiled_info.argtypes = [vp, i32, i32, ctypes.POINTER(TiledInfo)]
        L.patdnn_export_tiled.argtypes = [vp, i32, i32, vp, vp, vp]
        L.patdnn_selftest.argtypes = []
        L.patdnn_destroy.argtypes = [vp]
        L.patdnn_destroy.restype = None
        i64, size = ctypes.c_int64, ctypes.c_size_t
        L.patdnn_channels_last.argtypes = [vp, i32, i32, i32, i32, vp, i32, i64, i64, vp]
        L.patdnn_channels_first.argtypes = [vp, i32, i64, i64, i32, i32, i32, vp, i32, vp]
        L.patdnn_group_norm.argtypes = [ctypes.POINTER(NormDesc), vp, vp, vp, vp, vp, vp, vp, size, vp]
        L.patdnn_group_norm_backward.argtypes = [ctypes.POINTER(NormDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, size, vp]
        L.patdnn_group_norm_workspace_floats.argtypes = [ctypes.POINTER(NormDesc), i32]
        L.patdnn_group_norm_workspace_floats.restype = size
        L.patdnn_mxfp4_quantize.argtypes = [vp, i32, i32, i32, i64, vp, vp, vp]
        L.patdnn_mxfp4_dequantize.argtypes = [vp, vp, i32, i32, vp, i32, i64, vp]
        L.patdnn_mxfp4_linear.argtypes = [ctypes.POINTER(LinearDesc), vp, vp, vp, vp, vp, vp, vp, size, vp]
        L.patdnn_mxfp4_linear_workspace_bytes.argtypes = [ctypes.POINTER(LinearDesc)]
        L.patdnn_mxfp4_linear_workspace_bytes.restype = size
        L.patdnn_fp8_quantize.argtypes = [vp, i32, i32, i32, i64, i32, i32, vp, vp, vp]
        L.patdnn_fp8_dequantize.argtypes = [vp, vp, i32, i32, i32, vp, i32, i64, vp]
        L.patdnn_rms_norm.argtypes = [ctypes.POINTER(RmsDesc), vp, vp, vp, vp, vp, vp, vp, vp]
        L.patdnn_rms_norm_backward.argtypes = [ctypes.POINTER(RmsDesc), vp, vp, vp, vp, vp, vp, vp, vp, size, vp]
        L.patdnn_rms_norm_workspace_floats.argtypes = [ctypes.POINTER(RmsDesc)]
        L.patdnn_rms_norm_workspace_floats.restype = size
        L.patdnn_fp8_linear.argtypes = [ctypes.POINTER(Fp8Desc), vp, vp, vp, vp, vp, vp, vp, size, vp]
        L.patdnn_fp8_gated.argtypes = [ctypes.POINTER(Fp8Desc), vp, vp, vp, vp, vp, vp, vp, vp, vp, size, vp]
        L.patdnn_fp8_gated_backward.argtypes = [ctypes.POINTER(Fp8Desc), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, size, vp]
        for name in ("linear", "gated", "gated_backward"):
            getattr(L, f"patdnn_fp8_{name}_workspace_bytes").argtypes = [ctypes.POINTER(Fp8Desc)]
            getattr(L, f"patdnn_fp8_{name}_workspace_bytes").restype = size
        L.patdnn_status_string.argtypes = [i32]
        L.patdnn_status_string.restype = ctypes.c_char_p
        L.patdnn_last_error.argtypes = []
        L.patdnn_last_error.restype = ctypes.c_char_p
        for name in EXPORTS:
            if getattr(L, name).restype is ctypes.c_int:
                getattr(L, name).restype = ctypes.c_int32
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != PATDNN_OK:
        raise PatdnnError(status, (lib().patdnn_last_error() or b"").decode() or
                          lib().patdnn_status_string(status).decode())


def _host(a: Optional[np.ndarray], dtype) -> Tuple[Optional[np.ndarray], Optional[int]]:
    if a is None:
        return None, None
    a = np.ascontiguousarray(a, dtype=dtype)
    return a, a.ctypes.data


def _devptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    if not t.is_contiguous():
        raise ValueError("contiguous tensor expected")
    return t.data_ptr()


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        import torch
        if torch.cuda.is_initialized():
            # the current stream's handle without a Stream object around it (0.2 us, 2.7 with one: a third of a small
            # layer's call)
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) or None
        return torch.cuda.current_stream().cuda_stream or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


# ---------------------------------------------------------------------------
# functions named after the C entry points
# ---------------------------------------------------------------------------

def patdnn_mine_patterns(dense_weights, k: int) -> np.ndarray:
    """The k most frequent natural patterns of [c_out][kpf][3][3] weights (uint16 masks)."""
    w, wp = _host(dense_weights, np.float32)
    masks = np.zeros(k, np.uint16)
    found = ctypes.c_int32()
    _check(lib().patdnn_mine_patterns(wp, w.shape[0], w.shape[1], k, masks.ctypes.data, ctypes.byref(found)))
    return masks[:found.value]


def patdnn_project_patterns(dense_weights, pattern_masks):
    """-> (pattern_ids uint8 [c_out][kpf], projected fp32 weights)"""
    w, wp = _host(dense_weights, np.float32)
    pm, pp = _host(pattern_masks, np.uint16)
    ids = np.zeros(w.shape[:2], np.uint8)
    proj = np.empty_like(w)
    _check(lib().patdnn_project_patterns(wp, w.shape[0], w.shape[1], pp, len(pm), ids.ctypes.data,
                                         proj.ctypes.data))
    return ids, proj


def patdnn_project_connectivity(dense_weights, alpha: int) -> np.ndarray:
    """-> kernel_mask uint8 [c_out][kpf] keeping the alpha kernels of largest L2 norm"""
    w, wp = _host(dense_weights, np.float32)
    mask = np.zeros(w.shape[:2], np.uint8)
    _check(lib().patdnn_project_connectivity(wp, w.shape[0], w.shape[1], int(alpha), mask.ctypes.data))
    return mask


def patdnn_encode(dense_weights, pattern_ids, kernel_mask, pattern_masks, *, stride=1, pad=1,
                  groups=1, flags=0) -> int:
    """-> handle (int).  Host arrays as in the header; ``dense_weights`` is OIHW."""
    w, wp = _host(dense_weights, np.float32)
    if w.ndim != 4 or w.shape[2:] != (3, 3):
        raise ValueError("dense_weights must be [c_out][c_in/groups][3][3]")
    c_out, kpf = int(w.shape[0]), int(w.shape[1])
    c_in = kpf * groups
    ids, ip = _host(pattern_ids, np.uint8)
    km, kp = _host(kernel_mask, np.uint8)
    pm, pp = _host(pattern_masks, np.uint16)
    for a in (ids, km):
        if a is not None and a.shape != (c_out, kpf):
            raise ValueError("pattern_ids / kernel_mask must be [c_out][c_in/groups]")
    d = LayerDesc(c_out, c_in, groups, stride, pad, 0 if pm is None else len(pm), pp, flags)
    h = ctypes.c_void_p()
    _check(lib().patdnn_encode(ctypes.byref(d), wp, ip, kp, ctypes.byref(h)))
    return h.value


_Shape = ctypes.c_int32 * 4


def patdnn_output_shape(handle: int, n: int, h_in: int, w_in: int):
    out = _Shape()
    _check(lib().patdnn_output_shape(handle, n, h_in, w_in, ctypes.byref(out)))
    return tuple(out)


def patdnn_conv2d(handle: int, x, bias=None, out=None, *, fuse_relu=False, stream=None):
    """x: device tensor NCHW fp32.  Returns ``out`` (allocated with torch if None)."""
    import torch
    if x.dtype != torch.float32 or x.dim() != 4:
        raise ValueError("input must be a 4-d float32 tensor")
    n, _, h_in, w_in = x.shape
    shape = patdnn_output_shape(handle, n, h_in, w_in)
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=x.device)
    elif tuple(out.shape) != shape or out.dtype != torch.float32:
        raise ValueError(f"output must be float32 {shape}")
    if bias is not None and (bias.dtype != torch.float32 or bias.numel() != shape[1]):
        raise ValueError("bias must be float32 [c_out]")
    _check(lib().patdnn_conv2d(handle, _devptr(x), n, h_in, w_in, _devptr(bias), _devptr(out),
                               int(bool(fuse_relu)), _stream_ptr(stream)))
    return out


def patdnn_workspace_floats(handle: int, n: int, h_in: int, w_in: int) -> int:
    return int(lib().patdnn_workspace_floats(handle, n, h_in, w_in))


def patdnn_conv2d_ws(handle: int, x, bias=None, out=None, *, workspace=None, fuse_relu=False, pool=False,
                     stream=None):
    """patdnn_conv2d / patdnn_conv2d_pool with a caller-owned workspace (a float32 device tensor)
    for the partial sums of a configuration that splits the input channels."""
    import torch
    if x.dtype != torch.float32 or x.dim() != 4:
        raise ValueError("input must be a 4-d float32 tensor")
    n, _, h_in, w_in = x.shape
    full = patdnn_output_shape(handle, n, h_in, w_in)
    shape = (full[0], full[1], full[2] // 2, full[3] // 2) if pool else full
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=x.device)
    elif tuple(out.shape) != shape or out.dtype != torch.float32:
        raise ValueError(f"output must be float32 {shape}")
    if bias is not None and (bias.dtype != torch.float32 or bias.numel() != shape[1]):
        raise ValueError("bias must be float32 [c_out]")
    if workspace is not None and (workspace.dtype != torch.float32 or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous float32 tensor")
    _check(lib().patdnn_conv2d_ws(handle, _devptr(x), n, h_in, w_in, _devptr(bias), _devptr(out),
                                  int(bool(fuse_relu)), int(bool(pool)), _devptr(workspace),
                                  0 if workspace is None else workspace.numel(), _stream_ptr(stream)))
    return out


def patdnn_conv2d_f16(handle: int, x, bias=None, out=None, *, fuse_relu=False, stream=None):
    """x, out: float16 device tensors (half-precision storage); bias float32."""
    import torch
    if x.dtype != torch.float16 or x.dim() != 4:
        raise ValueError("input must be a 4-d float16 tensor")
    n, _, h_in, w_in = x.shape
    shape = patdnn_output_shape(handle, n, h_in, w_in)
    if out is None:
        out = torch.empty(shape, dtype=torch.float16, device=x.device)
    elif tuple(out.shape) != shape or out.dtype != torch.float16:
        raise ValueError(f"output must be float16 {shape}")
    if bias is not None and (bias.dtype != torch.float32 or bias.numel() != shape[1]):
        raise ValueError("bias must be float32 [c_out]")
    _check(lib().patdnn_conv2d_f16(handle, _devptr(x), n, h_in, w_in, _devptr(bias), _devptr(out),
                                   int(bool(fuse_relu)), _stream_ptr(stream)))
    return out


def patdnn_conv2d_pool(handle: int, x, bias=None, out=None, *, stream=None):
    """conv + bias + ReLU + 2x2 max pooling, fused.  Returns ``out`` [n][c_out][h_out/2][w_out/2]."""
    import torch
    if x.dtype != torch.float32 or x.dim() != 4:
        raise ValueError("input must be a 4-d float32 tensor")
    n, _, h_in, w_in = x.shape
    full = patdnn_output_shape(handle, n, h_in, w_in)
    shape = (full[0], full[1], full[2] // 2, full[3] // 2)
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=x.device)
    elif tuple(out.shape) != shape or out.dtype != torch.float32:
        raise ValueError(f"output must be float32 {shape}")
    _check(lib().patdnn_conv2d_pool(handle, _devptr(x), n, h_in, w_in, _devptr(bias), _devptr(out),
                                    _stream_ptr(stream)))
    return out


class Stack:
    """patdnn_stack_*: layers run back to back; ``layers`` = [(Layer, bias tensor or None, relu, pool2)]."""

    def __init__(self, layers, n: int, h_in: int, w_in: int):
        self._keep = list(layers)               # handles and bias tensors must outlive the stack
        arr = (StackLayer * len(layers))()
        for i, (L, bias, relu, pool) in enumerate(layers):
            arr[i] = StackLayer(L.handle, _devptr(bias), int(bool(relu)), int(bool(pool)))
        h = ctypes.c_void_p()
        _check(lib().patdnn_stack_create(arr, len(layers), n, h_in, w_in, ctypes.byref(h)))
        self.handle = h.value

    def output_shape(self):
        out = (ctypes.c_int32 * 4)()
        _check(lib().patdnn_stack_output_shape(self.handle, ctypes.byref(out)))
        return tuple(out)

    def run(self, x, out=None, *, graph=False, stream=None):
        import torch
        if out is None:
            out = torch.empty(self.output_shape(), dtype=torch.float32, device=x.device)
        _check(lib().patdnn_stack_run(self.handle, _devptr(x), _devptr(out), int(bool(graph)),
                                      _stream_ptr(stream)))
        return out

    def run_static(self, x, out, *, stream=None):
        """patdnn_stack_run_static: the library's built-in buffer instead of the stack's own."""
        _check(lib().patdnn_stack_run_static(self.handle, _devptr(x), _devptr(out), _stream_ptr(stream)))
        return out

    def close(self):
        if self.handle:
            lib().patdnn_stack_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def patdnn_layout_stats(handle: int) -> dict:
    s = Stats()
    _check(lib().patdnn_layout_stats(handle, ctypes.byref(s)))
    return {k: getattr(s, k) for k, _ in Stats._fields_}


def patdnn_decode(handle: int, c_out: int, kernels_per_filter: int):
    w = np.empty((c_out, kernels_per_filter, 3, 3), dtype=np.float32)
    ids = np.empty((c_out, kernels_per_filter), dtype=np.uint8)
    km = np.empty((c_out, kernels_per_filter), dtype=np.uint8)
    _check(lib().patdnn_decode(handle, w.ctypes.data, ids.ctypes.data, km.ctypes.data))
    return w, ids, km


def patdnn_export_fkw(handle: int, c_out: int) -> dict:
    st = patdnn_layout_stats(handle)
    kept, taps, P = st["kept_kernels"], st["taps"], st["num_patterns"]
    out = {"offset": np.empty(c_out + 1, np.int32), "reorder": np.empty(c_out, np.int32),
           "index": np.empty(kept, np.int32), "stride": np.empty((c_out, P + 1), np.int32),
           "weight": np.empty((kept, taps), np.float32)}
    _check(lib().patdnn_export_fkw(handle, *(out[k].ctypes.data for k in
                                             ("offset", "reorder", "index", "stride", "weight"))))
    return out


def patdnn_export_csr(handle: int, c_out: int) -> dict:
    nnz = ctypes.c_int64()
    _check(lib().patdnn_export_csr(handle, ctypes.byref(nnz), None, None, None))
    out = {"row_ptr": np.empty(c_out + 1, np.int32), "col": np.empty(nnz.value, np.int32),
           "val": np.empty(nnz.value, np.float32)}
    _check(lib().patdnn_export_csr(handle, None, out["row_ptr"].ctypes.data, out["col"].ctypes.data,
                                   out["val"].ctypes.data))
    return out


def patdnn_num_variants() -> int:
    return int(lib().patdnn_num_variants())


def patdnn_variant_name(v: int) -> Optional[str]:
    s = lib().patdnn_variant_name(v)
    return None if s is None else s.decode()


def patdnn_set_config(handle: int, variant: int, ck: int = 0, waves: int = 0, ksplit: int = 0) -> None:
    c = Config(variant, ck, waves, ksplit)
    _check(lib().patdnn_set_config(handle, ctypes.byref(c)))


def patdnn_get_config(handle: int) -> dict:
    c = Config()
    _check(lib().patdnn_get_config(handle, ctypes.byref(c)))
    return {"variant": c.variant, "ck": c.ck, "waves": c.waves, "ksplit": c.ksplit}


def patdnn_tune(handle: int, x, bias, out, *, workspace=None, stream=None) -> float:
    """Times every applicable configuration on the given buffers (split configurations with the
    workspace, a float32 device tensor, if one is given); returns best microseconds."""
    n, _, h_in, w_in = x.shape
    best = ctypes.c_float()
    if workspace is None:
        _check(lib().patdnn_tune(handle, _devptr(x), n, h_in, w_in, _devptr(bias), _devptr(out),
                                 _stream_ptr(stream), ctypes.byref(best)))
    else:
        _check(lib().patdnn_tune_ws(handle, _devptr(x), n, h_in, w_in, _devptr(bias), _devptr(out),
                                    _devptr(workspace), workspace.numel(), _stream_ptr(stream), ctypes.byref(best)))
    return float(best.value)


def patdnn_tiled_info(handle: int, variant: int, ck: int = 0) -> dict:
    t = TiledInfo()
    _check(lib().patdnn_tiled_info(handle, variant, ck, ctypes.byref(t)))
    return {k: getattr(t, k) for k, _ in TiledInfo._fields_}


def patdnn_export_tiled(handle: int, variant: int, ck: int = 0) -> dict:
    """The filter-group layout of a tiled sparse variant: info fields plus the arrays."""
    info = patdnn_tiled_info(handle, variant, ck)
    out = dict(info)
    out["slot_channel"] = np.empty((info["num_groups"], info["G"]), np.int32)
    out["chunk_ptr"] = np.empty((info["num_groups"], info["num_chunks"]), np.uint32)
    out["steps"] = np.empty((info["num_steps"], 24), np.uint32)
    _check(lib().patdnn_export_tiled(handle, variant, ck, out["slot_channel"].ctypes.data,
                                     out["chunk_ptr"].ctypes.data, out["steps"].ctypes.data))
    return out


def patdnn_selftest() -> None:
    """Raises PatdnnError (EUNSUPPORTED) if the device fails the scalar-relative-move check."""
    _check(lib().patdnn_selftest())


def patdnn_destroy(handle: Optional[int]) -> None:
    if handle:
        lib().patdnn_destroy(handle)


# ---------------------------------------------------------------------------
# what stands between and behind the convolutions: order of channels, group norm, MXFP4
# ---------------------------------------------------------------------------

_modules = {}
_types = {}


def _torch():
    if not _modules:
        import torch
        _modules["torch"] = torch
        _types.update({torch.float32: PATDNN_F32, torch.float16: PATDNN_F16, torch.bfloat16: PATDNN_BF16})
    return _modules["torch"]


def _type(dtype) -> int:
    kind = _types.get(dtype)
    if kind is None:
        _torch()
        kind = _types.get(dtype)
        if kind is None:
            raise ValueError(f"float32, float16 or bfloat16 expected, not {dtype}")
    return kind


def _act(act: str) -> int:
    try:
        return ACTIVATIONS[act]
    except KeyError:
        raise ValueError(f"act must be one of {', '.join(ACTIVATIONS)}") from None


def _new(shape, dtype, like, stream):
    """A tensor that the call's stream owns: what is allocated while another one is current may not be in use there
    any more before it is here, nor free here before it is there."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    torch = _torch()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream(like.device)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _float_vector(t, count: int, name: str) -> Optional[int]:
    if t is None:
        return None
    if _types.get(t.dtype) != PATDNN_F32 or t.numel() != count:
        raise ValueError(f"{name} must be float32 with {count} elements")
    if not (t.is_cuda and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous device tensor")
    return t.data_ptr()


def _channels_last_layout(t, name: str):
    """[n, ..., c] -> (n, pixels, c, image stride, pixel stride)."""
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    shape, strides = t.shape, t.stride()
    dims = len(shape)
    if dims < 3:
        raise ValueError(f"{name} must be [n, ..., channels]")
    c = shape[-1]
    if dims == 4 and strides[-1] == 1 and strides[1] == strides[2] * shape[2]:       # most calls'
        return shape[0], shape[1] * shape[2], c, strides[0], strides[2]
    if c > 1 and strides[-1] != 1 and t.numel():
        raise ValueError(f"the channels of {name} must be adjacent")
    pixel, pixels = strides[-2], shape[-2]
    for i in range(dims - 3, 0, -1):
        if pixels == 1:
            pixel = strides[i]
        elif shape[i] > 1 and strides[i] != pixel * pixels and t.numel():
            raise ValueError(f"the pixels of {name} must be evenly spaced")
        pixels *= shape[i]
    return shape[0], pixels, c, strides[0], pixel


def patdnn_channels_last(x, out=None, *, dtype=None, stream=None):
    """x [n, c, h, w], dense -> [n, h, w, c] of type ``dtype`` (x's if None); ``out`` may be a slice of the channels of a wider tensor."""
    if x.dim() != 4:
        raise ValueError("input must be a 4-d tensor")
    n, c, h, w = x.shape
    if out is None:
        out = _new((n, h, w, c), dtype or x.dtype, x, stream)
    elif tuple(out.shape) != (n, h, w, c) or (dtype and out.dtype != dtype):
        raise ValueError(f"output must be {(n, h, w, c)}, of type dtype if that is given")
    _, _, _, image, pixel = _channels_last_layout(out, "output")
    _check(lib().patdnn_channels_last(_devptr(x), _type(x.dtype), n, c, h * w, out.data_ptr(), _type(out.dtype), image, pixel,
                                      _stream_ptr(stream)))
    return out


def patdnn_channels_first(x, out=None, *, dtype=None, stream=None):
    """x [n, h, w, c], maybe a slice of the channels of a wider tensor -> [n, c, h, w], dense, of type ``dtype`` (x's if None)."""
    if x.dim() != 4:
        raise ValueError("input must be a 4-d tensor")
    n, h, w, c = x.shape
    _, _, _, image, pixel = _channels_last_layout(x, "input")
    if out is None:
        out = _new((n, c, h, w), dtype or x.dtype, x, stream)
    elif tuple(out.shape) != (n, c, h, w) or (dtype and out.dtype != dtype):
        raise ValueError(f"output must be {(n, c, h, w)}, of type dtype if that is given")
    _check(lib().patdnn_channels_first(x.data_ptr(), _type(x.dtype), image, pixel, n, c, h * w, _devptr(out), _type(out.dtype),
                                       _stream_ptr(stream)))
    return out


def _norm_room(desc, backward: int, shape, first, second, workspace, like, stream):
    """The two small float32 outputs and the workspace of a group norm call, those that are not given allocated (together where the workspace
    is small: an allocation costs the call 1.5 us, a third of a launch) -> (first, second, workspace's pointer, its floats, its owner).  The owner
    must be held until the call has returned: on the stream of the launches, freed memory is the next allocation's, also another thread's."""
    torch = _torch()
    if first is None and second is None and workspace is None:
        floats = lib().patdnn_group_norm_workspace_floats(desc, backward)
        if floats <= 1 << 16:
            count, strides = (shape[0], (1,)) if len(shape) == 1 else (shape[0] * shape[1], (shape[1], 1))
            room = _new((floats + 2 * count,), torch.float32, like, stream)
            return room.as_strided(shape, strides, 0), room.as_strided(shape, strides, count), room.data_ptr() + 8 * count, floats, room
        workspace = _new((floats,), torch.float32, like, stream)
    if first is None:
        first = _new(shape, torch.float32, like, stream)
    if second is None:
        second = _new(shape, torch.float32, like, stream)
    if workspace is None:
        workspace = _new((lib().patdnn_group_norm_workspace_floats(desc, backward),), torch.float32, like, stream)
    elif workspace.dtype != torch.float32:
        raise ValueError("workspace must be a float32 tensor")
    return first, second, _devptr(workspace), workspace.numel(), workspace


def patdnn_group_norm(x, groups: int, gamma=None, beta=None, out=None, *, eps=1e-5, act="none", mean=None, rstd=None, workspace=None,
                      stream=None):
    """x [n, ..., c] channels last -> (act(group norm) like x, mean, rstd float32 [n, groups]).  gamma, beta: float32 [c] or None.
    x and ``out`` may be slices of the channels of wider tensors, also of one.  Where the call allocates all of mean, rstd and its workspace, mean and rstd
    are views of one allocation, which lives as long as they do (up to 256 KB more than they hold)."""
    n, pixels, c, x_image, x_pixel = _channels_last_layout(x, "x")
    if out is None:
        out = _new(tuple(x.shape), x.dtype, x, stream)
    elif out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("output must have the shape and type of x")
    _, _, _, y_image, y_pixel = _channels_last_layout(out, "output")
    desc = ctypes.byref(NormDesc(n, pixels, c, groups, _type(x.dtype), _act(act), eps, x_image, x_pixel, y_image, y_pixel, 0, 0))
    mean, rstd, work, floats, owner = _norm_room(desc, 0, (n, max(groups, 0)), mean, rstd, workspace, x, stream)
    _check(lib().patdnn_group_norm(desc, x.data_ptr(), _float_vector(gamma, c, "gamma"), _float_vector(beta, c, "beta"),
                                   out.data_ptr(), _float_vector(mean, n * groups, "mean"), _float_vector(rstd, n * groups, "rstd"),
                                   work, floats, _stream_ptr(stream)))
    del owner
    return out, mean, rstd


def patdnn_group_norm_backward(dy, x, mean, rstd, groups: int, gamma=None, beta=None, out=None, *, act="none", dgamma=None, dbeta=None,
                               workspace=None, stream=None):
    """Gradients of patdnn_group_norm: (dx like x, dgamma, dbeta float32 [c]) from dy, x and the forward call's mean and rstd."""
    n, pixels, c, x_image, x_pixel = _channels_last_layout(x, "x")
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must have the shape and type of x")
    _, _, _, dy_image, dy_pixel = _channels_last_layout(dy, "dy")
    if out is None:
        out = _new(tuple(x.shape), x.dtype, x, stream)
    elif out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("output must have the shape and type of x")
    _, _, _, y_image, y_pixel = _channels_last_layout(out, "output")
    desc = ctypes.byref(NormDesc(n, pixels, c, groups, _type(x.dtype), _act(act), 0.0, x_image, x_pixel, y_image, y_pixel, dy_image, dy_pixel))
    dgamma, dbeta, work, floats, owner = _norm_room(desc, 1, (c,), dgamma, dbeta, workspace, x, stream)
    _check(lib().patdnn_group_norm_backward(
        desc, dy.data_ptr(), x.data_ptr(), _float_vector(mean, n * groups, "mean"), _float_vector(rstd, n * groups, "rstd"),
        _float_vector(gamma, c, "gamma"), _float_vector(beta, c, "beta"), out.data_ptr(), _float_vector(dgamma, c, "dgamma"),
        _float_vector(dbeta, c, "dbeta"), work, floats, _stream_ptr(stream)))
    del owner
    return out, dgamma, dbeta


def _rows(t, name: str) -> int:
    """Elements between the rows of a 2-d tensor whose rows' values are adjacent."""
    if t.dim() != 2:
        raise ValueError(f"{name} must be a 2-d tensor")
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    row, step = t.stride()
    if step != 1 and t.shape[1] > 1 and t.numel():
        raise ValueError(f"the values of a row of {name} must be adjacent")
    return row


def _codes(codes, scales, rows: int, cols: int):
    torch = _torch()
    pieces = -(-cols // 128)
    if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.shape != (rows, pieces * 64) or scales.shape != (rows, pieces * 4):
        raise ValueError(f"codes and scales must be uint8 {(rows, pieces * 64)} and {(rows, pieces * 4)}")
    return _devptr(codes), _devptr(scales)


def patdnn_mxfp4_quantize(x, codes=None, scales=None, *, stream=None):
    """x [rows, cols] -> (codes uint8 [rows, ceil(cols/128)*64], scales uint8 [rows, ceil(cols/128)*4])."""
    torch = _torch()
    row = _rows(x, "x")
    rows, cols = x.shape
    pieces = -(-cols // 128)
    if codes is None:
        codes = _new((rows, pieces * 64), torch.uint8, x, stream)
    if scales is None:
        scales = _new((rows, pieces * 4), torch.uint8, x, stream)
    cp, sp = _codes(codes, scales, rows, cols)
    _check(lib().patdnn_mxfp4_quantize(x.data_ptr(), _type(x.dtype), rows, cols, row, cp, sp, _stream_ptr(stream)))
    return codes, scales


def patdnn_mxfp4_dequantize(codes, scales, cols: int, out=None, *, dtype=None, stream=None):
    """The values [rows, cols] that codes and scales stand for, float32 unless ``out`` or ``dtype`` says otherwise."""
    torch = _torch()
    rows = codes.shape[0]
    cp, sp = _codes(codes, scales, rows, cols)
    if out is None:
        out = _new((rows, cols), dtype or torch.float32, codes, stream)
    elif tuple(out.shape) != (rows, cols) or (dtype and out.dtype != dtype):
        raise ValueError(f"output must be {(rows, cols)}, of type dtype if that is given")
    row = _rows(out, "output")
    _check(lib().patdnn_mxfp4_dequantize(cp, sp, rows, cols, out.data_ptr(), _type(out.dtype), row, _stream_ptr(stream)))
    return out


def patdnn_mxfp4_linear(x, w, w_scales, bias=None, out=None, *, x_scales=None, act="none", dtype=None, workspace=None, stream=None):
    """x [rows, in] times MXFP4 weights [out, in], plus bias (float32 [out]), activated.  x is float32 / float16 / bfloat16, or the codes
    of patdnn_mxfp4_quantize with ``x_scales``.  The result's type: ``out``'s, ``dtype``, or x's (float32 for codes)."""
    torch = _torch()
    row = _rows(x, "x")
    features = w.shape[0]
    if x_scales is None:
        rows, cols = x.shape
        kind, sp = _type(x.dtype), None
    else:
        rows, cols = x.shape[0], x.shape[1] * 2
        kind, row = PATDNN_MXFP4, 0
        _, sp = _codes(x, x_scales, rows, cols)
    wp, wsp = _codes(w, w_scales, features, cols)
    if out is None:
        out = _new((rows, features), dtype or (x.dtype if x_scales is None else torch.float32), x, stream)
    elif tuple(out.shape) != (rows, features) or (dtype and out.dtype != dtype):
        raise ValueError(f"output must be {(rows, features)}, of type dtype if that is given")
    desc = LinearDesc(rows, cols, features, kind, _type(out.dtype), _act(act), row, _rows(out, "output"))
    needs = lib().patdnn_mxfp4_linear_workspace_bytes(ctypes.byref(desc))
    if needs and workspace is None:
        workspace = _new((needs,), torch.uint8, x, stream)
    _check(lib().patdnn_mxfp4_linear(ctypes.byref(desc), x.data_ptr(), sp, wp, wsp, _float_vector(bias, features, "bias"), out.data_ptr(),
                                     _devptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                     _stream_ptr(stream)))
    return out


def patdnn_mxfp4_linear_workspace_bytes(rows: int, in_features: int, out_features: int, *, x_type: int, out_type: int) -> int:
    """Bytes of workspace for a call of patdnn_mxfp4_linear with dense rows."""
    desc = LinearDesc(rows, in_features, out_features, x_type, out_type, 0, in_features, out_features)
    return int(lib().patdnn_mxfp4_linear_workspace_bytes(ctypes.byref(desc)))


def patdnn_group_norm_workspace_floats(n: int, pixels: int, channels: int, groups: int, *, type: int = PATDNN_F32,
                                       backward: bool = False) -> int:
    """Floats of workspace for a call of patdnn_group_norm, or of its backward pass, on dense tensors."""
    image = pixels * channels
    desc = NormDesc(n, pixels, channels, groups, type, 0, 0.0, image, channels, image, channels, image, channels)
    return int(lib().patdnn_group_norm_workspace_floats(ctypes.byref(desc), int(bool(backward))))


# ---------------------------------------------------------------------------
# the feed-forward block in fp8: norm of rows, codes, linear layer, gated projections
# ---------------------------------------------------------------------------

def _call(device: int, stream, f, *args) -> None:
    """f(*args, stream) with this device current: without a stream its current one."""
    torch = _modules["torch"]
    if device == torch._C._cuda_getDevice():
        status = f(*args, (torch._C._cuda_getCurrentRawStream(device) or None) if stream is None else _stream_ptr(stream))
    else:
        with torch.cuda.device(device):
            status = f(*args, _stream_ptr(stream))
    if status:
        _check(status)


def _together(like, *tensors) -> int:
    """The device of all these tensors."""
    if not _modules:
        _torch()
    if not like.is_cuda:
        raise ValueError("device tensor expected")
    device = like.get_device()
    for t in tensors:
        if t is not None and (not t.is_cuda or t.get_device() != device):
            raise ValueError(f"all tensors must be on one device: {t.device} and {like.device}")
    return device


def _typed_rows(t, shape, dtype, name: str) -> int:
    """The row stride of a 2-d tensor that has to have this shape and type."""
    if t.shape != shape or t.dtype != dtype:
        raise ValueError(f"{name} must be {tuple(shape)} of type {dtype}")
    return _rows(t, name)


def _byte_codes(t, name: str):
    """Codes, as bytes or as torch's type of them."""
    torch = _modules["torch"]
    if t.dtype != torch.uint8 and t.dtype != torch.float8_e4m3fn:
        raise ValueError(f"{name} must be uint8 or float8_e4m3fn")
    shape = t.shape
    if len(shape) != 2 or shape[1] == 0 or shape[1] % 128:
        raise ValueError(f"{name} must be [rows, whole pieces of 128]")
    return _devptr(t)


def _byte_scales(t, rows: int, pieces: int, name: str, blocks=None):
    """Scales of codes [rows, pieces * 128] -> (their pointer, how they are laid out; of one row both layouts are the same)."""
    torch = _modules["torch"]
    if t.dtype != torch.uint8 and t.dtype != torch.float8_e8m0fnu:
        raise ValueError(f"{name} must be uint8 or float8_e8m0fnu")
    shape = t.shape
    if len(shape) == 2 and shape[1] == pieces:
        if shape[0] == rows and blocks != 1:
            return _devptr(t), 0
        if shape[0] == -(-rows // 128) and blocks != 0:
            return _devptr(t), 1
    raise ValueError(f"{name} must be {(rows, pieces)}" + ("" if blocks == 0 else f" or {(-(-rows // 128), pieces)}"))


def _new_codes(out, scales, rows: int, pieces: int, like, stream, name="output"):
    """Codes with blocks along the rows, and their scales, as given or allocated -> (codes, scales, their pointers)."""
    if out is None:
        out = _new((rows, pieces * 128), _modules["torch"].uint8, like, stream)
        op = out.data_ptr()
    else:
        if tuple(out.shape) != (rows, pieces * 128):
            raise ValueError(f"{name} must be {(rows, pieces * 128)}")
        op = _byte_codes(out, name) if pieces else _devptr(out)        # (of the transpose of no rows)
    if scales is None:
        scales = _new((rows, pieces), _modules["torch"].uint8, like, stream)
        return out, scales, op, scales.data_ptr()
    return out, scales, op, _byte_scales(scales, rows, pieces, "scales", 0)[0]


def patdnn_fp8_quantize(x, codes=None, scales=None, *, blocks="rows", transposed=False, stream=None):
    """x [rows, cols] -> (codes uint8 [rows, ceil(cols/128)*128], scales uint8): e4m3 with a power of two for each 1 x 128 (``blocks`` "rows", scales
    [rows, ceil(cols/128)]) or 128 x 128 values ("squares", [ceil(rows/128), ceil(cols/128)]).  ``transposed``: those of x's transpose."""
    torch = _torch()
    try:
        kind = FP8_BLOCKS[blocks]
    except KeyError:
        raise ValueError(f"blocks must be one of {', '.join(FP8_BLOCKS)}") from None
    device = _together(x, codes, scales)
    row = _rows(x, "x")
    rows, cols = x.shape
    r, c = (cols, rows) if transposed else (rows, cols)
    pieces = -(-c // 128)
    if not kind:
        codes, scales, cp, sp = _new_codes(codes, scales, r, pieces, x, stream, "codes")
    else:
        if codes is None:
            codes = _new((r, pieces * 128), torch.uint8, x, stream)
        elif tuple(codes.shape) != (r, pieces * 128):
            raise ValueError(f"codes must be {(r, pieces * 128)}")
        if scales is None:
            scales = _new((-(-r // 128), pieces), torch.uint8, x, stream)
        cp = _byte_codes(codes, "codes") if codes.numel() else _devptr(codes)
        sp, _ = _byte_scales(scales, r, pieces, "scales", kind if r != 1 else None)
    _call(device, stream, lib().patdnn_fp8_quantize, x.data_ptr(), _type(x.dtype), rows, cols, row, kind, 1 if transposed else 0, cp, sp)
    return codes, scales


def patdnn_fp8_dequantize(codes, scales, cols: int, out=None, *, dtype=None, stream=None):
    """The values [rows, cols] that codes and scales (of either layout) stand for, float32 unless ``out`` or ``dtype`` says otherwise."""
    torch = _torch()
    device = _together(codes, scales, out)
    cp = _byte_codes(codes, "codes")
    rows, pieces = codes.shape[0], codes.shape[1] // 128
    if not 0 < cols <= pieces * 128 or cols <= (pieces - 1) * 128:
        raise ValueError(f"{cols} columns are not {pieces} pieces of 128")
    sp, kind = _byte_scales(scales, rows, pieces, "scales")
    if out is None:
        out, row = _new((rows, cols), dtype or torch.float32, codes, stream), cols
    else:
        if tuple(out.shape) != (rows, cols) or (dtype and out.dtype != dtype):
            raise ValueError(f"output must be {(rows, cols)}, of type dtype if that is given")
        row = _rows(out, "output")
    _call(device, stream, lib().patdnn_fp8_dequantize, cp, sp, rows, cols, kind, out.data_ptr(), _type(out.dtype), row)
    return out


def _row_floats(t, count: int, name: str, like, stream):
    if t is None:
        t = _new((count,), _modules["torch"].float32, like, stream)
        return t, t.data_ptr()
    return t, _float_vector(t, count, name)


def patdnn_rms_norm(x, gamma=None, out=None, *, residual=None, sum=None, eps=1e-6, fp8=False, dtype=None, scales=None, rstd=None, stream=None):
    """Root-mean-square norm of the rows of x [rows, cols] (+ ``residual``) -> (out, scales, sum, rstd).

    gamma: float32 [cols] or None.  out: x's type, ``dtype``'s, or (``fp8``) the codes of patdnn_fp8_quantize, with their scales (None otherwise).
    sum: x + residual in x's type, x itself without a residual; ``sum=residual`` adds in place.  rstd: float32 [rows], for the backward call."""
    device = _together(x, gamma, out, residual, sum, scales, rstd)
    x_row = _rows(x, "x")
    shape, x_type = x.shape, x.dtype
    rows, cols = shape
    residual_row = sum_row = 0
    rp = total = None
    if residual is not None:
        residual_row, rp = _typed_rows(residual, shape, x_type, "residual"), residual.data_ptr()
        if sum is None:
            sum = _new((rows, cols), x_type, x, stream)
    if sum is not None:
        sum_row, total = _typed_rows(sum, shape, x_type, "sum"), sum.data_ptr()
    if fp8:
        if dtype is not None:
            raise ValueError("dtype is for results that are no codes")
        out, scales, yp, sp = _new_codes(out, scales, rows, -(-cols // 128), x, stream)
        y_type, y_row = PATDNN_FP8, 0
    else:
        if scales is not None:
            raise ValueError("scales are for codes")
        if out is None:
            out = _new((rows, cols), dtype or x_type, x, stream)
        elif out.shape != shape or (dtype and out.dtype != dtype):
            raise ValueError("output must have the shape of x, and type dtype if that is given")
        y_type, y_row, yp, sp = _type(out.dtype), _rows(out, "output"), out.data_ptr(), None
    rstd, root = _row_floats(rstd, rows, "rstd", x, stream)
    desc = RmsDesc(rows, cols, _type(x_type), y_type, eps, x_row, residual_row, sum_row, y_row)
    _call(device, stream, lib().patdnn_rms_norm, ctypes.byref(desc), x.data_ptr(), rp, _float_vector(gamma, cols, "gamma"), total, yp, sp, root)
    return out, scales, x if sum is None else sum, rstd


def patdnn_rms_norm_backward(dy, sum, rstd, gamma=None, out=None, *, dsum=None, dgamma=None, workspace=None, stream=None):
    """Gradients of patdnn_rms_norm: (dx like sum, dgamma float32 [cols]) from dy (of any type), the forward call's sum and rstd.  ``dsum``: the gradient that
    arrives along the residual stream, added to dx; ``out=dsum`` adds in place.  ``dgamma=False``: None in its place, which saves the call its workspace and second launch."""
    wanted = dgamma is not False
    if not wanted:
        dgamma = workspace = None
    device = _together(sum, dy, rstd, gamma, out, dsum, dgamma, workspace)
    torch = _modules["torch"]
    s_row = _rows(sum, "sum")
    rows, cols = sum.shape
    if dy.shape != sum.shape:
        raise ValueError("dy must have the shape of sum")
    if out is None:
        out = _new((rows, cols), sum.dtype, sum, stream)
    desc = RmsDesc(rows, cols, _type(sum.dtype), _type(dy.dtype), 0.0, s_row, 0 if dsum is None else _typed_rows(dsum, sum.shape, sum.dtype, "dsum"),
                   _typed_rows(out, sum.shape, sum.dtype, "output"), _rows(dy, "dy"))
    gp, wp, floats = None, None, 0
    if wanted:
        dgamma, gp = _row_floats(dgamma, cols, "dgamma", sum, stream)
        if workspace is None:
            workspace = _new((lib().patdnn_rms_norm_workspace_floats(ctypes.byref(desc)),), torch.float32, sum, stream)
        elif workspace.dtype != torch.float32:
            raise ValueError("workspace must be a float32 tensor")
        wp, floats = _devptr(workspace), workspace.numel()
    _call(device, stream, lib().patdnn_rms_norm_backward, ctypes.byref(desc), dy.data_ptr(), None if dsum is None else dsum.data_ptr(), sum.data_ptr(),
          _float_vector(rstd, rows, "rstd"), _float_vector(gamma, cols, "gamma"), out.data_ptr(), gp, wp, floats)
    return out, dgamma


def _fp8_operands(x, x_scales, weights):
    """-> (rows, in_features, out_features, layout of the weights' scales, the pointers)"""
    xp = _byte_codes(x, "x")
    rows, cols = x.shape
    pieces = cols // 128
    sp, _ = _byte_scales(x_scales, rows, pieces, "x_scales", 0)
    pointers, features, blocks = [xp, sp], None, None
    for w, s in weights:
        wp = _byte_codes(w, "weights")
        if w.shape[1] != cols:
            raise ValueError("the codes of x and of the weights must have rows of one length")
        if features is None:
            features = w.shape[0]
        elif w.shape[0] != features:
            raise ValueError("both projections must have the same number of outputs")
        p, kind = _byte_scales(s, features, pieces, "scales of the weights", blocks)
        blocks = kind
        pointers += [wp, p]
    return rows, cols, features, blocks, pointers


def _byte_workspace(sizes, desc, workspace, like, stream):
    """(workspace, its pointer, its bytes); allocated if it is needed and not given."""
    if workspace is None:
        needs = sizes(ctypes.byref(desc))
        if not needs:
            return None, None, 0
        workspace = _new((needs,), _torch().uint8, like, stream)
    return workspace, _devptr(workspace), workspace.numel() * workspace.element_size()


def patdnn_fp8_linear(x, x_scales, w, w_scales, bias=None, out=None, *, act="none", dtype=None, workspace=None, stream=None):
    """fp8 codes x [rows, in] times codes w [out, in], plus bias (float32 [out]), activated.  The weights' scales are of rows or of squares, as their shape
    says.  The result's type: ``out``'s or ``dtype``, float32 otherwise."""
    device = _together(x, x_scales, w, w_scales, bias, out, workspace)
    torch = _modules["torch"]
    rows, cols, features, blocks, pointers = _fp8_operands(x, x_scales, ((w, w_scales),))
    if out is None:
        out = _new((rows, features), dtype or torch.float32, x, stream)
    elif tuple(out.shape) != (rows, features) or (dtype and out.dtype != dtype):
        raise ValueError(f"output must be {(rows, features)}, of type dtype if that is given")
    desc = Fp8Desc(rows, cols, features, blocks, _type(out.dtype), _act(act), 0, _rows(out, "output"), 0)
    workspace, wp, size = _byte_workspace(lib().patdnn_fp8_linear_workspace_bytes, desc, workspace, x, stream)
    _call(device, stream, lib().patdnn_fp8_linear, ctypes.byref(desc), *pointers, _float_vector(bias, features, "bias"), out.data_ptr(), wp, size)
    return out


def patdnn_fp8_gated(x, x_scales, gate, gate_scales, up, up_scales, out=None, *, act="silu", fp8=False, dtype=None, scales=None, workspace=None,
                     stream=None):
    """act(x gate) * (x up) for fp8 codes x [rows, in] and gate, up [out, in]: values (of type ``out``'s or ``dtype``, float32 otherwise), or with
    ``fp8`` (codes, scales) of patdnn_fp8_quantize."""
    device = _together(x, x_scales, gate, gate_scales, up, up_scales, out, scales, workspace)
    rows, cols, features, blocks, pointers = _fp8_operands(x, x_scales, ((gate, gate_scales), (up, up_scales)))
    if fp8:
        if dtype is not None:
            raise ValueError("dtype is for results that are no codes")
        out, scales, op, sp = _new_codes(out, scales, rows, -(-features // 128), x, stream)
        kind, row = PATDNN_FP8, 0
    else:
        if scales is not None:
            raise ValueError("scales are for codes")
        if out is None:
            out = _new((rows, features), dtype or _modules["torch"].float32, x, stream)
        elif tuple(out.shape) != (rows, features) or (dtype and out.dtype != dtype):
            raise ValueError(f"output must be {(rows, features)}, of type dtype if that is given")
        op, kind, row, sp = out.data_ptr(), _type(out.dtype), _rows(out, "output"), None
    desc = Fp8Desc(rows, cols, features, blocks, kind, _act(act), 0, row, 0)
    workspace, wp, size = _byte_workspace(lib().patdnn_fp8_gated_workspace_bytes, desc, workspace, x, stream)
    _call(device, stream, lib().patdnn_fp8_gated, ctypes.byref(desc), *pointers, op, sp, wp, size)
    return (out, scales) if fp8 else out


def patdnn_fp8_gated_backward(dh, x, x_scales, gate, gate_scales, up, up_scales, out=None, *, act="silu", dtype=None, workspace=None, stream=None):
    """Gradients of the two projections of patdnn_fp8_gated from dh [rows, out], the gradient of its result: [rows, 2 * out], gate's beside up's, of type ``out``'s,
    ``dtype`` or dh's."""
    device = _together(x, x_scales, gate, gate_scales, up, up_scales, dh, out, workspace)
    rows, cols, features, blocks, pointers = _fp8_operands(x, x_scales, ((gate, gate_scales), (up, up_scales)))
    if tuple(dh.shape) != (rows, features):
        raise ValueError(f"dh must be {(rows, features)}")
    if out is None:
        out = _new((rows, 2 * features), dtype or dh.dtype, x, stream)
    elif tuple(out.shape) != (rows, 2 * features) or (dtype and out.dtype != dtype):
        raise ValueError(f"output must be {(rows, 2 * features)}, of type dtype if that is given")
    desc = Fp8Desc(rows, cols, features, blocks, _type(out.dtype), _act(act), _type(dh.dtype), _rows(out, "output"), _rows(dh, "dh"))
    workspace, wp, size = _byte_workspace(lib().patdnn_fp8_gated_backward_workspace_bytes, desc, workspace, x, stream)
    at = out.data_ptr()
    _call(device, stream, lib().patdnn_fp8_gated_backward, ctypes.byref(desc), dh.data_ptr(), *pointers, at, at + features * out.element_size(), wp, size)
    return out


# ---------------------------------------------------------------------------
# convenience wrapper owning one handle
# ---------------------------------------------------------------------------

class Layer:
    def __init__(self, dense_weights, pattern_ids, kernel_mask, pattern_masks, *, stride=1, pad=1,
                 depthwise=False, dense=False, strict=False, host_only=False):
        w = np.asarray(dense_weights)
        flags = (PATDNN_DENSE if dense else 0) | (PATDNN_STRICT if strict else 0) | \
                (PATDNN_HOST_ONLY if host_only else 0)
        self.c_out, self.kpf = int(w.shape[0]), int(w.shape[1])
        self.handle = patdnn_encode(w, pattern_ids, kernel_mask, pattern_masks, stride=stride,
                                    pad=pad, groups=self.c_out if depthwise else 1, flags=flags)

    @classmethod
    def from_workload(cls, layer: dict, **kw) -> "Layer":
        spec = layer["spec"]
        return cls(layer["weights"], layer["pattern_ids"], layer["kernel_mask"],
                   layer["pattern_masks"], stride=spec.stride, pad=spec.pad,
                   depthwise=spec.depthwise, dense=spec.dense, **kw)

    def conv2d(self, x, bias=None, out=None, *, relu=False, stream=None):
        return patdnn_conv2d(self.handle, x, bias, out, fuse_relu=relu, stream=stream)

    def conv2d_ws(self, x, bias=None, out=None, *, workspace=None, relu=False, pool=False, stream=None):
        return patdnn_conv2d_ws(self.handle, x, bias, out, workspace=workspace, fuse_relu=relu, pool=pool,
                                stream=stream)

    def workspace_floats(self, n, h, w):
        return patdnn_workspace_floats(self.handle, n, h, w)

    def conv2d_f16(self, x, bias=None, out=None, *, relu=False, stream=None):
        return patdnn_conv2d_f16(self.handle, x, bias, out, fuse_relu=relu, stream=stream)

    def conv2d_pool(self, x, bias=None, out=None, *, stream=None):
        return patdnn_conv2d_pool(self.handle, x, bias, out, stream=stream)

    def output_shape(self, n, h, w):
        return patdnn_output_shape(self.handle, n, h, w)

    def decode(self):
        return patdnn_decode(self.handle, self.c_out, self.kpf)

    def export_fkw(self):
        return patdnn_export_fkw(self.handle, self.c_out)

    def export_csr(self):
        return patdnn_export_csr(self.handle, self.c_out)

    def stats(self):
        return patdnn_layout_stats(self.handle)

    def set_config(self, variant, ck=0, waves=0, ksplit=0):
        patdnn_set_config(self.handle, variant, ck, waves, ksplit)

    def get_config(self):
        return patdnn_get_config(self.handle)

    def export_tiled(self, variant, ck=0):
        return patdnn_export_tiled(self.handle, variant, ck)

    def tune(self, x, bias, out, *, workspace=None, stream=None):
        return patdnn_tune(self.handle, x, bias, out, workspace=workspace, stream=stream)

    def close(self):
        patdnn_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
