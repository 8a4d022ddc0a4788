"""Thin ctypes binding of libvarco.so: argument marshalling only. Every step of the hot path runs in the
library's HIP kernels; torch tensors serve as device memory and torch streams as hipStream_t handles.

The library must have been built (python -m paper_2406_17611_amd.build, or __graft_entry__.build());
loading fails loudly otherwise - there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
import weakref

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvarco.so")

OK, ERR_INVALID_ARG, ERR_SHAPE, ERR_STATE, ERR_UNSUPPORTED, ERR_HIP = range(6)
CONV_GCN, CONV_SAGE = 0, 1
ACT_IDENTITY, ACT_RELU = 0, 1
ORDER_AGGREGATE_FIRST, ORDER_TRANSFORM_FIRST = 0, 1
F32 = 0
BF16 = 1
MAX_LAYERS = 16
MAX_CODE_WIDTH = 16384
CODE_BLOCK = 128          # columns of a row of codes that share a scale

EXPORTS = [
    "varco_partition_build", "varco_partition_view", "varco_partition_free",
    "varco_create", "varco_destroy", "varco_register_partition", "varco_prepare", "varco_last_error",
    "varco_begin_step", "varco_set_ratio", "varco_set_matmul_terms", "varco_set_layer_order", "varco_get_keep",
    "varco_compress", "varco_decompress", "varco_layer_fwd", "varco_layer_bwd",
    "varco_accumulate_returned", "varco_get_stats", "varco_reset_stats", "varco_profile_enable", "varco_profile_read",
    "varco_calibration_copy", "varco_sum_gradients", "varco_softmax_xent", "varco_sgd_step", "varco_schedule_ratio",
    "varco_step_table_enable", "varco_set_step", "varco_advance_step",
    "varco_aggregate_fwd", "varco_aggregate_bwd", "varco_transform_fwd", "varco_transform_bwd_weight",
    "varco_transform_bwd_input", "varco_transform_bwd_weight_static",
    "varco_link_partitions", "varco_network_forward", "varco_network_backward", "varco_network_compress",
    "varco_network_aggregate_fwd", "varco_network_aggregate_bwd",
    "varco_network_taps_fwd", "varco_network_taps_bwd_weight", "varco_network_taps_bwd_input",
    "varco_network_taps_bwd_last_hop",
    "varco_quantize_rows", "varco_quantize_weights", "varco_scaled_transform", "varco_scaled_weight_workspace",
    "varco_scaled_bwd_weight", "varco_rms_norm_fwd", "varco_rms_norm_workspace", "varco_rms_norm_bwd",
    "varco_gradient_norm_workspace", "varco_gradient_norm", "varco_clip_gradients", "varco_sgd_step_clipped",
]
KERNEL_CLASSES = ["compress", "decompress", "agg_fwd", "gemm_fwd", "gemm_wgrad", "gemm_dgrad", "agg_bwd_local",
                  "agg_bwd_halo", "reduce", "agg_bwd_halo_sum"]


class Config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_partitions", C.c_int32), ("conv", C.c_int32), ("dtype", C.c_int32),
                ("mask_key", C.c_uint64), ("widths", C.POINTER(C.c_int32)), ("act", C.POINTER(C.c_int32))]


_DESC_ARRAYS = [("rowptr", np.int32), ("colidx", np.int32), ("vals", np.float32), ("t_rowptr", np.int32),
                ("t_colidx", np.int32), ("t_vals", np.float32), ("local_gid", np.int32), ("halo_gid", np.int32),
                ("halo_owner_ptr", np.int32), ("boundary_rows", np.int32), ("halo_src_row", np.int32),
                ("halo_zrow", np.int32), ("ret_ptr", np.int32), ("ret_src", np.int32)]


class PartitionDesc(C.Structure):
    _fields_ = ([("n_local", C.c_int32), ("n_halo", C.c_int32), ("n_boundary", C.c_int32),
                 ("z_row_offset", C.c_int32), ("nnz", C.c_int64), ("halo_row_offset", C.c_int32),
                 ("n_returned", C.c_int32)] + [(name, C.c_void_p) for name, _ in _DESC_ARRAYS])


class Stats(C.Structure):
    _fields_ = [("fwd_elems", C.c_int64 * MAX_LAYERS), ("bwd_elems", C.c_int64 * MAX_LAYERS),
                ("full_fwd_elems", C.c_int64 * MAX_LAYERS), ("full_bwd_elems", C.c_int64 * MAX_LAYERS),
                ("bytes_per_elem", C.c_int32)]


class Profile(C.Structure):
    _fields_ = [("launches", C.c_int64 * 10), ("ms", C.c_double * 10), ("bytes", C.c_double * 10),
                ("flops", C.c_double * 10), ("stream_bytes", C.c_double * 10)]


class NetworkBuffers(C.Structure):
    """varco_network_buffers: device addresses of the arenas of a whole network."""
    _fields_ = [("x", C.c_void_p * (MAX_LAYERS + 1)), ("z", C.c_void_p * MAX_LAYERS), ("m", C.c_void_p * MAX_LAYERS),
                ("h1", C.c_void_p * MAX_LAYERS), ("h0", C.c_void_p * MAX_LAYERS), ("dh1", C.c_void_p * MAX_LAYERS),
                ("dh0", C.c_void_p * MAX_LAYERS), ("dx", C.c_void_p * (MAX_LAYERS + 1))]


class VarcoError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"varco status {code}: {text}")
        self.code = code


_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2406_17611_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u32, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32, C.c_uint64
        L.varco_partition_build.argtypes = [i32, vp, vp, vp, vp, i32, C.POINTER(vp)]
        L.varco_partition_view.argtypes = [vp, i32, C.POINTER(PartitionDesc)]
        L.varco_partition_free.argtypes = [vp]
        L.varco_partition_free.restype = None
        L.varco_create.argtypes = [C.POINTER(Config), C.POINTER(vp)]
        L.varco_destroy.argtypes = [vp]
        L.varco_register_partition.argtypes = [vp, i32, C.POINTER(PartitionDesc)]
        L.varco_prepare.argtypes = [vp, vp]
        L.varco_last_error.argtypes = [vp]
        L.varco_last_error.restype = C.c_char_p
        L.varco_begin_step.argtypes = [vp, u64]
        L.varco_set_matmul_terms.argtypes = [vp, C.c_int32]
        L.varco_set_layer_order.argtypes = [vp, i32, i32]
        L.varco_set_ratio.argtypes = [vp, i32, u32, u32]
        L.varco_get_keep.argtypes = [vp, i32, C.POINTER(i32)]
        L.varco_compress.argtypes = [vp, i32, vp, vp, i64, vp, i64, vp, vp]
        L.varco_decompress.argtypes = [vp, i32, vp, vp, i64, vp, vp, i64, i32, vp]
        L.varco_layer_fwd.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.varco_layer_bwd.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.varco_accumulate_returned.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp]
        L.varco_get_stats.argtypes = [vp, C.POINTER(Stats)]
        L.varco_reset_stats.argtypes = [vp]
        L.varco_calibration_copy.argtypes = [vp, vp, i64, vp]
        L.varco_sum_gradients.argtypes = [vp, vp, i64, vp]
        L.varco_softmax_xent.argtypes = [vp, vp, i64, vp, i64, i32, C.c_float, vp, i64, vp, vp, vp, vp]
        L.varco_sgd_step.argtypes = [vp, vp, i64, C.c_float, vp]
        L.varco_schedule_ratio.argtypes = [i32, i64, i64, C.c_uint32, C.c_uint32, C.c_uint32, C.POINTER(C.c_uint32),
                                           C.POINTER(C.c_uint32)]
        L.varco_step_table_enable.argtypes = [vp, vp]
        L.varco_set_step.argtypes = [vp, u64, vp]
        L.varco_advance_step.argtypes = [vp, vp]
        L.varco_aggregate_fwd.argtypes = [vp, i32, i32, vp, vp, vp, vp]
        L.varco_aggregate_bwd.argtypes = [vp, i32, i32, vp, vp, vp, vp]
        L.varco_transform_fwd.argtypes = [vp, i32, i64, vp, vp, vp, i32, i32, vp]
        L.varco_transform_bwd_weight.argtypes = [vp, i32, i64, vp, vp, vp, vp, vp]
        L.varco_transform_bwd_input.argtypes = [vp, i32, i64, vp, vp, vp, vp, i32, vp]
        L.varco_transform_bwd_weight_static.argtypes = [vp, i32, i64, vp, vp, vp, vp, vp]
        L.varco_link_partitions.argtypes = [vp]
        L.varco_network_forward.argtypes = [vp, C.POINTER(NetworkBuffers), vp]
        L.varco_network_backward.argtypes = [vp, C.POINTER(NetworkBuffers), vp]
        L.varco_network_compress.argtypes = [vp, i32, vp, vp, vp]
        L.varco_network_aggregate_fwd.argtypes = [vp, i32, vp, vp, vp, vp]
        L.varco_network_aggregate_bwd.argtypes = [vp, i32, vp, vp, i32, vp]
        L.varco_network_taps_fwd.argtypes = [vp, i32, i32, vp, vp, vp, vp]
        L.varco_network_taps_bwd_weight.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp]
        L.varco_network_taps_bwd_input.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp]
        L.varco_network_taps_bwd_last_hop.argtypes = [vp, i32, vp, vp, vp, vp, C.POINTER(i32), vp]
        f32 = C.c_float
        L.varco_quantize_rows.argtypes = [i32, i64, i32, vp, i64, vp, i64, vp, vp, vp]
        L.varco_quantize_weights.argtypes = [i32, i32, vp, i64, vp, vp, vp, vp, vp]
        L.varco_scaled_transform.argtypes = [i32, i64, i32, i32, vp, vp, vp, vp, vp, i64, i32, i32, vp]
        L.varco_scaled_weight_workspace.argtypes = [i64, i32, i32, C.POINTER(i64)]
        L.varco_scaled_bwd_weight.argtypes = [i64, i32, i32, vp, vp, vp, vp, vp, i64, i32, vp, i64, vp]
        L.varco_rms_norm_fwd.argtypes = [i32, i64, i32, vp, i64, vp, i64, vp, f32, vp, i64, vp, i64, vp, vp, vp, vp]
        L.varco_rms_norm_workspace.argtypes = [i32, i64, i32, C.POINTER(i64)]
        L.varco_rms_norm_bwd.argtypes = [i32, i64, i32, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, i32, vp, i64, vp]
        L.varco_gradient_norm_workspace.argtypes = [i32, vp, C.POINTER(i64)]
        L.varco_gradient_norm.argtypes = [i32, i32, vp, vp, f32, vp, vp, i64, vp]
        L.varco_clip_gradients.argtypes = [i32, i32, vp, vp, vp, f32, vp, vp, i64, vp]
        L.varco_sgd_step_clipped.argtypes = [i32, vp, vp, vp, f32, f32, vp, vp, i64, vp]
        L.varco_profile_enable.argtypes = [vp, i32]
        L.varco_profile_read.argtypes = [vp, C.POINTER(Profile), i32]
        for name in EXPORTS:
            if name not in ("varco_partition_free", "varco_last_error"):
                getattr(L, name).restype = i32
        _lib = L
    return _lib


def _check(code: int, ctx=None):
    if code != OK:
        text = lib().varco_last_error(ctx)
        raise VarcoError(code, text.decode() if text else "")


def _ptr(t):
    """Device (or host) address of a torch tensor / numpy array, None -> NULL."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # the handle itself: a tenth of the cost of a Stream object
        if raw is not None:
            return raw(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def calibration_copy(dst, src, stream=None):
    """Copies the bytes of tensor `src` into `dst` with the library's plain copy kernel."""
    _check(lib().varco_calibration_copy(_ptr(dst), _ptr(src), src.numel() * src.element_size(), _stream(stream)))


SCHED_LINEAR, SCHED_FIXED_INCREMENT, SCHED_EXPONENTIAL = 0, 1, 2


def tap(layer: int, hop: int) -> int:
    """Address of hop `hop` of a K-tap layer (VARCO_TAP of the header)."""
    return layer + MAX_LAYERS * hop


def schedule_ratio(kind: int, step: int, n_steps: int, c_max: int, c_min: int, param: int):
    """(num, den) of the compression ratio at iteration `step` (host only)."""
    num, den = C.c_uint32(), C.c_uint32()
    _check(lib().varco_schedule_ratio(kind, step, n_steps, c_max, c_min, param, C.byref(num), C.byref(den)))
    return num.value, den.value


def sgd_step(w, dw, lr: float, stream=None):
    """w -= lr * dw (fp32 device tensors of equal size)."""
    assert w.numel() == dw.numel() and w.dtype == dw.dtype
    _check(lib().varco_sgd_step(_ptr(w), _ptr(dw), w.numel(), lr, _stream(stream)))


def sum_gradients(dst, src, stream=None):
    """dst += src (fp32 device tensors of equal size)."""
    assert dst.numel() == src.numel() and dst.dtype == src.dtype
    _check(lib().varco_sum_gradients(_ptr(dst), _ptr(src), dst.numel(), _stream(stream)))


# ---------------------------------------------------------------------------------------------------------
# normalised rows, 8-bit codes and their products, limited gradient steps
# ---------------------------------------------------------------------------------------------------------

def code_ld(width: int) -> int:
    """Bytes of a row of `width` codes (VARCO_CODE_LD of the header)."""
    return (width + 15) // 16 * 16


def scale_ld(width: int) -> int:
    """Bytes of the scales of a row of `width` codes (VARCO_SCALE_LD of the header)."""
    return (width + 511) // 512 * 4


def _refuse(code, text):
    raise VarcoError(code, text)


_DTYPES = {}
_torch = _device = _handle = None


def _load_torch():
    """torch, looked up once: an import statement and two device queries are a fifth of what a small call takes on the host."""
    global _torch, _device, _handle
    import torch
    _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _handle = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _DTYPES.update({torch.float32: F32, torch.bfloat16: BF16})
    _torch = torch


def _dtype(t):
    if _torch is None:
        _load_torch()
    code = _DTYPES.get(t.dtype)
    if code is None:
        _refuse(ERR_UNSUPPORTED, f"{t.dtype}: neither float32 nor bfloat16")
    return code


def _on_device(stream, *tensors):
    """The handle of a call's stream. Stream and tensors are of the device that is current (a launch goes to the stream's, whatever device
    the memory is on)."""
    if _torch is None:
        _load_torch()
    current = _device()
    for t in tensors:
        if t is not None and t.get_device() != current:
            _refuse(ERR_INVALID_ARG, f"a tensor on {t.device}, the current device is cuda:{current}")
    if stream is None and _handle is not None:
        return _handle(current)
    if getattr(stream, "device_index", current) != current:
        _refuse(ERR_INVALID_ARG, f"a stream of cuda:{stream.device_index}, the current device is cuda:{current}")
    return _stream(stream)


def _matrix(t, shape, like, what):
    """(address, leading dimension) of a matrix whose rows' elements are consecutive; None -> NULL."""
    if t is None:
        return None, 0
    if t.shape != shape:
        _refuse(ERR_SHAPE, f"{what}: {tuple(t.shape)} where {tuple(shape)} is needed")
    if t.dtype != like:
        _refuse(ERR_UNSUPPORTED, f"{what}: {t.dtype} where {like} is needed")
    ld, one = t.stride()
    if one != 1 and shape[1] > 1:
        _refuse(ERR_SHAPE, f"{what}: the elements of a row are not consecutive")
    return t.data_ptr(), ld if shape[0] > 1 else shape[1]


def _rows(t, what):
    """(rows, width) of a matrix."""
    if t.dim() != 2:
        _refuse(ERR_SHAPE, f"{what}: a matrix is needed, got {tuple(t.shape)}")
    return t.shape


def _vector(t, n, what):
    if t is None:
        return None
    if t.dtype != _torch.float32 or t.numel() != n or not t.is_contiguous():
        _refuse(ERR_SHAPE, f"{what}: {n} consecutive float32 values are needed")
    return t.data_ptr()


def _code_rows(codes, scales, rows, width, scale_rows, what):
    """Addresses of rows of codes and of their scales: whole buffers of bytes (uint8, or the 8-bit float types)."""
    if codes is None and scales is None:
        return None, None
    if codes is None or scales is None:
        _refuse(ERR_INVALID_ARG, f"{what}: codes without scales")
    for t, n, ld in ((codes, rows, code_ld(width)), (scales, scale_rows, scale_ld(width))):
        if t.element_size() != 1 or t.shape != (n, ld) or not t.is_contiguous():
            _refuse(ERR_SHAPE, f"{what}: {tuple(t.shape)} where {n} whole rows of {ld} bytes are needed")
    return codes.data_ptr(), scales.data_ptr()


def _scratch(need, workspace, device, stream):
    """(address, bytes, tensor to hold) of a call's scratch memory: the caller's, or a new one that torch's allocator keeps for work of
    the call's stream."""
    if workspace is None:
        if need == 0:
            return None, 0, None
        if stream is None:
            workspace = _torch.empty(need, dtype=_torch.uint8, device=device)
        else:
            if not hasattr(stream, "cuda_stream"):               # a handle; 0 is the default stream's
                stream = _torch.cuda.ExternalStream(stream) if stream else _torch.cuda.default_stream()
            with _torch.cuda.stream(stream):
                workspace = _torch.empty(need, dtype=_torch.uint8, device=device)
    elif not workspace.is_contiguous():
        _refuse(ERR_SHAPE, "a workspace that is not consecutive in memory")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def quantize_rows(x, codes, scales, gate=None, stream=None):
    """codes [n, code_ld(width)], scales [n, scale_ld(width)] of the rows of x (of x where gate > 0)."""
    dt, (n, w) = _dtype(x), _rows(x, "x")
    at = _on_device(stream, x, codes, scales, gate)
    px, ldx = _matrix(x, (n, w), x.dtype, "x")
    pg, ldg = _matrix(gate, (n, w), x.dtype, "gate")
    pc, ps = _code_rows(codes, scales, n, w, n, "codes")
    _check(lib().varco_quantize_rows(dt, n, w, px, ldx, pg, ldg, pc, ps, at))


def quantize_weights(h, turned=None, turned_scales=None, codes=None, scales=None, stream=None):
    """Codes of fp32 weights h [n_in, n_out]: turned [n_out, code_ld(n_in)] for the forward product, codes [n_in, code_ld(n_out)] for
    the input gradient; their scales have a row for each 128 rows of codes."""
    n_in, n_out = _rows(h, "h")
    at = _on_device(stream, h, turned, turned_scales, codes, scales)
    ph, ldh = _matrix(h, (n_in, n_out), _torch.float32, "h")
    pt, pts = _code_rows(turned, turned_scales, n_out, n_in, -(-n_out // CODE_BLOCK), "turned")
    pc, ps = _code_rows(codes, scales, n_in, n_out, -(-n_in // CODE_BLOCK), "codes")
    _check(lib().varco_quantize_weights(n_in, n_out, ph, ldh, pt, pts, pc, ps, at))


def scaled_transform(codes, scales, w_codes, w_scales, n_in, c, accumulate=False, act=ACT_IDENTITY, stream=None):
    """c = act((c +) X W): X rows of n_in codes, W the weights whose rows of codes are c's columns."""
    dt, (n, n_out) = _dtype(c), _rows(c, "c")
    at = _on_device(stream, codes, scales, w_codes, w_scales, c)
    pc, ldc = _matrix(c, (n, n_out), c.dtype, "c")
    px, pxs = _code_rows(codes, scales, n, n_in, n, "codes")
    pw, pws = _code_rows(w_codes, w_scales, n_out, n_in, -(-n_out // CODE_BLOCK), "w_codes")
    _check(lib().varco_scaled_transform(dt, n, n_in, n_out, px, pxs, pw, pws, pc, ldc, int(accumulate), act, at))


def scaled_weight_workspace(n_rows, n_in, n_out) -> int:
    out = C.c_int64()
    _check(lib().varco_scaled_weight_workspace(n_rows, n_in, n_out, C.byref(out)))
    return out.value


def scaled_bwd_weight(y_codes, y_scales, d_codes, d_scales, dh, accumulate=False, workspace=None, stream=None):
    """dh (+)= Y^T D, dh [n_in, n_out] fp32, from rows of codes of the inputs and of the errors."""
    n, (n_in, n_out) = y_codes.shape[0], _rows(dh, "dh")
    at = _on_device(stream, y_codes, y_scales, d_codes, d_scales, dh, workspace)
    ph, ldh = _matrix(dh, (n_in, n_out), _torch.float32, "dh")
    py, pys = _code_rows(y_codes, y_scales, n, n_in, n, "y_codes")
    pd, pds = _code_rows(d_codes, d_scales, n, n_out, n, "d_codes")
    pw, size, held = _scratch(scaled_weight_workspace(n, n_in, n_out) if workspace is None else 0, workspace, dh.device, stream)
    _check(lib().varco_scaled_bwd_weight(n, n_in, n_out, py, pys, pd, pds, ph, ldh, int(accumulate), pw, size, at))


def rms_norm_fwd(x, gain, eps, residual=None, total=None, y=None, codes=None, scales=None, inv_rms=None, stream=None):
    """u = x + residual, y = u gain / sqrt(mean u^2 + eps); writes what is given of total (u), y, codes with scales, inv_rms."""
    dt, (n, w) = _dtype(x), _rows(x, "x")
    at = _on_device(stream, x, gain, residual, total, y, codes, scales, inv_rms)
    px, ldx = _matrix(x, (n, w), x.dtype, "x")
    pr, ldr = _matrix(residual, (n, w), x.dtype, "residual")
    pt, ldt = _matrix(total, (n, w), x.dtype, "total")
    py, ldy = _matrix(y, (n, w), x.dtype, "y")
    pc, ps = _code_rows(codes, scales, n, w, n, "codes")
    _check(lib().varco_rms_norm_fwd(dt, n, w, px, ldx, pr, ldr, _vector(gain, w, "gain"), eps, pt, ldt, py, ldy, pc, ps,
                                    _vector(inv_rms, n, "inv_rms"), at))


def rms_norm_workspace(dtype, n_rows, width) -> int:
    out = C.c_int64()
    _check(lib().varco_rms_norm_workspace(dtype, n_rows, width, C.byref(out)))
    return out.value


def rms_norm_bwd(dy, u, gain, inv_rms, dx=None, dgain=None, dtotal=None, accumulate=False, workspace=None, stream=None):
    """dx = gradient of u through the norm (+ dtotal); dgain (+)= the gain's gradient."""
    dt, (n, w) = _dtype(dy), _rows(dy, "dy")
    at = _on_device(stream, dy, u, gain, inv_rms, dx, dgain, dtotal, workspace)
    pd, ldd = _matrix(dy, (n, w), dy.dtype, "dy")
    pu, ldu = _matrix(u, (n, w), dy.dtype, "u")
    pt, ldt = _matrix(dtotal, (n, w), dy.dtype, "dtotal")
    px, ldx = _matrix(dx, (n, w), dy.dtype, "dx")
    pw, size, held = _scratch(rms_norm_workspace(dt, n, w) if workspace is None and dgain is not None else 0, workspace, dy.device, stream)
    _check(lib().varco_rms_norm_bwd(dt, n, w, pd, ldd, pu, ldu, _vector(gain, w, "gain"), _vector(inv_rms, n, "inv_rms"), pt, ldt, px, ldx,
                                    _vector(dgain, w, "dgain"), int(accumulate), pw, size, at))


class TensorList:
    """Addresses and sizes of tensors that a program updates together, made once: device tensors of one type, each consecutive in
    memory, none overlapping another. Holds the tensors; one that has been given other memory since (t.data = ...) is taken where it is
    when the list is used."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self._take()

    def _take(self):
        self.dtype = _dtype(self.tensors[0]) if self.tensors else F32
        for t in self.tensors:
            if _dtype(t) != self.dtype:
                _refuse(ERR_UNSUPPORTED, "tensors of different types")
            if not t.is_contiguous():
                _refuse(ERR_SHAPE, "a tensor that is not consecutive in memory")
            if t.get_device() != self.tensors[0].get_device() or not t.is_cuda:
                _refuse(ERR_INVALID_ARG, "tensors on different devices or not on one")
        at, counts = [t.data_ptr() for t in self.tensors], [t.numel() for t in self.tensors]
        spans = sorted((p, p + n * t.element_size(), i) for i, (p, n, t) in enumerate(zip(at, counts, self.tensors)) if n)
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            _refuse(ERR_INVALID_ARG, "tensors that overlap")
        self._spans, self._apart = spans, None
        self.pointers = (C.c_void_p * len(at))(*at)
        self.sizes = (C.c_int64 * len(at))(*counts)
        self.need = gradient_norm_workspace(self)
        self._at = list(zip(self.tensors, at, counts))

    def current(self):
        """The list itself, of the memory that its tensors have now: a step on memory that was given up would write to what has taken its
        place."""
        for t, p, n in self._at:
            if t.data_ptr() != p or t.numel() != n:
                self._take()
                break
        return self

    def __len__(self):
        return len(self.tensors)


def _listed(tensors):
    return tensors.current() if isinstance(tensors, TensorList) else TensorList(tensors)


def gradient_norm_workspace(tensors) -> int:
    out = C.c_int64()
    _check(lib().varco_gradient_norm_workspace(len(tensors), tensors.sizes, C.byref(out)))
    return out.value


def _same_sizes(a, b):
    if len(a) != len(b) or a.dtype != b.dtype or bytes(a.sizes) != bytes(b.sizes):
        _refuse(ERR_SHAPE, "lists of tensors that do not match")


def _check_apart(written, read, in_place):
    """Refuses to write a list that overlaps the one that is read: workgroups would overwrite what others have yet to read. in_place: a tensor
    may be the one at its place in the other list. The last verdict stays with the list: a pair that a program steps with is compared once."""
    known = written._apart
    if known is not None and known[0]() is read and known[1] is read._at and known[2] == in_place:
        return
    if not (in_place and written is read):
        a, b = written._spans, read._spans
        i = j = 0
        while i < len(a) and j < len(b):
            (start, end, k), (other, other_end, m) = a[i], b[j]
            if start < other_end and other < end and not (in_place and start == other and k == m):
                _refuse(ERR_INVALID_ARG, "lists of tensors that overlap")
            if end <= other_end:
                i += 1
            else:
                j += 1
    written._apart = weakref.ref(read), read._at, in_place


def _limit_out(out):
    if out is None or out.dtype != _torch.float32 or out.numel() != 2 or not out.is_contiguous():
        _refuse(ERR_SHAPE, "out: 2 consecutive float32 values are needed")
    return out.data_ptr()


def gradient_norm(grads, max_norm, out, workspace=None, stream=None):
    """out[0] = norm of all tensors of `grads` together, out[1] = min(1, max_norm / norm)."""
    g = _listed(grads)
    at = _on_device(stream, out, workspace, *g.tensors[:1])
    pw, size, held = _scratch(g.need, workspace, out.device, stream)
    _check(lib().varco_gradient_norm(g.dtype, len(g), g.pointers, g.sizes, max_norm, _limit_out(out), pw, size, at))


def clip_gradients(grads, max_norm, out, into=None, workspace=None, stream=None):
    """gradient_norm, and into[t] = out[1] * grads[t] (into None: in place; else into[t] is grads[t] or overlaps none of them)."""
    g = _listed(grads)
    to = g if into is None else _listed(into)
    _same_sizes(g, to)
    _check_apart(to, g, True)
    at = _on_device(stream, out, workspace, *g.tensors[:1], *to.tensors[:1])
    pw, size, held = _scratch(g.need, workspace, out.device, stream)
    _check(lib().varco_clip_gradients(g.dtype, len(g), g.pointers, to.pointers, g.sizes, max_norm, _limit_out(out), pw, size, at))


def sgd_step_clipped(w, dw, lr, max_norm, out, workspace=None, stream=None):
    """gradient_norm of dw, and w[t] -= lr * out[1] * dw[t] (fp32; w overlaps no gradient)."""
    g, to = _listed(dw), _listed(w)
    _same_sizes(g, to)
    _check_apart(to, g, False)
    if g.dtype != F32:
        _refuse(ERR_UNSUPPORTED, "weights and their gradients are float32")
    at = _on_device(stream, out, workspace, *g.tensors[:1], *to.tensors[:1])
    pw, size, held = _scratch(g.need, workspace, out.device, stream)
    _check(lib().varco_sgd_step_clipped(len(g), to.pointers, g.pointers, g.sizes, lr, max_norm, _limit_out(out), pw, size, at))


# ---------------------------------------------------------------------------------------------------------
# host-side partition builder
# ---------------------------------------------------------------------------------------------------------

class HostPartition:
    """numpy copies of one partition's index structures, as built by varco_partition_build."""

    def __init__(self, desc: PartitionDesc):
        self.n_local, self.n_halo, self.n_boundary = desc.n_local, desc.n_halo, desc.n_boundary
        self.z_row_offset, self.nnz = desc.z_row_offset, desc.nnz
        self.halo_row_offset, self.n_returned = desc.halo_row_offset, desc.n_returned
        sizes = {"rowptr": self.n_local + 1, "colidx": self.nnz, "vals": self.nnz,
                 "t_rowptr": self.n_local + self.n_halo + 1, "t_colidx": self.nnz, "t_vals": self.nnz,
                 "local_gid": self.n_local, "halo_gid": self.n_halo, "halo_owner_ptr": None,
                 "boundary_rows": self.n_boundary, "halo_src_row": self.n_halo, "halo_zrow": self.n_halo,
                 "ret_ptr": self.n_boundary + 1, "ret_src": self.n_returned}
        self._sizes = sizes

    def _fill(self, desc, n_parts):
        self._sizes["halo_owner_ptr"] = n_parts + 1
        for name, dt in _DESC_ARRAYS:
            n = self._sizes[name]
            addr = getattr(desc, name)
            if n == 0 or not addr:
                arr = np.empty(0, dtype=dt)
            else:
                arr = np.ctypeslib.as_array(C.cast(addr, C.POINTER(np.ctypeslib.as_ctypes_type(dt))), shape=(n,)).copy()
            setattr(self, name, arr)


def partition_build(n: int, rowptr: np.ndarray, colidx: np.ndarray, vals: np.ndarray, part: np.ndarray,
                    n_parts: int) -> list[HostPartition]:
    """Runs the library's host-side builder and returns numpy copies of every partition's arrays."""
    L = lib()
    rowptr = np.ascontiguousarray(rowptr, dtype=np.int64)
    colidx = np.ascontiguousarray(colidx, dtype=np.int32)
    vals = np.ascontiguousarray(vals, dtype=np.float32)
    part = np.ascontiguousarray(part, dtype=np.int32)
    if rowptr.shape[0] != n + 1 or part.shape[0] != n or colidx.shape[0] != vals.shape[0]:
        raise VarcoError(ERR_SHAPE, "partition_build: array lengths do not match n")
    h = C.c_void_p()
    _check(L.varco_partition_build(n, rowptr.ctypes.data, colidx.ctypes.data, vals.ctypes.data, part.ctypes.data,
                                   n_parts, C.byref(h)))
    try:
        out = []
        for q in range(n_parts):
            d = PartitionDesc()
            _check(L.varco_partition_view(h, q, C.byref(d)))
            hp = HostPartition(d)
            hp._fill(d, n_parts)
            out.append(hp)
        return out
    finally:
        L.varco_partition_free(h)


# ---------------------------------------------------------------------------------------------------------
# context
# ---------------------------------------------------------------------------------------------------------

class Context:
    def __init__(self, widths, act, conv: int, n_partitions: int, mask_key: int, dtype: int = F32):
        L = lib()
        self._widths = (C.c_int32 * len(widths))(*widths)
        self._act = (C.c_int32 * len(act))(*act)
        cfg = Config(len(act), n_partitions, conv, dtype, mask_key, self._widths, self._act)
        self._h = C.c_void_p()
        _check(L.varco_create(C.byref(cfg), C.byref(self._h)))
        self.widths = list(widths)
        self.n_layers = len(act)
        self.n_partitions = n_partitions
        self.step_on_device = False
        self._keep = {}          # device tensors of registered partitions (kept alive)
        self.parts = {}

    def close(self):
        if self._h:
            lib().varco_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def register_partition(self, q: int, hp: HostPartition, device="cuda"):
        """Uploads a HostPartition's arrays (torch tensors, kept alive by this object) and registers them."""
        import torch
        dev = {}
        d = PartitionDesc()
        d.n_local, d.n_halo, d.n_boundary = hp.n_local, hp.n_halo, hp.n_boundary
        d.z_row_offset, d.nnz = hp.z_row_offset, hp.nnz
        d.halo_row_offset, d.n_returned = hp.halo_row_offset, hp.n_returned
        for name, _ in _DESC_ARRAYS:
            t = torch.from_numpy(getattr(hp, name)).to(device)
            dev[name] = t
            setattr(d, name, t.data_ptr() if t.numel() else None)
        _check(lib().varco_register_partition(self._h, q, C.byref(d)), self._h)
        self._keep[q] = dev
        self.parts[q] = hp
        return dev

    def register_raw(self, q: int, desc: PartitionDesc):
        _check(lib().varco_register_partition(self._h, q, C.byref(desc)), self._h)

    def prepare(self, stream=None):
        """Workspace set of `stream` (torch's current stream when None) and the tables of the kept positions."""
        _check(lib().varco_prepare(self._h, _stream(stream)), self._h)

    def begin_step(self, step: int):
        _check(lib().varco_begin_step(self._h, step), self._h)

    def step_table_enable(self, stream=None):
        _check(lib().varco_step_table_enable(self._h, _stream(stream)), self._h)
        self.step_on_device = True

    def set_step(self, step: int, stream=None):
        _check(lib().varco_set_step(self._h, step, _stream(stream)), self._h)

    def advance_step(self, stream=None):
        _check(lib().varco_advance_step(self._h, _stream(stream)), self._h)

    def set_matmul_terms(self, terms: int):
        _check(lib().varco_set_matmul_terms(self._h, terms), self._h)

    def set_layer_order(self, layer: int, order: int):
        _check(lib().varco_set_layer_order(self._h, layer, order), self._h)

    def set_ratio(self, layer: int, num: int, den: int = 1):
        _check(lib().varco_set_ratio(self._h, layer, num, den), self._h)

    def keep(self, layer: int) -> int:
        k = C.c_int32()
        _check(lib().varco_get_keep(self._h, layer, C.byref(k)), self._h)
        return k.value

    def compress(self, layer, gids, rows, n_rows, x, ldx, z, stream=None):
        _check(lib().varco_compress(self._h, layer, _ptr(gids), _ptr(rows), n_rows, _ptr(x), ldx, _ptr(z),
                                    _stream(stream)), self._h)

    def decompress(self, layer, gids, rows, n_rows, z, x, ldx, accumulate, stream=None):
        _check(lib().varco_decompress(self._h, layer, _ptr(gids), _ptr(rows), n_rows, _ptr(z), _ptr(x), ldx,
                                      int(accumulate), _stream(stream)), self._h)

    def layer_fwd(self, layer, q, x_local, z_in, h1, h0, x_out, z_out, m_saved, stream=None):
        _check(lib().varco_layer_fwd(self._h, layer, q, _ptr(x_local), _ptr(z_in), _ptr(h1), _ptr(h0), _ptr(x_out),
                                     _ptr(z_out), _ptr(m_saved), _stream(stream)), self._h)

    def layer_bwd(self, layer, q, dx_out, x_out, x_local, m_saved, h1, h0, dh1, dh0, dx_local, dz_halo, stream=None):
        _check(lib().varco_layer_bwd(self._h, layer, q, _ptr(dx_out), _ptr(x_out), _ptr(x_local), _ptr(m_saved),
                                     _ptr(h1), _ptr(h0), _ptr(dh1), _ptr(dh0), _ptr(dx_local), _ptr(dz_halo),
                                     _stream(stream)), self._h)

    def accumulate_returned(self, layer, p, ret_ptr, ret_src, returned, dx_local, stream=None):
        _check(lib().varco_accumulate_returned(self._h, layer, p, _ptr(ret_ptr), _ptr(ret_src), _ptr(returned),
                                               _ptr(dx_local), _stream(stream)), self._h)

    def aggregate_fwd(self, tap, q, y_local, z_in, y_out, stream=None):
        _check(lib().varco_aggregate_fwd(self._h, tap, q, _ptr(y_local), _ptr(z_in), _ptr(y_out), _stream(stream)), self._h)

    def aggregate_bwd(self, tap, q, g_out, g_local, dz_halo, stream=None):
        _check(lib().varco_aggregate_bwd(self._h, tap, q, _ptr(g_out), _ptr(g_local), _ptr(dz_halo), _stream(stream)),
               self._h)

    def transform_fwd(self, layer, y, h, c, accumulate, apply_act, stream=None):
        _check(lib().varco_transform_fwd(self._h, layer, y.shape[0], _ptr(y), _ptr(h), _ptr(c), int(accumulate),
                                         int(apply_act), _stream(stream)), self._h)

    def transform_bwd_weight(self, layer, y, dx_out, x_out, dh, stream=None):
        _check(lib().varco_transform_bwd_weight(self._h, layer, y.shape[0], _ptr(y), _ptr(dx_out), _ptr(x_out), _ptr(dh),
                                                _stream(stream)), self._h)

    def transform_bwd_weight_static(self, layer, y, dx_out, x_out, dh, stream=None):
        _check(lib().varco_transform_bwd_weight_static(self._h, layer, y.shape[0], _ptr(y), _ptr(dx_out), _ptr(x_out),
                                                       _ptr(dh), _stream(stream)), self._h)

    def transform_bwd_input(self, layer, dx_out, x_out, h, g_out, accumulate, stream=None):
        _check(lib().varco_transform_bwd_input(self._h, layer, dx_out.shape[0], _ptr(dx_out), _ptr(x_out), _ptr(h),
                                               _ptr(g_out), int(accumulate), _stream(stream)), self._h)

    def link_partitions(self):
        """Joins all registered partitions for the network_* calls; False when they are too large for that (2^31 entries, or
        no room on the device): the per-partition calls serve them then."""
        code = lib().varco_link_partitions(self._h)
        if code == ERR_UNSUPPORTED:
            return False
        _check(code, self._h)
        return True

    def network_forward(self, buffers, stream=None):
        _check(lib().varco_network_forward(self._h, C.byref(buffers), _stream(stream)), self._h)

    def network_backward(self, buffers, stream=None):
        _check(lib().varco_network_backward(self._h, C.byref(buffers), _stream(stream)), self._h)

    def network_compress(self, tap, x, z, stream=None):
        _check(lib().varco_network_compress(self._h, tap, _ptr(x), _ptr(z), _stream(stream)), self._h)

    def network_aggregate_fwd(self, tap, y, z_in, y_out, stream=None):
        _check(lib().varco_network_aggregate_fwd(self._h, tap, _ptr(y), _ptr(z_in), _ptr(y_out), _stream(stream)), self._h)

    def network_aggregate_bwd(self, tap, g_out, g_in, accumulate=False, stream=None):
        _check(lib().varco_network_aggregate_bwd(self._h, tap, _ptr(g_out), _ptr(g_in), int(accumulate), _stream(stream)), self._h)

    @staticmethod
    def _ptrs(tensors):
        return (C.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])

    def network_taps_fwd(self, layer, y, h, c, stream=None):
        _check(lib().varco_network_taps_fwd(self._h, layer, len(y), self._ptrs(y), self._ptrs(h), _ptr(c), _stream(stream)), self._h)

    def network_taps_bwd_weight(self, layer, y, dx_out, x_out, dh, stream=None):
        _check(lib().varco_network_taps_bwd_weight(self._h, layer, len(y), self._ptrs(y), _ptr(dx_out), _ptr(x_out), self._ptrs(dh),
                                                   _stream(stream)), self._h)

    def network_taps_bwd_input(self, layer, dx_out, x_out, h, g, stream=None):
        _check(lib().varco_network_taps_bwd_input(self._h, layer, len(h), _ptr(dx_out), _ptr(x_out), self._ptrs(h), self._ptrs(g),
                                                  _stream(stream)), self._h)

    def network_taps_bwd_last_hop(self, tap, dx_out, h_last, h_next, g_in, stream=None) -> bool:
        formed = C.c_int32(0)
        _check(lib().varco_network_taps_bwd_last_hop(self._h, tap, _ptr(dx_out), _ptr(h_last), _ptr(h_next), _ptr(g_in), C.byref(formed),
                                                     _stream(stream)), self._h)
        return bool(formed.value)

    def softmax_xent(self, logits, labels, n_classes, scale, dlogits, row_loss, row_correct, totals, stream=None):
        n_rows = logits.shape[0]
        _check(lib().varco_softmax_xent(self._h, _ptr(logits), logits.stride(0) if n_rows else n_classes, _ptr(labels),
                                        n_rows, n_classes, scale, _ptr(dlogits),
                                        dlogits.stride(0) if dlogits is not None and n_rows else n_classes,
                                        _ptr(row_loss), _ptr(row_correct), _ptr(totals), _stream(stream)), self._h)

    def stats(self) -> dict:
        s = Stats()
        _check(lib().varco_get_stats(self._h, C.byref(s)), self._h)
        n = self.n_layers
        return dict(fwd_elems=list(s.fwd_elems)[:n], bwd_elems=list(s.bwd_elems)[:n],
                    full_fwd_elems=list(s.full_fwd_elems)[:n], full_bwd_elems=list(s.full_bwd_elems)[:n],
                    bytes_per_elem=s.bytes_per_elem)

    def reset_stats(self):
        _check(lib().varco_reset_stats(self._h), self._h)

    def profile_enable(self, on: bool):
        _check(lib().varco_profile_enable(self._h, int(on)), self._h)

    def profile_read(self, reset: bool = True) -> dict:
        """Per kernel class: launches, total ms, algorithmic bytes and flops of the bracketed launches."""
        p = Profile()
        _check(lib().varco_profile_read(self._h, C.byref(p), int(reset)), self._h)
        return {name: dict(launches=p.launches[i], ms=p.ms[i], bytes=p.bytes[i], flops=p.flops[i],
                           stream_bytes=p.stream_bytes[i])
                for i, name in enumerate(KERNEL_CLASSES)}
