"""ctypes binding of libcct.so (include/cct.h).  Argument marshalling only.

Every function here has the name of the C entry point it calls.  Tensors are
torch tensors on the GPU (contiguous fp32); the binding passes their
``data_ptr()`` and the current HIP stream.  Nothing is computed in Python and
there is no fallback: importing this module raises if libcct.so is missing.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcct.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        "libcct.so has not been built (run `python -m paper_1504_04343_amd.build` or "
        "`__graft_entry__.build()`); there is no CPU fallback")

_lib = ctypes.CDLL(LIB_PATH)

LOWER_AUTO, LOWER_TYPE1, LOWER_TYPE2, LOWER_TYPE3, LOWER_FUSED = 0, 1, 2, 3, 4
PREC_F32, PREC_BF16_IN_F32_ACC = 0, 1
PASS_FORWARD, PASS_BACKWARD_DATA, PASS_BACKWARD_WEIGHTS = 0, 1, 2
PASS_BACKWARD = 3  # of the feed-forward operators, whose gradients are one call
TYPE_F32, TYPE_BF16, TYPE_F16 = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU, ACT_GELU_TANH = 0, 1, 2, 3, 4
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
OK, EINVAL, EWORKSPACE, EUNSUPPORTED, EHIP, ESCRATCH = 0, -1, -2, -3, -4, -5
STATIC_SCRATCH_BYTES = 32 << 20

EXPORTS = [
    "cct_strerror", "cct_last_hip_error", "cct_conv_output_dims", "cct_lowered_shape",
    "cct_pick_lowering", "cct_lowering_cost", "cct_conv_workspace_bytes",
    "cct_conv_workspace_bytes_for_chunk", "cct_conv_forward", "cct_conv_backward_data",
    "cct_conv_backward_weights", "cct_lowered_ld", "cct_lower", "cct_profile_enable",
    "cct_profile_read", "cct_calibration_copy", "cct_conv_forward_static",
    "cct_relu_forward", "cct_relu_backward", "cct_pool_output_dims", "cct_maxpool_forward",
    "cct_maxpool_backward", "cct_lrn_forward", "cct_lrn_backward",
    "cct_dropout_forward", "cct_dropout_backward", "cct_softmax_loss_forward",
    "cct_softmax_loss_backward", "cct_linear_workspace_bytes", "cct_gated_workspace_bytes",
    "cct_linear_forward", "cct_linear_backward", "cct_gated_forward", "cct_gated_backward",
    "cct_grad_norm_workspace_bytes", "cct_grad_norm", "cct_grad_scale", "cct_sgd_update",
    "cct_residual_norm_forward", "cct_residual_norm_workspace_bytes", "cct_residual_norm_backward",
    "cct_mx_quantize", "cct_mx_dequantize", "cct_mx_linear_workspace_bytes", "cct_mx_linear_forward",
    "cct_moe_workspace_bytes", "cct_moe_forward",
]


class ConvDesc(ctypes.Structure):
    """cct_conv_desc_t."""
    _fields_ = [(k, ctypes.c_int32) for k in
                ("N", "C", "H", "W", "O", "K", "stride", "pad", "groups", "lowering", "precision")]


class CctError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__("%s: %s (code %d)" % (where, strerror(code), code))


_vp, _sz, _i32, _i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64
_dp = ctypes.POINTER(ConvDesc)
_lib.cct_strerror.restype = ctypes.c_char_p
_lib.cct_strerror.argtypes = [ctypes.c_int]
_lib.cct_last_hip_error.restype = ctypes.c_int
_lib.cct_last_hip_error.argtypes = []
_lib.cct_conv_output_dims.argtypes = [_dp, ctypes.POINTER(_i32), ctypes.POINTER(_i32)]
_lib.cct_lowered_shape.argtypes = [_dp, ctypes.c_int, ctypes.POINTER(_i64), ctypes.POINTER(_i64),
                                   ctypes.POINTER(_i64)]
_lib.cct_lowered_ld.argtypes = [_dp, ctypes.c_int, ctypes.POINTER(_i64)]
_lib.cct_pick_lowering.argtypes = [_dp, ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
_lib.cct_lowering_cost.argtypes = [_dp, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_double)]
_lib.cct_conv_workspace_bytes.argtypes = [_dp, ctypes.c_int, ctypes.POINTER(_sz)]
_lib.cct_conv_workspace_bytes_for_chunk.argtypes = [_dp, ctypes.c_int, _i32, ctypes.POINTER(_sz)]
_lib.cct_conv_forward.argtypes = [_dp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.cct_conv_forward_static.argtypes = [_dp, _vp, _vp, _vp, _vp, _vp]
_lib.cct_conv_backward_data.argtypes = [_dp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.cct_conv_backward_weights.argtypes = [_dp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.cct_lower.argtypes = [_dp, ctypes.c_int, _vp, _vp, _vp]


class PoolDesc(ctypes.Structure):
    """cct_pool_desc_t."""
    _fields_ = [(k, ctypes.c_int32) for k in ("N", "C", "H", "W", "K", "stride", "pad")]


class LrnDesc(ctypes.Structure):
    """cct_lrn_desc_t."""
    _fields_ = [(k, ctypes.c_int32) for k in ("N", "C", "H", "W", "size")] + \
               [(k, ctypes.c_float) for k in ("alpha", "beta", "k")]


_pp = ctypes.POINTER(PoolDesc)
_lib.cct_relu_forward.argtypes = [_vp, _vp, _i64, _vp]
_lib.cct_relu_backward.argtypes = [_vp, _vp, _vp, _i64, _vp]
_lib.cct_pool_output_dims.argtypes = [_pp, ctypes.POINTER(_i32), ctypes.POINTER(_i32)]
_lib.cct_maxpool_forward.argtypes = [_pp, _vp, _vp, _vp, _vp]
_lib.cct_maxpool_backward.argtypes = [_pp, _vp, _vp, _vp, _vp]
_lib.cct_lrn_forward.argtypes = [ctypes.POINTER(LrnDesc), _vp, _vp, _vp]
_lib.cct_lrn_backward.argtypes = [ctypes.POINTER(LrnDesc), _vp, _vp, _vp, _vp]
_lib.cct_dropout_forward.argtypes = [_vp, _vp, ctypes.c_float, _vp, _i64, _vp]
_lib.cct_dropout_backward.argtypes = [_vp, _vp, ctypes.c_float, _vp, _i64, _vp]
_lib.cct_softmax_loss_forward.argtypes = [_i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.cct_softmax_loss_backward.argtypes = [_i32, _i32, _vp, _vp, _vp, _vp]


class LinearDesc(ctypes.Structure):
    """cct_linear_desc_t."""
    _fields_ = [(k, ctypes.c_int32) for k in ("M", "N", "K", "type", "activation")]


class GatedDesc(ctypes.Structure):
    """cct_gated_desc_t."""
    _fields_ = [(k, ctypes.c_int32) for k in ("M", "F", "K", "type", "activation")]


class Tensor(ctypes.Structure):
    """cct_tensor_t."""
    _fields_ = [("data", _vp), ("n", _i64), ("type", _i32), ("reserved", _i32)]


_lp, _gp, _tp = ctypes.POINTER(LinearDesc), ctypes.POINTER(GatedDesc), ctypes.POINTER(Tensor)
_f32 = ctypes.c_float
_lib.cct_linear_workspace_bytes.argtypes = [_lp, _i32, ctypes.POINTER(_sz)]
_lib.cct_gated_workspace_bytes.argtypes = [_gp, _i32, ctypes.POINTER(_sz)]
_lib.cct_linear_forward.argtypes = [_lp, _vp, _i64, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _sz, _vp]
_lib.cct_linear_backward.argtypes = [_lp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp,
                                     _sz, _vp]
_lib.cct_gated_forward.argtypes = [_gp] + [_vp, _i64] * 6 + [_vp, _sz, _vp]
_lib.cct_gated_backward.argtypes = [_gp] + [_vp, _i64] * 9 + [_vp, _sz, _vp]
_lib.cct_grad_norm_workspace_bytes.argtypes = [_tp, _i32, ctypes.POINTER(_sz)]
_lib.cct_grad_norm.argtypes = [_tp, _i32, _f32, _vp, _vp, _sz, _vp]
_lib.cct_grad_scale.argtypes = [_tp, _i32, _vp, _tp, _vp]
_lib.cct_sgd_update.argtypes = [_tp, _i32, _vp, _tp, _tp, _tp, _f32, _f32, _f32, _vp]


class ResidualNormDesc(ctypes.Structure):
    """cct_residual_norm_desc_t."""
    _fields_ = [(k, ctypes.c_int32) for k in ("M", "D", "type", "before", "after", "gate_rows")] + \
               [(k, ctypes.c_float) for k in ("eps", "scale")]


_np = ctypes.POINTER(ResidualNormDesc)
_lib.cct_residual_norm_forward.argtypes = [_np] + [_vp, _i64] * 3 + [_vp] * 4 + [_vp, _i64] * 2 + [_vp]
_lib.cct_residual_norm_workspace_bytes.argtypes = [_np, ctypes.POINTER(_sz)]
_lib.cct_residual_norm_backward.argtypes = [_np] + [_vp, _i64] * 3 + [_vp] * 3 + [_vp, _i64] * 5 + [_vp] * 4 + [_vp, _sz, _vp]


_lib.cct_mx_quantize.argtypes = [_i32, _i32, _i32] + [_vp, _i64] * 3 + [_vp]
_lib.cct_mx_dequantize.argtypes = [_i32, _i32, _i32] + [_vp, _i64] * 3 + [_vp]
_lib.cct_mx_linear_workspace_bytes.argtypes = [_lp, _i32, ctypes.POINTER(_sz)]
_lib.cct_mx_linear_forward.argtypes = [_lp] + [_vp, _i64] * 4 + [_vp] + [_vp, _i64] * 3 + [_vp, _sz, _vp]


class MoeDesc(ctypes.Structure):
    """cct_moe_desc_t."""
    _fields_ = [(k, ctypes.c_int32) for k in ("tokens", "experts", "chosen", "D", "F", "type", "activation", "normalize")]


_mp = ctypes.POINTER(MoeDesc)
_lib.cct_moe_workspace_bytes.argtypes = [_mp, ctypes.POINTER(_sz)]
_lib.cct_moe_forward.argtypes = [_mp] + [_vp, _i64] * 2 + [_vp, _i64, _i64] * 3 + [_vp, _i64] * 2 + [_vp, _vp, _vp, _sz, _vp]


class ProfileEntry(ctypes.Structure):
    """cct_profile_entry_t."""
    _fields_ = [("name", ctypes.c_char * 96), ("launches", _i64), ("total_ms", ctypes.c_double),
                ("flops", ctypes.c_double), ("bytes", ctypes.c_double)]


_lib.cct_calibration_copy.argtypes = [_vp, _vp, _sz, _vp]
_lib.cct_profile_enable.argtypes = [ctypes.c_int]
_lib.cct_profile_read.argtypes = [ctypes.POINTER(ProfileEntry), _i32, ctypes.POINTER(_i32)]
for _name in EXPORTS:
    if _name not in ("cct_strerror",):
        getattr(_lib, _name).restype = ctypes.c_int


def make_desc(N, C, H, W, O, K, stride=1, pad=0, groups=1, lowering=LOWER_AUTO,
              precision=PREC_F32) -> ConvDesc:
    return ConvDesc(N, C, H, W, O, K, stride, pad, groups, lowering, precision)


def strerror(code: int) -> str:
    return _lib.cct_strerror(int(code)).decode()


def _check(rc, where):
    if rc != OK:
        raise CctError(rc, where)


def cct_last_hip_error() -> int:
    return int(_lib.cct_last_hip_error())


def cct_conv_output_dims(desc: ConvDesc):
    ho, wo = _i32(), _i32()
    _check(_lib.cct_conv_output_dims(ctypes.byref(desc), ctypes.byref(ho), ctypes.byref(wo)),
           "cct_conv_output_dims")
    return ho.value, wo.value


def cct_lowered_shape(desc: ConvDesc, lowering: int):
    r, c, rc_ = _i64(), _i64(), _i64()
    _check(_lib.cct_lowered_shape(ctypes.byref(desc), int(lowering), ctypes.byref(r),
                                  ctypes.byref(c), ctypes.byref(rc_)), "cct_lowered_shape")
    return r.value, c.value, rc_.value


def cct_lowered_ld(desc: ConvDesc, lowering: int) -> int:
    ld = _i64()
    _check(_lib.cct_lowered_ld(ctypes.byref(desc), int(lowering), ctypes.byref(ld)),
           "cct_lowered_ld")
    return ld.value


def cct_pick_lowering(desc: ConvDesc, pass_: int = PASS_FORWARD) -> int:
    out = ctypes.c_int()
    _check(_lib.cct_pick_lowering(ctypes.byref(desc), int(pass_), ctypes.byref(out)),
           "cct_pick_lowering")
    return out.value


def cct_lowering_cost(desc: ConvDesc, pass_: int, lowering: int) -> float:
    out = ctypes.c_double()
    _check(_lib.cct_lowering_cost(ctypes.byref(desc), int(pass_), int(lowering), ctypes.byref(out)),
           "cct_lowering_cost")
    return out.value


def cct_conv_workspace_bytes(desc: ConvDesc, pass_: int) -> int:
    out = _sz()
    _check(_lib.cct_conv_workspace_bytes(ctypes.byref(desc), int(pass_), ctypes.byref(out)),
           "cct_conv_workspace_bytes")
    return out.value


def cct_conv_workspace_bytes_for_chunk(desc: ConvDesc, pass_: int, images_per_chunk: int) -> int:
    out = _sz()
    _check(_lib.cct_conv_workspace_bytes_for_chunk(ctypes.byref(desc), int(pass_),
                                                   int(images_per_chunk), ctypes.byref(out)),
           "cct_conv_workspace_bytes_for_chunk")
    return out.value


def cct_profile_enable(on: bool) -> None:
    _check(_lib.cct_profile_enable(1 if on else 0), "cct_profile_enable")


def cct_profile_read(max_entries: int = 64):
    """List of dicts (name, launches, total_ms, flops, bytes), one per kernel name."""
    arr = (ProfileEntry * max_entries)()
    n = _i32()
    _check(_lib.cct_profile_read(arr, max_entries, ctypes.byref(n)), "cct_profile_read")
    return [dict(name=arr[i].name.decode(), launches=int(arr[i].launches),
                 total_ms=float(arr[i].total_ms), flops=float(arr[i].flops),
                 bytes=float(arr[i].bytes)) for i in range(n.value)]


def cct_calibration_copy(src, dst) -> None:
    """Plain device copy of src into dst (same-size contiguous GPU tensors)."""
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes or not (src.is_cuda and dst.is_cuda):
        raise ValueError("src and dst must be GPU tensors of the same byte size")
    _check(_lib.cct_calibration_copy(src.data_ptr(), dst.data_ptr(), nbytes, _stream()),
           "cct_calibration_copy")


# ---- device entry points -----------------------------------------------------------------

# A call of a small layer is as long as what happens here and in the launches, so that every tensor is looked at
# with few calls (shapes compare as tuples without a copy), the shapes of a descriptor are asked once per value of
# it, and the stream is asked for its number only (a Stream object for it takes 1.5 us).

def _ptr(t, name, shape=None, optional=False):
    if t is None:
        if optional:
            return None
        raise ValueError("%s is required" % name)
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a torch tensor on the GPU" % name)
    if t.dtype is not torch.float32 or not t.is_contiguous():
        raise TypeError("%s must be contiguous fp32" % name)
    if shape is not None and t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)
if _raw_stream is not None and _device is not None:
    def _stream():  # the tensors of the call have initialised the device
        return _raw_stream(_device())
else:
    def _stream():
        return torch.cuda.current_stream().cuda_stream


def _ws(workspace):
    if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda or \
            workspace.dtype is not torch.uint8 or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous uint8 torch tensor on the GPU")
    return workspace.data_ptr(), workspace.numel()


def alloc_workspace(desc: ConvDesc, pass_: int, images_per_chunk: int | None = None):
    """Caller-side helper: a uint8 device tensor of the queried size."""
    n = cct_conv_workspace_bytes(desc, pass_) if images_per_chunk is None else \
        cct_conv_workspace_bytes_for_chunk(desc, pass_, images_per_chunk)
    return torch.empty(n, dtype=torch.uint8, device="cuda")


@functools.lru_cache(maxsize=1024)
def _shapes_of(fields: bytes):
    desc = ConvDesc.from_buffer_copy(fields)
    ho, wo = cct_conv_output_dims(desc)
    return ((desc.N, desc.C, desc.H, desc.W), (desc.O, desc.C // desc.groups, desc.K, desc.K),
            (desc.N, desc.O, ho, wo))


def _shapes(desc: ConvDesc):
    return _shapes_of(bytes(desc))


def cct_conv_forward(desc: ConvDesc, x, w, bias, y, workspace) -> None:
    xs, ws_, ys = _shapes(desc)
    wp, wn = _ws(workspace)
    _check(_lib.cct_conv_forward(ctypes.byref(desc), _ptr(x, "x", xs), _ptr(w, "w", ws_),
                                 _ptr(bias, "bias", (desc.O,), optional=True), _ptr(y, "y", ys),
                                 wp, wn, _stream()), "cct_conv_forward")


def cct_conv_forward_static(desc: ConvDesc, x, w, bias, y) -> None:
    xs, ws_, ys = _shapes(desc)
    _check(_lib.cct_conv_forward_static(ctypes.byref(desc), _ptr(x, "x", xs), _ptr(w, "w", ws_),
                                        _ptr(bias, "bias", (desc.O,), optional=True),
                                        _ptr(y, "y", ys), _stream()), "cct_conv_forward_static")


def cct_conv_backward_data(desc: ConvDesc, w, dy, dx, workspace) -> None:
    xs, ws_, ys = _shapes(desc)
    wp, wn = _ws(workspace)
    _check(_lib.cct_conv_backward_data(ctypes.byref(desc), _ptr(w, "w", ws_), _ptr(dy, "dy", ys),
                                       _ptr(dx, "dx", xs), wp, wn, _stream()),
           "cct_conv_backward_data")


def cct_conv_backward_weights(desc: ConvDesc, x, dy, dw, dbias, workspace) -> None:
    xs, ws_, ys = _shapes(desc)
    wp, wn = _ws(workspace)
    _check(_lib.cct_conv_backward_weights(ctypes.byref(desc), _ptr(x, "x", xs), _ptr(dy, "dy", ys),
                                          _ptr(dw, "dw", ws_),
                                          _ptr(dbias, "dbias", (desc.O,), optional=True), wp, wn,
                                          _stream()), "cct_conv_backward_weights")


def cct_lower(desc: ConvDesc, lowering: int, x, dhat) -> None:
    xs, _, _ = _shapes(desc)
    _, cols, _ = cct_lowered_shape(desc, lowering)
    ld = cct_lowered_ld(desc, lowering)
    _check(_lib.cct_lower(ctypes.byref(desc), int(lowering), _ptr(x, "x", xs),
                          _ptr(dhat, "dhat", (desc.groups * cols, ld)), _stream()), "cct_lower")


# ---- ReLU and max pooling -------------------------------------------------------------------

def make_pool_desc(N, C, H, W, K, stride, pad=0) -> PoolDesc:
    return PoolDesc(N, C, H, W, K, stride, pad)


def cct_pool_output_dims(desc: PoolDesc):
    ho, wo = _i32(), _i32()
    _check(_lib.cct_pool_output_dims(ctypes.byref(desc), ctypes.byref(ho), ctypes.byref(wo)),
           "cct_pool_output_dims")
    return ho.value, wo.value


@functools.lru_cache(maxsize=1024)
def _pool_shapes_of(fields: bytes):
    desc = PoolDesc.from_buffer_copy(fields)
    ho, wo = cct_pool_output_dims(desc)
    return (desc.N, desc.C, desc.H, desc.W), (desc.N, desc.C, ho, wo)


def cct_relu_forward(x, y) -> None:
    _check(_lib.cct_relu_forward(_ptr(x, "x"), _ptr(y, "y", x.shape), x.numel(), _stream()),
           "cct_relu_forward")


def cct_relu_backward(x, dy, dx) -> None:
    _check(_lib.cct_relu_backward(_ptr(x, "x"), _ptr(dy, "dy", x.shape), _ptr(dx, "dx", x.shape),
                                  x.numel(), _stream()), "cct_relu_backward")


def _iptr(t, name, shape):
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype is not torch.int32 or \
            not t.is_contiguous() or t.shape != shape:
        raise TypeError("%s must be a contiguous int32 GPU tensor of shape %s" % (name, tuple(shape)))
    return t.data_ptr()


def cct_maxpool_forward(desc: PoolDesc, x, y, argmax=None) -> None:
    xs, ys = _pool_shapes_of(bytes(desc))
    _check(_lib.cct_maxpool_forward(ctypes.byref(desc), _ptr(x, "x", xs),
                                    _ptr(y, "y", ys),
                                    None if argmax is None else _iptr(argmax, "argmax", ys),
                                    _stream()), "cct_maxpool_forward")


def cct_maxpool_backward(desc: PoolDesc, dy, argmax, dx) -> None:
    xs, ys = _pool_shapes_of(bytes(desc))
    _check(_lib.cct_maxpool_backward(ctypes.byref(desc), _ptr(dy, "dy", ys), _iptr(argmax, "argmax", ys),
                                     _ptr(dx, "dx", xs), _stream()),
           "cct_maxpool_backward")


def make_lrn_desc(N, C, H, W, size=5, alpha=1e-4, beta=0.75, k=1.0) -> LrnDesc:
    return LrnDesc(N, C, H, W, size, alpha, beta, k)


def cct_lrn_forward(desc: LrnDesc, x, y) -> None:
    shape = (desc.N, desc.C, desc.H, desc.W)
    _check(_lib.cct_lrn_forward(ctypes.byref(desc), _ptr(x, "x", shape), _ptr(y, "y", shape), _stream()),
           "cct_lrn_forward")


def cct_lrn_backward(desc: LrnDesc, x, dy, dx) -> None:
    shape = (desc.N, desc.C, desc.H, desc.W)
    _check(_lib.cct_lrn_backward(ctypes.byref(desc), _ptr(x, "x", shape), _ptr(dy, "dy", shape),
                                 _ptr(dx, "dx", shape), _stream()), "cct_lrn_backward")


def _u8ptr(t, name, shape):
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype is not torch.uint8 or \
            not t.is_contiguous() or t.shape != shape:
        raise TypeError("%s must be a contiguous uint8 GPU tensor of shape %s" % (name, tuple(shape)))
    return t.data_ptr()


def cct_dropout_forward(x, mask, scale, y) -> None:
    _check(_lib.cct_dropout_forward(_ptr(x, "x"), _u8ptr(mask, "mask", x.shape), scale,
                                    _ptr(y, "y", x.shape), x.numel(), _stream()), "cct_dropout_forward")


def cct_dropout_backward(dy, mask, scale, dx) -> None:
    _check(_lib.cct_dropout_backward(_ptr(dy, "dy"), _u8ptr(mask, "mask", dy.shape), scale,
                                     _ptr(dx, "dx", dy.shape), dy.numel(), _stream()),
           "cct_dropout_backward")


def cct_softmax_loss_forward(x, label, prob, image_loss, loss) -> None:
    """x, prob: [N, C] fp32; label: [N] int32; image_loss: [N] fp32; loss: [1] fp32."""
    N, C = x.shape
    _check(_lib.cct_softmax_loss_forward(N, C, _ptr(x, "x"), _iptr(label, "label", (N,)),
                                         _ptr(prob, "prob", (N, C)), _ptr(image_loss, "image_loss", (N,)),
                                         _ptr(loss, "loss", (1,)), _stream()), "cct_softmax_loss_forward")


def cct_softmax_loss_backward(prob, label, dx) -> None:
    N, C = prob.shape
    _check(_lib.cct_softmax_loss_backward(N, C, _ptr(prob, "prob"), _iptr(label, "label", (N,)),
                                          _ptr(dx, "dx", (N, C)), _stream()), "cct_softmax_loss_backward")


# ---- feed-forward blocks ----------------------------------------------------------------------
# A matrix is a two-dimensional tensor whose values are consecutive along a row; its rows may lie further apart.

_DTYPES = (torch.float32, torch.bfloat16, torch.float16)  # by TYPE_*


def make_linear_desc(M, N, K, type=TYPE_F32, activation=ACT_NONE) -> LinearDesc:
    return LinearDesc(M, N, K, type, activation)


def make_gated_desc(M, F, K, type=TYPE_F32, activation=ACT_SILU) -> GatedDesc:
    return GatedDesc(M, F, K, type, activation)


def cct_linear_workspace_bytes(desc: LinearDesc, pass_: int) -> int:
    out = _sz()
    _check(_lib.cct_linear_workspace_bytes(ctypes.byref(desc), int(pass_ != PASS_FORWARD), ctypes.byref(out)),
           "cct_linear_workspace_bytes")
    return out.value


def cct_gated_workspace_bytes(desc: GatedDesc, pass_: int) -> int:
    out = _sz()
    _check(_lib.cct_gated_workspace_bytes(ctypes.byref(desc), int(pass_ != PASS_FORWARD), ctypes.byref(out)),
           "cct_gated_workspace_bytes")
    return out.value


def alloc_linear_workspace(desc: LinearDesc, pass_: int):
    return torch.empty(cct_linear_workspace_bytes(desc, pass_), dtype=torch.uint8, device="cuda")


def alloc_gated_workspace(desc: GatedDesc, pass_: int):
    return torch.empty(cct_gated_workspace_bytes(desc, pass_), dtype=torch.uint8, device="cuda")


def _mat(t, name, rows, cols, dtype, optional=False):
    """Address and row stride of a matrix."""
    if t is None:
        if optional:
            return None, 0
        raise ValueError("%s is required" % name)
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a torch tensor on the GPU" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    if t.shape != (rows, cols):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), (rows, cols)))
    ld, one = t.stride()
    if one != 1 and cols > 1:
        raise TypeError("%s must have consecutive values along a row" % name)
    if rows <= 1:
        ld = cols
    elif ld < cols:
        raise TypeError("%s has rows that overlap" % name)
    return t.data_ptr(), ld


def _vec(t, name, n, dtype):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype is not dtype or t.shape != (n,) or \
            not t.is_contiguous():
        raise TypeError("%s must be a contiguous %s GPU tensor of shape (%d,)" % (name, dtype, n))
    return t.data_ptr()


def _dtype_of(desc):
    if not 0 <= desc.type < len(_DTYPES):
        raise CctError(EINVAL, "type %d" % desc.type)
    return _DTYPES[desc.type]


def cct_linear_forward(desc: LinearDesc, x, w, bias, residual, y, z, workspace) -> None:
    """y = act(x w^T + bias) + residual; bias, residual and z (the product before the activation) may be None."""
    M, N, K, dt = desc.M, desc.N, desc.K, _dtype_of(desc)
    _check(_lib.cct_linear_forward(
        ctypes.byref(desc), *_mat(x, "x", M, K, dt), *_mat(w, "w", N, K, dt), _vec(bias, "bias", N, dt),
        *_mat(residual, "residual", M, N, dt, True), *_mat(y, "y", M, N, dt), *_mat(z, "z", M, N, dt, True),
        *_ws(workspace), _stream()), "cct_linear_forward")


def cct_linear_backward(desc: LinearDesc, x, w, z, dy, dx, dw, dbias, workspace) -> None:
    """dx, dw and dbias from dy; each may be None, then x (without dw) and w (without dx) may be too."""
    M, N, K, dt = desc.M, desc.N, desc.K, _dtype_of(desc)
    _check(_lib.cct_linear_backward(
        ctypes.byref(desc), *_mat(x, "x", M, K, dt, dw is None), *_mat(w, "w", N, K, dt, dx is None),
        *_mat(z, "z", M, N, dt, True), *_mat(dy, "dy", M, N, dt), *_mat(dx, "dx", M, K, dt, True),
        *_mat(dw, "dw", N, K, dt, True), _vec(dbias, "dbias", N, dt), *_ws(workspace), _stream()),
        "cct_linear_backward")


def cct_gated_forward(desc: GatedDesc, x, wg, wu, h, g, u, workspace) -> None:
    """h = act(x wg^T) * (x wu^T); g and u, the two products, are kept if given."""
    M, F, K, dt = desc.M, desc.F, desc.K, _dtype_of(desc)
    _check(_lib.cct_gated_forward(
        ctypes.byref(desc), *_mat(x, "x", M, K, dt), *_mat(wg, "wg", F, K, dt), *_mat(wu, "wu", F, K, dt),
        *_mat(h, "h", M, F, dt), *_mat(g, "g", M, F, dt, True), *_mat(u, "u", M, F, dt, True), *_ws(workspace),
        _stream()), "cct_gated_forward")


def cct_gated_backward(desc: GatedDesc, x, wg, wu, g, u, dh, dx, dwg, dwu, workspace) -> None:
    """dx, dwg and dwu from dh and the products that the forward pass kept."""
    M, F, K, dt = desc.M, desc.F, desc.K, _dtype_of(desc)
    none = dx is None
    _check(_lib.cct_gated_backward(
        ctypes.byref(desc), *_mat(x, "x", M, K, dt, dwg is None), *_mat(wg, "wg", F, K, dt, none),
        *_mat(wu, "wu", F, K, dt, none), *_mat(g, "g", M, F, dt), *_mat(u, "u", M, F, dt), *_mat(dh, "dh", M, F, dt),
        *_mat(dx, "dx", M, K, dt, True), *_mat(dwg, "dwg", F, K, dt, True), *_mat(dwu, "dwu", F, K, dt, True),
        *_ws(workspace), _stream()), "cct_gated_backward")


# ---- norms and gates on a residual stream -------------------------------------------------------

def make_residual_norm_desc(M, D, type=TYPE_F32, before=NORM_RMS, after=NORM_NONE, gate_rows=1, eps=1e-6,
                            scale=1.0) -> ResidualNormDesc:
    return ResidualNormDesc(M, D, type, before, after, gate_rows, eps, scale)


def cct_residual_norm_workspace_bytes(desc: ResidualNormDesc) -> int:
    """Of the backward pass; the forward pass needs none."""
    out = _sz()
    _check(_lib.cct_residual_norm_workspace_bytes(ctypes.byref(desc), ctypes.byref(out)),
           "cct_residual_norm_workspace_bytes")
    return out.value


def alloc_residual_norm_workspace(desc: ResidualNormDesc):
    return torch.empty(cct_residual_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda")


def _gate_count(desc):
    return -(-desc.M // max(1, desc.gate_rows))


def cct_residual_norm_forward(desc: ResidualNormDesc, r, b, gate, w_after, c_after, w_before, c_before, s, h) -> None:
    """s = r + scale * gate * N_after(b), h = N_before(s); b, gate, the norms' vectors, and s or h may be None.  gate: a row
    for each gate_rows rows of r."""
    M, D, dt = desc.M, desc.D, _dtype_of(desc)
    _check(_lib.cct_residual_norm_forward(
        ctypes.byref(desc), *_mat(r, "r", M, D, dt), *_mat(b, "b", M, D, dt, True),
        *_mat(gate, "gate", _gate_count(desc), D, dt, True), _vec(w_after, "w_after", D, dt),
        _vec(c_after, "c_after", D, dt), _vec(w_before, "w_before", D, dt), _vec(c_before, "c_before", D, dt),
        *_mat(s, "s", M, D, dt, True), *_mat(h, "h", M, D, dt, True), _stream()), "cct_residual_norm_forward")


def cct_residual_norm_backward(desc: ResidualNormDesc, s, b, gate, w_after, c_after, w_before, ds, dh, dr, db, dgate,
                               dw_after, dc_after, dw_before, dc_before, workspace) -> None:
    """The gradients of r, b, the gate and the norms' vectors, each of which may be None, from those of s and h."""
    M, D, dt, n = desc.M, desc.D, _dtype_of(desc), _gate_count(desc)
    _check(_lib.cct_residual_norm_backward(
        ctypes.byref(desc), *_mat(s, "s", M, D, dt, True), *_mat(b, "b", M, D, dt, True),
        *_mat(gate, "gate", n, D, dt, True), _vec(w_after, "w_after", D, dt), _vec(c_after, "c_after", D, dt),
        _vec(w_before, "w_before", D, dt), *_mat(ds, "ds", M, D, dt, True), *_mat(dh, "dh", M, D, dt, True),
        *_mat(dr, "dr", M, D, dt, True), *_mat(db, "db", M, D, dt, True), *_mat(dgate, "dgate", n, D, dt, True),
        _vec(dw_after, "dw_after", D, dt), _vec(dc_after, "dc_after", D, dt), _vec(dw_before, "dw_before", D, dt),
        _vec(dc_before, "dc_before", D, dt), *_ws(workspace), _stream()), "cct_residual_norm_backward")


# ---- microscaled 4-bit floating point -------------------------------------------------------------

class MxMatrix:
    """A matrix in microscaled 4-bit floating point: codes (rows x 16 bytes for each 32 columns) and scales (rows x a multiple
    of 4 bytes, one for each 32 columns), uint8 tensors on the GPU, allocated here where they are not given."""

    def __init__(self, rows, cols, codes=None, scales=None):
        self.rows, self.cols = rows, cols
        blocks = -(-cols // 32)
        shapes = ((rows, blocks * 16), (rows, -(-blocks // 4) * 4))
        given = [torch.empty(s, dtype=torch.uint8, device="cuda") if t is None else t for t, s in
                 zip((codes, scales), shapes)]
        self.codes, self.scales = given
        self.codes_at, self.scales_at = (_mat(t, n, *s, torch.uint8) for t, n, s in
                                         zip(given, ("codes", "scales"), shapes))


def _mx(m, name, rows, cols):
    if not isinstance(m, MxMatrix):
        raise TypeError("%s must be an MxMatrix" % name)
    if (m.rows, m.cols) != (rows, cols):
        raise ValueError("%s is %d x %d, expected %d x %d" % (name, m.rows, m.cols, rows, cols))
    return (*m.codes_at, *m.scales_at)


def _type_of(t, name):
    if not isinstance(t, torch.Tensor) or t.dtype not in _DTYPES or t.dim() != 2:
        raise TypeError("%s must be a matrix of fp32, bf16 or fp16" % name)
    return _DTYPES.index(t.dtype)


def cct_mx_quantize(x, mx: MxMatrix) -> None:
    """x (fp32, bf16 or fp16) rounded to microscaled 4 bits."""
    ty = _type_of(x, "x")
    _check(_lib.cct_mx_quantize(mx.rows, mx.cols, ty, *_mat(x, "x", mx.rows, mx.cols, x.dtype),
                                *_mx(mx, "mx", mx.rows, mx.cols), _stream()), "cct_mx_quantize")


def cct_mx_dequantize(mx: MxMatrix, x) -> None:
    """The values of mx in x's type."""
    ty = _type_of(x, "x")
    _check(_lib.cct_mx_dequantize(mx.rows, mx.cols, ty, *_mx(mx, "mx", mx.rows, mx.cols),
                                  *_mat(x, "x", mx.rows, mx.cols, x.dtype), _stream()), "cct_mx_dequantize")


def cct_mx_linear_workspace_bytes(desc: LinearDesc, quantize: bool) -> int:
    out = _sz()
    _check(_lib.cct_mx_linear_workspace_bytes(ctypes.byref(desc), int(quantize), ctypes.byref(out)),
           "cct_mx_linear_workspace_bytes")
    return out.value


def alloc_mx_linear_workspace(desc: LinearDesc, quantize: bool = True):
    return torch.empty(cct_mx_linear_workspace_bytes(desc, quantize), dtype=torch.uint8, device="cuda")


def cct_mx_linear_forward(desc: LinearDesc, x, w: MxMatrix, bias, residual, y, z, workspace) -> None:
    """y = act(x w^T + bias) + residual; x is an MxMatrix, or a tensor that is quantised first."""
    M, N, K, dt = desc.M, desc.N, desc.K, _dtype_of(desc)
    at = _mx(x, "x", M, K) if isinstance(x, MxMatrix) else (*_mat(x, "x", M, K, dt), None, 0)
    _check(_lib.cct_mx_linear_forward(
        ctypes.byref(desc), *at, *_mx(w, "w", N, K), _vec(bias, "bias", N, dt),
        *_mat(residual, "residual", M, N, dt, True), *_mat(y, "y", M, N, dt), *_mat(z, "z", M, N, dt, True),
        *_ws(workspace), _stream()), "cct_mx_linear_forward")


# ---- experts ----------------------------------------------------------------------------------------

def make_moe_desc(tokens, experts, chosen, D, F, type=TYPE_F32, activation=ACT_SILU, normalize=True) -> MoeDesc:
    return MoeDesc(tokens, experts, chosen, D, F, type, activation, int(normalize))


def cct_moe_workspace_bytes(desc: MoeDesc) -> int:
    out = _sz()
    _check(_lib.cct_moe_workspace_bytes(ctypes.byref(desc), ctypes.byref(out)), "cct_moe_workspace_bytes")
    return out.value


def alloc_moe_workspace(desc: MoeDesc):
    return torch.empty(cct_moe_workspace_bytes(desc), dtype=torch.uint8, device="cuda")


def _experts(t, name, E, rows, cols, dtype):
    """Address, row stride and expert stride of a tensor of matrices."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a torch tensor on the GPU" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    if t.shape != (E, rows, cols):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), (E, rows, cols)))
    apart, ld, one = t.stride()
    if one != 1 and cols > 1:
        raise TypeError("%s must have consecutive values along a row" % name)
    if rows <= 1:
        ld = cols
    elif ld < cols:
        raise TypeError("%s has rows that overlap" % name)
    if E <= 1:
        apart = rows * ld
    elif apart < (rows - 1) * ld + cols:
        raise TypeError("%s has experts that overlap" % name)
    return t.data_ptr(), ld, apart


def _out(t, name, shape, dtype):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype is not dtype or t.shape != shape or \
            not t.is_contiguous():
        raise TypeError("%s must be a contiguous %s GPU tensor of shape %s" % (name, dtype, shape))
    return t.data_ptr()


def cct_moe_forward(desc: MoeDesc, x, router, wg, wu, wd, residual, y, chosen, weights, workspace) -> None:
    """y = the chosen experts' weighted sum (+ residual); chosen (int32) and weights (fp32), tokens x chosen, may be None.
    wg, wu: experts x F x D, wd: experts x D x F."""
    T, E, k, D, F, dt = desc.tokens, desc.experts, desc.chosen, desc.D, desc.F, _dtype_of(desc)
    _check(_lib.cct_moe_forward(
        ctypes.byref(desc), *_mat(x, "x", T, D, dt), *_mat(router, "router", E, D, dt), *_experts(wg, "wg", E, F, D, dt),
        *_experts(wu, "wu", E, F, D, dt), *_experts(wd, "wd", E, D, F, dt), *_mat(residual, "residual", T, D, dt, True),
        *_mat(y, "y", T, D, dt), _out(chosen, "chosen", (T, k), torch.int32), _out(weights, "weights", (T, k), torch.float32),
        *_ws(workspace), _stream()), "cct_moe_forward")


# ---- gradient norm and weight update ------------------------------------------------------------

class TensorList:
    """The tensors of a list and their descriptors, made once and passed to any number of calls.  The tensors are
    held: their addresses stay valid as long as the list lives (do not resize them)."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        for i, t in enumerate(self.tensors):
            if not isinstance(t, torch.Tensor) or not t.is_cuda:
                raise TypeError("tensor %d must be a torch tensor on the GPU" % i)
            if t.dtype not in _DTYPES or not t.is_contiguous():
                raise TypeError("tensor %d must be contiguous fp32, bf16 or fp16" % i)
        self.count = len(self.tensors)
        self.array = (Tensor * max(1, self.count))(
            *(Tensor(t.data_ptr(), t.numel(), _DTYPES.index(t.dtype), 0) for t in self.tensors))


def make_tensor_list(tensors) -> TensorList:
    return TensorList(tensors)


def cct_grad_norm_workspace_bytes(grads: TensorList) -> int:
    out = _sz()
    _check(_lib.cct_grad_norm_workspace_bytes(grads.array, grads.count, ctypes.byref(out)),
           "cct_grad_norm_workspace_bytes")
    return out.value


def alloc_norm_workspace(grads: TensorList):
    return torch.empty(cct_grad_norm_workspace_bytes(grads), dtype=torch.uint8, device="cuda")


def _same(a: TensorList, b: TensorList, name):
    if b.count != a.count:
        raise ValueError("%s has %d tensors, expected %d" % (name, b.count, a.count))
    return b.array


def cct_grad_norm(grads: TensorList, max_norm, clip, workspace) -> None:
    """clip (2 fp32 values on the GPU): the norm of all gradients, and what they are to be multiplied by."""
    _check(_lib.cct_grad_norm(grads.array, grads.count, max_norm, _ptr(clip, "clip", (2,)), *_ws(workspace),
                              _stream()), "cct_grad_norm")


def cct_grad_scale(grads: TensorList, clip, out: TensorList) -> None:
    """out = grads * clip[1]; out may be grads itself."""
    _check(_lib.cct_grad_scale(grads.array, grads.count, _ptr(clip, "clip", (2,)), _same(grads, out, "out"),
                               _stream()), "cct_grad_scale")


def cct_sgd_update(grads: TensorList, clip, weights: TensorList, moments: TensorList, copies, rate, momentum=0.9,
                   decay=0.0) -> None:
    """One step of the weights, in place; clip may be None, copies too (else: the weights in other types)."""
    _check(_lib.cct_sgd_update(grads.array, grads.count, _ptr(clip, "clip", (2,), optional=True),
                               _same(grads, weights, "weights"), _same(grads, moments, "moments"),
                               None if copies is None else _same(grads, copies, "copies"), rate, momentum, decay,
                               _stream()), "cct_sgd_update")
