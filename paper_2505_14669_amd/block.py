"""Binding of include/quartet_block.h: what a transformer block runs around the quantized linear layers.

As binding.py: every function has the name and argument order of its C entry point, takes torch CUDA tensors (or raw device
addresses) for the pointer arguments and returns the C return code, which `check()` turns into an exception.  No arithmetic here.
"""
import ctypes

from . import binding as _q
from .binding import (QUARTET_DTYPE_BF16, QUARTET_DTYPE_F32, QUARTET_EHIP, QUARTET_EINVAL, QUARTET_ENOTSUP, QUARTET_OK,  # noqa: F401
                      QuartetError, check)

QUARTET_ACT_NONE = 0
QUARTET_ACT_RELU = 1
QUARTET_ACT_GELU = 2
QUARTET_ACT_SILU = 3
ACTIVATIONS = {"none": QUARTET_ACT_NONE, "relu": QUARTET_ACT_RELU, "gelu": QUARTET_ACT_GELU, "silu": QUARTET_ACT_SILU}
QUARTET_FORMAT_NONE = 0
QUARTET_FORMAT_MXFP4 = 1
QUARTET_FORMAT_MXFP8 = 2
QUARTET_KIND_NORM = 8
QUARTET_KIND_ACT = 9
QUARTET_KIND_CLIP = 10

EXPORTS = ["quartet_mxfp4_gemm_act", "quartet_act_bwd_workspace_bytes", "quartet_act_bwd", "quartet_rmsnorm_fwd", "quartet_rmsnorm_bwd_workspace_bytes",
           "quartet_rmsnorm_bwd", "quartet_grad_clip_workspace_bytes", "quartet_grad_clip"]

_lib, _ptr, _stream = _q._lib, _q._ptr, _q._stream
_i64, _p, _int, _f, _size = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
_lib.quartet_mxfp4_gemm_act.argtypes = [_p, _p, _p, _p, _i64, _i64, _i64, _f, _p, _int, _int, _p, _i64, _p, _int, _i64, _p, _i64, _p, _int, _i64, _p]
_lib.quartet_act_bwd_workspace_bytes.restype = _size
_lib.quartet_act_bwd_workspace_bytes.argtypes = [_i64, _i64]
_lib.quartet_act_bwd.argtypes = [_p, _i64, _p, _i64, _p, _i64, _i64, _i64, _int, _p, _i64, _p, _i64, _p, _p, _size, _p]
_lib.quartet_rmsnorm_fwd.argtypes = [_p, _int, _i64, _p, _i64, _i64, _i64, _p, _int, _f, _p, _int, _i64, _p, _i64, _int, _p, _p, _p, _p, _p]
_lib.quartet_rmsnorm_bwd_workspace_bytes.restype = _size
_lib.quartet_rmsnorm_bwd_workspace_bytes.argtypes = [_i64, _i64]
_lib.quartet_rmsnorm_bwd.argtypes = [_p, _i64, _p, _int, _i64, _i64, _i64, _p, _int, _p, _p, _i64, _p, _i64, _p, _i64, _p, _p, _size, _p]


class GradTensor(ctypes.Structure):
    """quartet_grad_tensor: one gradient and its copy (host structure of device pointers)"""
    _fields_ = [("grad", _p), ("out", _p), ("size", _i64), ("grad_dtype", _int), ("out_dtype", _int)]


_lib.quartet_grad_clip_workspace_bytes.restype = _size
_lib.quartet_grad_clip_workspace_bytes.argtypes = []
_lib.quartet_grad_clip.argtypes = [_p, _i64, _f, _p, _p, _size, _p]


# Calls go through the torch node where that takes the arguments (binding.py says why), else through ctypes.

def quartet_mxfp4_gemm_act(a_codes, a_scales, b_codes, b_scales, m, n, k, alpha, bias, bias_dtype, activation, multiplier_bf16, ldmul, residual,
                           residual_dtype, ldres, pre_bf16, ldpre, d, d_dtype, ldd, stream=None):
    if _q._native is not None:
        rc = _q._native.quartet_mxfp4_gemm_act(a_codes, a_scales, b_codes, b_scales, m, n, k, alpha, bias, bias_dtype, activation, multiplier_bf16,
                                               ldmul, residual, residual_dtype, ldres, pre_bf16, ldpre, d, d_dtype, ldd, stream)
        if rc is not NotImplemented:
            return rc
    return _lib.quartet_mxfp4_gemm_act(_ptr(a_codes), _ptr(a_scales), _ptr(b_codes), _ptr(b_scales), m, n, k, alpha, _ptr(bias), bias_dtype,
                                       activation, _ptr(multiplier_bf16), ldmul, _ptr(residual), residual_dtype, ldres, _ptr(pre_bf16), ldpre,
                                       _ptr(d), d_dtype, ldd, _stream(stream))


def quartet_act_bwd_workspace_bytes(m, n):
    return _lib.quartet_act_bwd_workspace_bytes(m, n)


def quartet_act_bwd(dy_bf16, lddy, pre_bf16, ldpre, multiplier_bf16, ldmul, m, n, activation, dz_bf16, lddz, dmul_bf16, lddmul, dbias, workspace,
                    workspace_bytes, stream=None):
    if _q._native is not None:
        rc = _q._native.quartet_act_bwd(dy_bf16, lddy, pre_bf16, ldpre, multiplier_bf16, ldmul, m, n, activation, dz_bf16, lddz, dmul_bf16, lddmul,
                                        dbias, workspace, workspace_bytes, stream)
        if rc is not NotImplemented:
            return rc
    return _lib.quartet_act_bwd(_ptr(dy_bf16), lddy, _ptr(pre_bf16), ldpre, _ptr(multiplier_bf16), ldmul, m, n, activation, _ptr(dz_bf16), lddz,
                                _ptr(dmul_bf16), lddmul, _ptr(dbias), _ptr(workspace), workspace_bytes, _stream(stream))


def quartet_rmsnorm_fwd(x, x_dtype, ldx, residual, ldres, rows, n, weight, weight_dtype, eps, h, h_dtype, ldh, y_bf16, ldy, format, codes, scales, mask,
                        rstd, stream=None):
    if _q._native is not None:
        rc = _q._native.quartet_rmsnorm_fwd(x, x_dtype, ldx, residual, ldres, rows, n, weight, weight_dtype, eps, h, h_dtype, ldh, y_bf16, ldy,
                                            format, codes, scales, mask, rstd, stream)
        if rc is not NotImplemented:
            return rc
    return _lib.quartet_rmsnorm_fwd(_ptr(x), x_dtype, ldx, _ptr(residual), ldres, rows, n, _ptr(weight), weight_dtype, eps, _ptr(h), h_dtype, ldh,
                                    _ptr(y_bf16), ldy, format, _ptr(codes), _ptr(scales), _ptr(mask), _ptr(rstd), _stream(stream))


def quartet_rmsnorm_bwd_workspace_bytes(rows, n):
    return _lib.quartet_rmsnorm_bwd_workspace_bytes(rows, n)


def quartet_rmsnorm_bwd(dy_bf16, lddy, h, h_dtype, ldh, rows, n, weight, weight_dtype, rstd, dh, lddh, dx, lddx, dx16, lddx16, dweight, workspace,
                        workspace_bytes, stream=None):
    if _q._native is not None:
        rc = _q._native.quartet_rmsnorm_bwd(dy_bf16, lddy, h, h_dtype, ldh, rows, n, weight, weight_dtype, rstd, dh, lddh, dx, lddx, dx16, lddx16,
                                            dweight, workspace, workspace_bytes, stream)
        if rc is not NotImplemented:
            return rc
    return _lib.quartet_rmsnorm_bwd(_ptr(dy_bf16), lddy, _ptr(h), h_dtype, ldh, rows, n, _ptr(weight), weight_dtype, _ptr(rstd), _ptr(dh), lddh,
                                    _ptr(dx), lddx, _ptr(dx16), lddx16, _ptr(dweight), _ptr(workspace), workspace_bytes, _stream(stream))


class GradTensors:
    """The `tensors` argument of quartet_grad_clip: an array of quartet_grad_tensor on the host, which keeps the torch tensors in it alive."""

    def __init__(self, pairs):
        self.kept = list(pairs)
        self.array = (GradTensor * max(1, len(self.kept)))()
        for entry, (g, out) in zip(self.array, self.kept):
            entry.grad, entry.out, entry.size = _ptr(g), _ptr(out), g.numel()
            entry.grad_dtype, entry.out_dtype = _dtype(g), _dtype(out)
        self.address = ctypes.addressof(self.array)

    def __len__(self):
        return len(self.kept)


def _dtype(t):
    import torch
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise QuartetError(f"gradients and their copies are fp32 or bf16, not {t.dtype}")
    return QUARTET_DTYPE_F32 if t.dtype == torch.float32 else QUARTET_DTYPE_BF16


def grad_tensors(grads, outs=None):
    """The list of quartet_grad_clip for contiguous CUDA tensors; outs: their copies (default: scaled in place).  May be kept while they live."""
    grads = list(grads)
    outs = grads if outs is None else list(outs)
    if len(grads) != len(outs) or any(g.numel() != o.numel() for g, o in zip(grads, outs)):
        raise QuartetError("every gradient needs a copy of its size")
    return GradTensors(zip(grads, outs))


def quartet_grad_clip_workspace_bytes():
    return _lib.quartet_grad_clip_workspace_bytes()


def quartet_grad_clip(tensors, count, max_norm, norm, workspace, workspace_bytes, stream=None):
    address = tensors.address if isinstance(tensors, GradTensors) else tensors
    if _q._native is not None:
        rc = _q._native.quartet_grad_clip(address, count, max_norm, norm, workspace, workspace_bytes, stream)
        if rc is not NotImplemented:
            return rc
    return _lib.quartet_grad_clip(address, count, max_norm, _ptr(norm), _ptr(workspace), workspace_bytes, _stream(stream))


for _name in EXPORTS:
    getattr(_lib, _name)  # AttributeError here = the library does not export what the header declares
