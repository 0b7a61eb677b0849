"""ctypes binding of the operators of ``libhpsgd.so`` (``include/hpsgd_ops.h``): same names as the C ABI, argument
marshalling only.  What a call needs every time (a table of tensors, an argument block) is built once by a ``make_*``
function and passed again and again; the buffers it names have to stay alive, which the returned object sees to.

A call goes to the ``stream`` it is given (0 is CUDA's legacy default stream); left out, to torch's current stream where the
process uses torch on CUDA, so that it is ordered with the torch operations around it.
"""
from __future__ import annotations

import ctypes
import sys

from . import binding as _b
from .binding import _ci, _f64, _i64, _ptr, _stream, _u64, _vp

__all__ = ["HPSGD_GRAD_NORM_WORKSPACE", "HPSGD_FP8", "hpsgd_adamw_tensor", "make_adamw_table", "hpsgd_adamw_step", "hpsgd_grad_norm",
           "make_rmsnorm_forward", "hpsgd_rmsnorm_forward", "make_rmsnorm_backward", "hpsgd_rmsnorm_backward", "hpsgd_rmsnorm_backward_bytes",
           "make_quantize_fp8", "hpsgd_quantize_fp8", "make_gemm_fp8", "hpsgd_gemm_fp8", "hpsgd_gemm_fp8_bytes", "hpsgd_ops_check",
           "hpsgd_ops_debug_stall"]

HPSGD_GRAD_NORM_WORKSPACE = 65536
HPSGD_FP8 = 2


class hpsgd_adamw_tensor(ctypes.Structure):
    _fields_ = [("param", _vp), ("grad", _vp), ("m", _vp), ("v", _vp), ("m_scale", _vp), ("v_scale", _vp), ("copy", _vp),
                ("n", _i64), ("rng_offset", _u64), ("weight_decay", _f64)]


class hpsgd_rmsnorm_forward_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("eps", _f64), ("dtype", _ci), ("weight_dtype", _ci)] + \
        [(n, _vp) for n in ("x", "residual", "weight", "h", "y", "y8", "y_scale", "rstd")] + \
        [(n, _i64) for n in ("ldx", "ldres", "ldh", "ldy", "ldy8", "ldys")]


class hpsgd_rmsnorm_backward_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("dtype", _ci), ("weight_dtype", _ci)] + \
        [(n, _vp) for n in ("h", "weight", "rstd", "dy", "dres", "dx", "dweight", "workspace")] + \
        [(n, _i64) for n in ("ldh", "lddy", "lddres", "lddx")]


class hpsgd_quantize_fp8_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("dtype", _ci)] + \
        [(n, _vp) for n in ("x", "x_scale", "q", "scale", "qt", "scale_t")] + \
        [(n, _i64) for n in ("ldx", "ldxs", "ldq", "lds", "ldqt", "ldst")]


class hpsgd_gemm_fp8_args(ctypes.Structure):
    _fields_ = [(n, _i64) for n in ("M", "N", "K")] + [(n, _vp) for n in ("a", "a_scale", "b", "b_scale", "d", "workspace")] + \
        [("workspace_bytes", ctypes.c_size_t)] + [(n, _i64) for n in ("lda", "ldsa", "ldb", "ldsb", "ldd")] + [("d_dtype", _ci), ("accumulate", _ci)]


SIGNATURES = {
    "hpsgd_gemm_fp8_bytes": (ctypes.c_size_t, [_i64, _i64, _i64]),
    "hpsgd_gemm_fp8": (_ci, [_vp, _vp]),
    "hpsgd_ops_check": (_ci, [_vp]),
    "hpsgd_ops_debug_stall": (_ci, [_ci]),
    "hpsgd_rmsnorm_forward": (_ci, [_vp, _vp]),
    "hpsgd_rmsnorm_backward_bytes": (ctypes.c_size_t, [_i64, _i64]),
    "hpsgd_rmsnorm_backward": (_ci, [_vp, _vp]),
    "hpsgd_quantize_fp8": (_ci, [_vp, _vp]),
    "hpsgd_adamw_step": (_ci, [_vp, _ci, _ci, _ci, _ci, _f64, _f64, _f64, _f64, _i64, _u64, _vp, _vp]),
    "hpsgd_grad_norm": (_ci, [_vp, _ci, _ci, _f64, _vp, _vp, _vp]),
}


def _on(stream):
    """The stream of a call: the one that is given, or torch's current one."""
    if stream is not None:
        return _stream(stream)
    torch = sys.modules.get("torch")
    if torch is None or not torch.cuda.is_initialized():
        return None
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # a tenth of the time that a Stream object takes (0.2 against 3.3 us)
    return raw(torch._C._cuda_getDevice()) if raw else torch.cuda.current_stream().cuda_stream


# ---- AdamW over many tensors -----------------------------------------------------------
class AdamWTable:
    """The tensors of a step (see make_adamw_table)."""

    def __init__(self, rows, param_dtype, grad_dtype, state_bits):
        self.array = (hpsgd_adamw_tensor * len(rows))()
        self.address = ctypes.addressof(self.array)
        self.count, self.param_dtype, self.grad_dtype, self.state_bits = len(rows), int(param_dtype), int(grad_dtype), int(state_bits)
        self.keep = rows


def make_adamw_table(rows, param_dtype, grad_dtype, state_bits):
    """A table for hpsgd_adamw_step / hpsgd_grad_norm from dicts with the fields of ``hpsgd_adamw_tensor`` (tensors or addresses;
    what is left out is NULL or 0).  ``rng_offset`` left out: the tensors follow one another in the order given."""
    table = AdamWTable(list(rows), param_dtype, grad_dtype, state_bits)
    names = {f[0] for f in hpsgd_adamw_tensor._fields_}
    at = 0
    for item, row in zip(table.array, table.keep):
        unknown = set(row) - names
        if unknown:
            raise TypeError("not a field of hpsgd_adamw_tensor: %s" % sorted(unknown))
        for name in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy"):
            setattr(item, name, _ptr(row.get(name)))
        item.n = int(row["n"])
        item.weight_decay = float(row.get("weight_decay", 0.0))
        item.rng_offset = int(row.get("rng_offset", at))
        at = item.rng_offset + item.n
    return table


def hpsgd_adamw_step(table, lr, beta1, beta2, eps, step, seed=0, grad_scale=None, stream=None):
    return _b._check(_b.load().hpsgd_adamw_step(table.address, table.count, table.param_dtype, table.grad_dtype, table.state_bits,
                                                lr, beta1, beta2, eps, step, seed, _ptr(grad_scale), _on(stream)))


def hpsgd_grad_norm(table, max_norm, workspace, out, stream=None):
    return _b._check(_b.load().hpsgd_grad_norm(table.address, table.count, table.grad_dtype, max_norm, _ptr(workspace), _ptr(out),
                                               _on(stream)))


# ---- argument blocks -------------------------------------------------------------------
class Args:
    """A filled argument struct with its address, and what it points to."""

    def __init__(self, struct, pointers, strides, **plain):
        self.struct, self.keep = struct(), pointers
        kinds = dict(struct._fields_)
        for name, value in pointers.items():
            setattr(self.struct, name, _ptr(value))
        for name, value in {**strides, **plain}.items():
            if name not in kinds or kinds[name] is _vp:
                raise TypeError("not a field of %s: %s" % (struct.__name__, name))
            setattr(self.struct, name, value)
        self.address = ctypes.addressof(self.struct)


def make_rmsnorm_forward(rows, cols, eps, dtype, x, weight, residual=None, h=None, y=None, y8=None, y_scale=None, rstd=None,
                         weight_dtype=None, **strides):
    return Args(hpsgd_rmsnorm_forward_args, dict(x=x, residual=residual, weight=weight, h=h, y=y, y8=y8, y_scale=y_scale, rstd=rstd), strides,
                rows=rows, cols=cols, eps=eps, dtype=dtype, weight_dtype=dtype if weight_dtype is None else weight_dtype)


def hpsgd_rmsnorm_forward(args, stream=None):
    return _b._check(_b.load().hpsgd_rmsnorm_forward(args.address, _on(stream)))


def hpsgd_rmsnorm_backward_bytes(rows, cols):
    return int(_b.load().hpsgd_rmsnorm_backward_bytes(rows, cols))


def make_rmsnorm_backward(rows, cols, dtype, h, weight, rstd, dy, dx, dweight, workspace, dres=None, weight_dtype=None, **strides):
    return Args(hpsgd_rmsnorm_backward_args, dict(h=h, weight=weight, rstd=rstd, dy=dy, dres=dres, dx=dx, dweight=dweight, workspace=workspace),
                strides, rows=rows, cols=cols, dtype=dtype, weight_dtype=dtype if weight_dtype is None else weight_dtype)


def hpsgd_rmsnorm_backward(args, stream=None):
    return _b._check(_b.load().hpsgd_rmsnorm_backward(args.address, _on(stream)))


def make_quantize_fp8(rows, cols, dtype, x, q=None, scale=None, qt=None, scale_t=None, x_scale=None, **strides):
    return Args(hpsgd_quantize_fp8_args, dict(x=x, x_scale=x_scale, q=q, scale=scale, qt=qt, scale_t=scale_t), strides,
                rows=rows, cols=cols, dtype=dtype)


def hpsgd_quantize_fp8(args, stream=None):
    return _b._check(_b.load().hpsgd_quantize_fp8(args.address, _on(stream)))


def hpsgd_gemm_fp8_bytes(M, N, K):
    return int(_b.load().hpsgd_gemm_fp8_bytes(M, N, K))


def make_gemm_fp8(M, N, K, a, a_scale, b, b_scale, d, d_dtype, accumulate=False, workspace=None, workspace_bytes=None, **strides):
    """``workspace_bytes`` left out: the size of the tensor given as workspace."""
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    return Args(hpsgd_gemm_fp8_args, dict(a=a, a_scale=a_scale, b=b, b_scale=b_scale, d=d, workspace=workspace), strides,
                M=M, N=N, K=K, d_dtype=d_dtype, accumulate=int(accumulate), workspace_bytes=workspace_bytes)


def hpsgd_gemm_fp8(args, stream=None):
    return _b._check(_b.load().hpsgd_gemm_fp8(args.address, _on(stream)))


def hpsgd_ops_check(stream=None):
    return _b._check(_b.load().hpsgd_ops_check(_on(stream)))


def hpsgd_ops_debug_stall(enable):
    return _b._check(_b.load().hpsgd_ops_debug_stall(int(enable)))
