"""ctypes binding of the operators of ``libhpsgd.so`` (``include/hpsgd_ops.h``): same names as the C ABI, argument
marshalling only.  What a call needs every time (a table of tensors, an argument block) is built once by a ``make_*``
function and passed again and again; the buffers it names have to stay alive, which the returned object sees to.

Tensors are checked when they are named: on a CUDA device, of the type that the call reads there, rows of consecutive elements as far apart
as the call is told, and as much memory as it will touch (HPSGD_E_BADARG).  Those of one argument block are on one device, which has to be the current
one when it is called with.  Plain addresses are taken as they are.

A call goes to the ``stream`` it is given (0 is CUDA's legacy default stream); left out, to torch's current stream where the
process uses torch on CUDA, so that it is ordered with the torch operations around it.
"""
from __future__ import annotations

import ctypes
import struct
import sys
from collections import defaultdict

from . import binding as _b
from .binding import _ci, _f64, _i64, _stream, _u64, _vp

__all__ = ["HPSGD_GRAD_NORM_WORKSPACE", "HPSGD_FP8", "hpsgd_adamw_tensor", "make_adamw_table", "hpsgd_adamw_step", "hpsgd_grad_norm",
           "make_rmsnorm_forward", "hpsgd_rmsnorm_forward", "make_rmsnorm_backward", "hpsgd_rmsnorm_backward", "hpsgd_rmsnorm_backward_bytes",
           "make_quantize_fp8", "hpsgd_quantize_fp8", "make_gemm_fp8", "hpsgd_gemm_fp8", "hpsgd_gemm_fp8_bytes",
           "make_gated_scan_forward", "hpsgd_gated_scan_forward", "make_gated_scan_backward", "hpsgd_gated_scan_backward", "hpsgd_gated_scan_saved_bytes",
           "make_distill_loss", "hpsgd_distill_loss", "hpsgd_distill_loss_backward",
           "HPSGD_SILU", "HPSGD_GELU", "make_gated_ffn_forward", "hpsgd_gated_ffn_forward", "make_gated_ffn_backward", "hpsgd_gated_ffn_backward",
           "hpsgd_ops_check",
           "hpsgd_ops_debug_stall"]

HPSGD_GRAD_NORM_WORKSPACE = 65536
HPSGD_FP8 = 2
HPSGD_SILU, HPSGD_GELU = 0, 1


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


class hpsgd_gated_scan_forward_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("sequences", _i64), ("dtype", _ci)] + \
        [(n, _vp) for n in ("f", "v", "o", "offsets", "h0", "h_last", "y", "saved")] + \
        [(n, _i64) for n in ("ldf", "ldv", "ldo", "ldy", "ldh0", "ldlast")]


class hpsgd_gated_scan_backward_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("sequences", _i64), ("dtype", _ci)] + \
        [(n, _vp) for n in ("f", "v", "o", "offsets", "h0", "saved", "dy", "dh_last", "df", "dv", "d_o", "dh0")] + \
        [(n, _i64) for n in ("ldf", "ldv", "ldo", "ldh0", "lddy", "lddlast", "lddf", "lddv", "lddo", "lddh0")]


class hpsgd_distill_loss_args(ctypes.Structure):
    _fields_ = [(n, _i64) for n in ("rows", "vocab", "k")] + [(n, _f64) for n in ("temperature", "label_weight", "teacher_weight", "grad_scale")] + \
        [("dtype", _ci), ("teacher_dtype", _ci)] + \
        [(n, _vp) for n in ("logits", "labels", "teacher_index", "teacher_logits", "loss", "lse", "dlogits", "dloss")] + \
        [(n, _i64) for n in ("ldlogits", "ldteacher", "lddlogits")]


class hpsgd_gated_ffn_forward_args(ctypes.Structure):
    _fields_ = [(n, _i64) for n in ("M", "N", "K")] + [("act", _ci), ("z_dtype", _ci)] + \
        [(n, _vp) for n in ("x", "x_scale", "w", "w_scale", "z8", "z_scale", "z", "gu")] + \
        [(n, _i64) for n in ("ldx", "ldsx", "ldw", "ldsw", "ldz8", "ldsz", "ldz", "ldgu")]


class hpsgd_gated_ffn_backward_args(ctypes.Structure):
    _fields_ = [(n, _i64) for n in ("M", "N")] + [("act", _ci), ("dz_dtype", _ci)] + \
        [(n, _vp) for n in ("gu", "dz", "dq", "dq_scale", "dqt", "dqt_scale", "dgu")] + \
        [(n, _i64) for n in ("ldgu", "lddz", "lddq", "ldsdq", "lddqt", "ldsdqt", "lddgu")]


SIGNATURES = {
    "hpsgd_gated_ffn_forward": (_ci, [_vp, _vp]),
    "hpsgd_gated_ffn_backward": (_ci, [_vp, _vp]),
    "hpsgd_distill_loss": (_ci, [_vp, _vp]),
    "hpsgd_distill_loss_backward": (_ci, [_vp, _vp]),
    "hpsgd_gated_scan_saved_bytes": (ctypes.c_size_t, [_i64, _i64]),
    "hpsgd_gated_scan_forward": (_ci, [_vp, _vp]),
    "hpsgd_gated_scan_backward": (_ci, [_vp, _vp]),
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


def _current_device():
    return sys.modules["torch"]._C._cuda_getDevice()


def _on(stream, device=None):
    """The stream of a call: the one that is given, or torch's current one.  ``device``: where the call's tensors are, which has to be the current one."""
    if device is not None and device != _current_device():
        raise _b.HpsgdError(_b.HPSGD_E_BADARG, "the call's tensors are on device %d, the current one is %d" % (device, _current_device()))
    if stream is not None:
        return _stream(stream)
    torch = sys.modules.get("torch")
    if torch is None or not torch.cuda.is_initialized():
        return None
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # a tenth of the time that a Stream object takes (0.2 against 3.3 us)
    return raw(torch._C._cuda_getDevice()) if raw else torch.cuda.current_stream().cuda_stream


# ---- what a tensor has to be -----------------------------------------------------------
_BYTE = 8                       # beside HPSGD_F32 and HPSGD_BF16: codes and scales
_INT32, _INT64 = 32, 64         # positions
_TYPES = {_b.HPSGD_F32: ("torch.float32", "torch.int32", "torch.uint32"), _b.HPSGD_BF16: ("torch.bfloat16", "torch.int16", "torch.uint16"),
          _BYTE: ("torch.uint8", "torch.int8", "torch.float8_e4m3fn", "torch.float8_e8m0fnu"),
          _INT32: ("torch.int32",), _INT64: ("torch.int64",)}
_SIZE = {_b.HPSGD_F32: 4, _b.HPSGD_BF16: 2, _BYTE: 1, _INT32: 4, _INT64: 8}
_known = defaultdict(set)       # kind -> torch's types that may stand there, of those seen so far


def _refuse(name, why):
    raise _b.HpsgdError(_b.HPSGD_E_BADARG, "%s %s" % (name, why))


def _on_device(name, x):
    """Address of a tensor on a CUDA device (or the plain address, or None)."""
    if x is None or isinstance(x, int):
        return x
    if not getattr(x, "is_cuda", False):
        _refuse(name, "is not a tensor on a CUDA device")
    return x.data_ptr()


def _typed(name, x, kind):
    if x.dtype not in _known[kind]:
        if kind in _TYPES and str(x.dtype) not in _TYPES[kind]:
            _refuse(name, "has elements of type %s" % x.dtype)
        _known[kind].add(x.dtype)


def _vector(name, x, kind, n):
    """Address of n consecutive elements."""
    if x is None:
        return None
    try:
        if x.is_cuda and x.dtype in _known[kind] and x.numel() >= n and x.is_contiguous():
            return x.data_ptr()
    except AttributeError:
        pass
    at = _on_device(name, x)
    if not isinstance(x, int):
        _typed(name, x, kind)
        if x.numel() < n or not x.is_contiguous():
            _refuse(name, "is not %d consecutive elements" % n)
    return at


def _matrix(name, x, kind, rows, cols, ld, last=None):
    """Address of rows that are ld elements apart; `last`: elements of the last row that are touched (cols)."""
    if x is None or x.__class__ is int:
        return x
    need = (rows - 1) * ld + (cols if last is None else last)
    at = _on_device(name, x)
    if isinstance(x, int) or rows <= 0 or cols <= 0:
        return at
    _typed(name, x, kind)
    shape, step = x.shape, x.stride()
    if shape and shape[-1] > 1 and step[-1] != 1:
        _refuse(name, "has rows whose elements are not next to one another")
    if len(shape) > 1 and rows > 1 and shape[-1] >= cols and x.numel() == rows * shape[-1]:
        # a tensor of just these rows: its leading dimensions are one axis, ld elements from row to row
        want = ld
        for k in range(len(shape) - 2, -1, -1):
            if shape[k] > 1 and step[k] != want:
                _refuse(name, "has rows that are %d elements apart, not %d" % (step[k], want))
            want *= shape[k]
    _room(name, x, need * _SIZE.get(kind, 1))
    return at


def _room(name, x, need):
    """At least that many bytes behind a tensor's first element."""
    if x is None or isinstance(x, int) or need <= 0:
        return
    if x.is_contiguous() and x.numel() * x.element_size() >= need:
        return
    have = x.untyped_storage().nbytes() - x.storage_offset() * x.element_size()
    if have < need:
        _refuse(name, "has %d bytes of memory, not %d" % (max(0, have), need))


def _bytes(name, x, need):
    """Address of that many bytes, of whatever type."""
    at = _on_device(name, x)
    _room(name, x, need)
    return at


def _up(n, a):
    return -(-n // a) * a


def _scales(name, x, rows, cols, lds):
    """Address of the scales of a matrix [rows, cols] in the block format."""
    if x is not None and not isinstance(x, int):
        _on_device(name, x)
        _typed(name, x, _BYTE)
        if not x.is_contiguous():
            _refuse(name, "is not contiguous")
    return _bytes(name, x, _up(_up(cols, 128) // 128, 4) * (lds or rows) if rows > 0 and cols > 0 else 0)


def _codes(name, x, rows, cols, ld, last):
    """Address of the codes of a matrix [rows, cols] in the block format; `last`: the last row's bytes that are touched."""
    return _matrix(name, x, _BYTE, rows, cols, ld or _up(cols, 16), last)


# ---- AdamW over many tensors -----------------------------------------------------------
class AdamWTable:
    """The tensors of a step (see make_adamw_table)."""

    def __init__(self, rows, param_dtype, grad_dtype, state_bits):
        self.array = (hpsgd_adamw_tensor * len(rows))()
        self.address = ctypes.addressof(self.array)
        self.count, self.param_dtype, self.grad_dtype, self.state_bits = len(rows), int(param_dtype), int(grad_dtype), int(state_bits)
        self.keep = rows


_FIELDS = frozenset(f[0] for f in hpsgd_adamw_tensor._fields_)
_ITEM = struct.Struct("=7QqQd")
assert _ITEM.size == ctypes.sizeof(hpsgd_adamw_tensor)


def make_adamw_table(rows, param_dtype, grad_dtype, state_bits):
    """A table for hpsgd_adamw_step / hpsgd_grad_norm from dicts with the fields of ``hpsgd_adamw_tensor`` (tensors or addresses;
    what is left out is NULL or 0).  ``rng_offset`` left out: the tensors follow one another in the order given."""
    table = AdamWTable(list(rows), param_dtype, grad_dtype, state_bits)
    moment = _BYTE if table.state_bits == 8 else _b.HPSGD_F32
    pack, array, size, vector, fields, at = _ITEM.pack_into, table.array, _ITEM.size, _vector, _FIELDS, 0
    pd, gd = table.param_dtype, table.grad_dtype
    for k, row in enumerate(table.keep):
        if not fields.issuperset(row):
            raise TypeError("not a field of hpsgd_adamw_tensor: %s" % sorted(set(row) - _FIELDS))
        get, n = row.get, int(row["n"])
        ms, vs, copy, at = get("m_scale"), get("v_scale"), get("copy"), int(get("rng_offset", at))
        pack(array, k * size, vector("param", get("param"), pd, n) or 0, vector("grad", get("grad"), gd, n) or 0, vector("m", get("m"), moment, n) or 0,
             vector("v", get("v"), moment, n) or 0, 0 if ms is None else vector("m_scale", ms, _BYTE, -(-n // 128)),
             0 if vs is None else vector("v_scale", vs, _BYTE, -(-n // 128)), 0 if copy is None else vector("copy", copy, _b.HPSGD_BF16, n), n,
             at & 0xFFFFFFFFFFFFFFFF, float(get("weight_decay", 0.0)))
        at += n
    return table


def hpsgd_adamw_step(table, lr, beta1, beta2, eps, step, seed=0, grad_scale=None, stream=None):
    return _b._check(_b.load().hpsgd_adamw_step(table.address, table.count, table.param_dtype, table.grad_dtype, table.state_bits,
                                                lr, beta1, beta2, eps, step, seed, _on_device("grad_scale", grad_scale), _on(stream)))


def hpsgd_grad_norm(table, max_norm, workspace, out, stream=None):
    if getattr(workspace, "nbytes", HPSGD_GRAD_NORM_WORKSPACE) < HPSGD_GRAD_NORM_WORKSPACE:
        _refuse("workspace", "has %d bytes, not %d" % (workspace.nbytes, HPSGD_GRAD_NORM_WORKSPACE))
    return _b._check(_b.load().hpsgd_grad_norm(table.address, table.count, table.grad_dtype, max_norm, _on_device("workspace", workspace),
                                               _vector("out", out, _b.HPSGD_F32, 2), _on(stream)))


# ---- argument blocks -------------------------------------------------------------------
def _one_device(pointers):
    """The device that all of the tensors are on, or None where there are addresses only."""
    device = None
    for name, x in pointers.items():
        if x is None or x.__class__ is int:
            continue
        here = x.get_device()
        if device is None:
            device = here
        elif here != device:
            _refuse(name, "is on device %d, others on %d" % (here, device))
    return device


class Args:
    """A filled argument struct with its address, and what it points to (`pointers`, as given; `addresses`, as checked)."""

    def __init__(self, struct, pointers, addresses, strides, **plain):
        self.struct, self.keep, self.device = struct(), pointers, _one_device(pointers)
        for name, value in {**addresses, **strides, **plain}.items():
            setattr(self.struct, name, value)
        self.address = ctypes.addressof(self.struct)


def _strides(struct, given):
    """Row strides by their names in the struct, 0 where none is given."""
    names = [n for n, t in struct._fields_ if t is _i64 and n.startswith("ld")]
    unknown = set(given) - set(names)
    if unknown:
        raise TypeError("not a stride of %s: %s" % (struct.__name__, sorted(unknown)))
    return {n: int(given.get(n, 0)) for n in names}


def make_rmsnorm_forward(rows, cols, eps, dtype, x, weight, residual=None, h=None, y=None, y8=None, y_scale=None, rstd=None,
                         weight_dtype=None, **strides):
    weight_dtype = dtype if weight_dtype is None else weight_dtype
    pointers = dict(x=x, residual=residual, weight=weight, h=h, y=y, y8=y8, y_scale=y_scale, rstd=rstd)
    ld = _strides(hpsgd_rmsnorm_forward_args, strides)
    at = {name: _matrix(name, pointers[name], dtype, rows, cols, ld[s] or cols) for name, s in (("x", "ldx"), ("residual", "ldres"), ("h", "ldh"), ("y", "ldy"))}
    at.update(weight=_vector("weight", weight, weight_dtype, cols), y8=_codes("y8", y8, rows, cols, ld["ldy8"], _up(cols, 16)),
              y_scale=_scales("y_scale", y_scale, rows, cols, ld["ldys"]), rstd=_vector("rstd", rstd, _b.HPSGD_F32, rows))
    return Args(hpsgd_rmsnorm_forward_args, pointers, at, ld, rows=rows, cols=cols, eps=eps, dtype=dtype, weight_dtype=weight_dtype)


def hpsgd_rmsnorm_forward(args, stream=None):
    return _b._check(_b.load().hpsgd_rmsnorm_forward(args.address, _on(stream, args.device)))


def hpsgd_rmsnorm_backward_bytes(rows, cols):
    return int(_b.load().hpsgd_rmsnorm_backward_bytes(rows, cols))


def make_rmsnorm_backward(rows, cols, dtype, h, weight, rstd, dy, dx, dweight, workspace, dres=None, weight_dtype=None, **strides):
    weight_dtype = dtype if weight_dtype is None else weight_dtype
    pointers = dict(h=h, weight=weight, rstd=rstd, dy=dy, dres=dres, dx=dx, dweight=dweight, workspace=workspace)
    ld = _strides(hpsgd_rmsnorm_backward_args, strides)
    at = {name: _matrix(name, pointers[name], dtype, rows, cols, ld["ld" + name] or cols) for name in ("h", "dy", "dres", "dx")}
    at.update(weight=_vector("weight", weight, weight_dtype, cols), rstd=_vector("rstd", rstd, _b.HPSGD_F32, rows),
              dweight=_vector("dweight", dweight, _b.HPSGD_F32, cols), workspace=_bytes("workspace", workspace, hpsgd_rmsnorm_backward_bytes(rows, cols)))
    return Args(hpsgd_rmsnorm_backward_args, pointers, at, ld, rows=rows, cols=cols, dtype=dtype, weight_dtype=weight_dtype)


def hpsgd_rmsnorm_backward(args, stream=None):
    return _b._check(_b.load().hpsgd_rmsnorm_backward(args.address, _on(stream, args.device)))


def make_quantize_fp8(rows, cols, dtype, x, q=None, scale=None, qt=None, scale_t=None, x_scale=None, **strides):
    pointers = dict(x=x, x_scale=x_scale, q=q, scale=scale, qt=qt, scale_t=scale_t)
    ld = _strides(hpsgd_quantize_fp8_args, strides)
    at = dict(x=_codes("x", x, rows, cols, ld["ldx"], _up(cols, 8)) if dtype == HPSGD_FP8 else _matrix("x", x, dtype, rows, cols, ld["ldx"] or cols),
              x_scale=_scales("x_scale", x_scale, rows, cols, ld["ldxs"]), q=_codes("q", q, rows, cols, ld["ldq"], _up(cols, 16)),
              scale=_scales("scale", scale, rows, cols, ld["lds"]), qt=_codes("qt", qt, cols, rows, ld["ldqt"], _up(rows, 16)),
              scale_t=_scales("scale_t", scale_t, cols, rows, ld["ldst"]))
    return Args(hpsgd_quantize_fp8_args, pointers, at, ld, rows=rows, cols=cols, dtype=dtype)


def hpsgd_quantize_fp8(args, stream=None):
    return _b._check(_b.load().hpsgd_quantize_fp8(args.address, _on(stream, args.device)))


def hpsgd_gemm_fp8_bytes(M, N, K):
    return int(_b.load().hpsgd_gemm_fp8_bytes(M, N, K))


def make_gemm_fp8(M, N, K, a, a_scale, b, b_scale, d, d_dtype, accumulate=False, workspace=None, workspace_bytes=None, **strides):
    """``workspace_bytes`` left out: the size of the tensor given as workspace."""
    if workspace_bytes is None:
        workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    pointers = dict(a=a, a_scale=a_scale, b=b, b_scale=b_scale, d=d, workspace=workspace)
    ld = _strides(hpsgd_gemm_fp8_args, strides)
    at = dict(a=_codes("a", a, M, K, ld["lda"], K), a_scale=_scales("a_scale", a_scale, M, K, ld["ldsa"]), b=_codes("b", b, N, K, ld["ldb"], K),
              b_scale=_scales("b_scale", b_scale, N, K, ld["ldsb"]), d=_matrix("d", d, d_dtype, M, N, ld["ldd"] or N),
              workspace=_bytes("workspace", workspace, workspace_bytes))
    return Args(hpsgd_gemm_fp8_args, pointers, at, ld, M=M, N=N, K=K, d_dtype=d_dtype, accumulate=int(accumulate), workspace_bytes=workspace_bytes)


def hpsgd_gemm_fp8(args, stream=None):
    return _b._check(_b.load().hpsgd_gemm_fp8(args.address, _on(stream, args.device)))


# ---- a gated linear recurrence ---------------------------------------------------------
def hpsgd_gated_scan_saved_bytes(rows, cols):
    return int(_b.load().hpsgd_gated_scan_saved_bytes(rows, cols))


def make_gated_scan_forward(rows, cols, sequences, dtype, f, v, y, o=None, offsets=None, h0=None, h_last=None, saved=None, **strides):
    pointers = dict(f=f, v=v, o=o, offsets=offsets, h0=h0, h_last=h_last, y=y, saved=saved)
    ld = _strides(hpsgd_gated_scan_forward_args, strides)
    at = {name: _matrix(name, pointers[name], dtype, rows, cols, ld["ld" + name] or cols) for name in ("f", "v", "o", "y")}
    at.update({name: _matrix(name, pointers[name], _b.HPSGD_F32, sequences, cols, ld[s] or cols) for name, s in (("h0", "ldh0"), ("h_last", "ldlast"))})
    at.update(offsets=_vector("offsets", offsets, _INT64, sequences + 1), saved=_bytes("saved", saved, hpsgd_gated_scan_saved_bytes(rows, cols)))
    return Args(hpsgd_gated_scan_forward_args, pointers, at, ld, rows=rows, cols=cols, sequences=sequences, dtype=dtype)


def hpsgd_gated_scan_forward(args, stream=None):
    return _b._check(_b.load().hpsgd_gated_scan_forward(args.address, _on(stream, args.device)))


def make_gated_scan_backward(rows, cols, sequences, dtype, f, v, saved, dy, df, dv, o=None, do=None, offsets=None, h0=None, dh_last=None, dh0=None, **strides):
    pointers = dict(f=f, v=v, o=o, offsets=offsets, h0=h0, saved=saved, dy=dy, dh_last=dh_last, df=df, dv=dv, do=do, dh0=dh0)
    ld = _strides(hpsgd_gated_scan_backward_args, strides)
    at = {name: _matrix(name, pointers[name], dtype, rows, cols, ld["ld" + name] or cols) for name in ("f", "v", "o", "dy", "df", "dv")}
    at["d_o"] = _matrix("do", do, dtype, rows, cols, ld["lddo"] or cols)
    at.update({name: _matrix(name, pointers[name], _b.HPSGD_F32, sequences, cols, ld[s] or cols) for name, s in (("h0", "ldh0"), ("dh_last", "lddlast"), ("dh0", "lddh0"))})
    at.update(offsets=_vector("offsets", offsets, _INT64, sequences + 1), saved=_bytes("saved", saved, hpsgd_gated_scan_saved_bytes(rows, cols)))
    return Args(hpsgd_gated_scan_backward_args, pointers, at, ld, rows=rows, cols=cols, sequences=sequences, dtype=dtype)


def hpsgd_gated_scan_backward(args, stream=None):
    return _b._check(_b.load().hpsgd_gated_scan_backward(args.address, _on(stream, args.device)))


# ---- the loss --------------------------------------------------------------------------
def make_distill_loss(rows, vocab, k, dtype, logits, labels=None, teacher_index=None, teacher_logits=None, temperature=1.0, label_weight=1.0,
                      teacher_weight=0.0, loss=None, lse=None, dlogits=None, dloss=None, grad_scale=1.0, teacher_dtype=None, **strides):
    """``teacher_dtype`` left out: that of the tensor given as teacher_logits (fp32 for an address)."""
    if teacher_dtype is None:
        teacher_dtype = _b.HPSGD_BF16 if str(getattr(teacher_logits, "dtype", "")) == "torch.bfloat16" else _b.HPSGD_F32
    pointers = dict(logits=logits, labels=labels, teacher_index=teacher_index, teacher_logits=teacher_logits, loss=loss, lse=lse, dlogits=dlogits, dloss=dloss)
    ld = _strides(hpsgd_distill_loss_args, strides)
    at = {name: _matrix(name, pointers[name], dtype, rows, vocab, ld["ld" + name] or vocab) for name in ("logits", "dlogits")}
    at.update(labels=_vector("labels", labels, _INT64, rows), loss=_vector("loss", loss, _b.HPSGD_F32, rows), dloss=_vector("dloss", dloss, _b.HPSGD_F32, rows),
              lse=_vector("lse", lse, _b.HPSGD_F32, 2 * rows), teacher_index=_matrix("teacher_index", teacher_index, _INT32, rows, k, ld["ldteacher"] or k),
              teacher_logits=_matrix("teacher_logits", teacher_logits, teacher_dtype, rows, k, ld["ldteacher"] or k))
    return Args(hpsgd_distill_loss_args, pointers, at, ld, rows=rows, vocab=vocab, k=k, dtype=dtype, teacher_dtype=teacher_dtype, temperature=temperature,
                label_weight=label_weight, teacher_weight=teacher_weight, grad_scale=grad_scale)


def hpsgd_distill_loss(args, stream=None):
    return _b._check(_b.load().hpsgd_distill_loss(args.address, _on(stream, args.device)))


def hpsgd_distill_loss_backward(args, stream=None):
    return _b._check(_b.load().hpsgd_distill_loss_backward(args.address, _on(stream, args.device)))


# ---- the gated feed-forward layer ------------------------------------------------------
def make_gated_ffn_forward(M, N, K, act, x, x_scale, w, w_scale, z8=None, z_scale=None, z=None, z_dtype=_b.HPSGD_BF16, gu=None, **strides):
    pointers = dict(x=x, x_scale=x_scale, w=w, w_scale=w_scale, z8=z8, z_scale=z_scale, z=z, gu=gu)
    ld = _strides(hpsgd_gated_ffn_forward_args, strides)
    at = dict(x=_codes("x", x, M, K, ld["ldx"], K), x_scale=_scales("x_scale", x_scale, M, K, ld["ldsx"]), w=_codes("w", w, 2 * N, K, ld["ldw"], K),
              w_scale=_scales("w_scale", w_scale, 2 * N, K, ld["ldsw"]), z8=_codes("z8", z8, M, N, ld["ldz8"], _up(N, 16)),
              z_scale=_scales("z_scale", z_scale, M, N, ld["ldsz"]), z=_matrix("z", z, z_dtype, M, N, ld["ldz"] or N),
              gu=_matrix("gu", gu, _b.HPSGD_BF16, M, 2 * N, ld["ldgu"] or 2 * N))
    return Args(hpsgd_gated_ffn_forward_args, pointers, at, ld, M=M, N=N, K=K, act=act, z_dtype=z_dtype)


def hpsgd_gated_ffn_forward(args, stream=None):
    return _b._check(_b.load().hpsgd_gated_ffn_forward(args.address, _on(stream, args.device)))


def make_gated_ffn_backward(M, N, act, gu, dz, dz_dtype, dq=None, dq_scale=None, dqt=None, dqt_scale=None, dgu=None, **strides):
    pointers = dict(gu=gu, dz=dz, dq=dq, dq_scale=dq_scale, dqt=dqt, dqt_scale=dqt_scale, dgu=dgu)
    ld = _strides(hpsgd_gated_ffn_backward_args, strides)
    at = dict(gu=_matrix("gu", gu, _b.HPSGD_BF16, M, 2 * N, ld["ldgu"] or 2 * N), dz=_matrix("dz", dz, dz_dtype, M, N, ld["lddz"] or N),
              dq=_codes("dq", dq, M, 2 * N, ld["lddq"], _up(2 * N, 16)), dq_scale=_scales("dq_scale", dq_scale, M, 2 * N, ld["ldsdq"]),
              dqt=_codes("dqt", dqt, 2 * N, M, ld["lddqt"], _up(M, 16)), dqt_scale=_scales("dqt_scale", dqt_scale, 2 * N, M, ld["ldsdqt"]),
              dgu=_matrix("dgu", dgu, _b.HPSGD_BF16, M, 2 * N, ld["lddgu"] or 2 * N))
    return Args(hpsgd_gated_ffn_backward_args, pointers, at, ld, M=M, N=N, act=act, dz_dtype=dz_dtype)


def hpsgd_gated_ffn_backward(args, stream=None):
    return _b._check(_b.load().hpsgd_gated_ffn_backward(args.address, _on(stream, args.device)))


def hpsgd_ops_check(stream=None):
    return _b._check(_b.load().hpsgd_ops_check(_on(stream)))


def hpsgd_ops_debug_stall(enable):
    return _b._check(_b.load().hpsgd_ops_debug_stall(int(enable)))
