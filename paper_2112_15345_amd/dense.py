"""Dense operators on gathered rows (include/hg.h, last section): root-mean-square
norm, matrix product with an epilogue, distillation from a teacher's top logits,
forward and backward.

Argument marshalling only, in the native module.  Matrices are 2-D tensors; rows may have any stride, and
a tensor whose columns are not contiguous is copied first.  Outputs and workspaces
are made on `stream` (default: the current stream), where the work runs; as with any
torch call, tensors made on another stream have to be ready, and kept until it is done.

Nothing is recorded for autograd: rms_norm, linear, and distill without its gradient refuse
(ValueError) tensors that require one, unless gradients are off (torch.no_grad(), or the
forward of a torch.autograd.Function).  The backward passes are calls of their own; distill's
gradient can be given to logits.backward(grad).

    y, h, scale = rms_norm(x, weight, residual=r)            # h = x + r
    z, pre = linear(y, w, bias=b, act="gelu", residual=h, keep_pre=True)
    loss, grad = distill(logits, top_ids, top_logits, temperature=2.0, want_grad=True)
    dx, dw, db = linear_grad(dz, y, w, pre=pre, act="gelu")
    dx, dweight = rms_norm_grad(dy, h, weight, dsum=dh)
"""
from __future__ import annotations

import ctypes

import torch

from . import HG_DT_BF16, HG_DT_F16, HG_DT_F32, HG_DT_NONE, _check, load_library  # noqa: F401

HG_DT_E4M3 = 4
HG_MAX_TOP = 1024
HG_ACT_NONE, HG_ACT_RELU, HG_ACT_GELU, HG_ACT_SILU = 0, 1, 2, 3
_ACTS = {None: HG_ACT_NONE, "none": HG_ACT_NONE, "relu": HG_ACT_RELU, "gelu": HG_ACT_GELU,
         "silu": HG_ACT_SILU}
_P, _I64, _I32, _F = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float


# The entry points' argument structures, for programs that call the library through ctypes.
class NormArgs(ctypes.Structure):
    _fields_ = [("rows", _I64), ("dim", _I64), ("dtype", _I32), ("out_dtype", _I32),
                ("weight_dtype", _I32), ("eps", _F), ("x", _P), ("x_stride", _I64),
                ("x_rows", _I64), ("ids", _P), ("residual", _P), ("residual_stride", _I64),
                ("weight", _P), ("y", _P), ("y_stride", _I64), ("scale", _P), ("sum", _P),
                ("sum_stride", _I64)]


class NormGradArgs(ctypes.Structure):
    _fields_ = [("rows", _I64), ("dim", _I64), ("dtype", _I32), ("weight_dtype", _I32),
                ("eps", _F), ("x", _P), ("x_stride", _I64), ("x_rows", _I64), ("ids", _P),
                ("weight", _P), ("dy", _P), ("dy_stride", _I64), ("dsum", _P),
                ("dsum_stride", _I64), ("dx", _P), ("dx_stride", _I64), ("dweight", _P),
                ("workspace", _P), ("workspace_bytes", _I64)]


class LinearArgs(ctypes.Structure):
    _fields_ = [("m", _I64), ("k", _I64), ("n", _I64), ("dtype", _I32), ("out_dtype", _I32),
                ("bias_dtype", _I32), ("act", _I32), ("x", _P), ("x_stride", _I64),
                ("x_scale", _P), ("w", _P), ("w_stride", _I64), ("w_scale", _P), ("bias", _P),
                ("residual", _P), ("residual_stride", _I64), ("y", _P), ("y_stride", _I64),
                ("pre", _P), ("pre_stride", _I64), ("workspace", _P), ("workspace_bytes", _I64)]


class LinearGradArgs(ctypes.Structure):
    _fields_ = [("m", _I64), ("k", _I64), ("n", _I64), ("dtype", _I32), ("dw_dtype", _I32),
                ("act", _I32), ("dy", _P), ("dy_stride", _I64), ("pre", _P),
                ("pre_stride", _I64), ("x", _P), ("x_stride", _I64), ("w", _P),
                ("w_stride", _I64), ("dx", _P), ("dx_stride", _I64), ("dw", _P),
                ("dw_stride", _I64), ("dbias", _P), ("workspace", _P), ("workspace_bytes", _I64)]


class DistillArgs(ctypes.Structure):
    _fields_ = [("rows", _I64), ("classes", _I64), ("top", _I32), ("dtype", _I32),
                ("teacher_dtype", _I32), ("temperature", _F), ("logits", _P),
                ("logits_stride", _I64), ("ids", _P), ("ids_stride", _I64), ("teacher", _P),
                ("teacher_stride", _I64), ("row_weight", _P), ("loss", _P), ("grad", _P),
                ("grad_stride", _I64)]


_native = None


def _module():
    """The native module _hgdense (csrc/hg_dense_py.cpp), which checks the tensors, makes the
    outputs and calls the library."""
    global _native
    if _native is None:
        load_library()
        from . import _dense
        _native = _dense
    return _native


def _call(name, stream, *args):
    f = getattr(_native or _module(), name)
    if stream is None:
        r = f(*args)
    else:
        for a in args:
            if isinstance(a, torch.Tensor) and a.device != stream.device:
                raise ValueError(f"a tensor on {a.device} and a stream of {stream.device}")
        with torch.cuda.stream(stream):
            r = f(*args)
    if type(r) is int:
        _check(r)
    return r


def _act(act) -> int:
    if act not in _ACTS:
        raise ValueError(f"act: {act!r} is none of None, relu, gelu, silu")
    return _ACTS[act]


def rms_norm(x, weight=None, residual=None, ids=None, eps: float = 1e-6, out_dtype=None,
             stream=None):
    """(y, sum, scale): y = h weight / sqrt(mean(h^2) + eps) per row, h = x + residual
    (hg_rms_norm).  ids: int64 [rows], row i is x[ids[i]] (out of range: a row of NaN).
    out_dtype: x's dtype, or torch.float8_e4m3fn, with scale [rows] (else None).  sum: h,
    when there is a residual (else None)."""
    return _call("rms_norm", stream, x, weight, residual, ids, eps, out_dtype)


def rms_norm_grad(dy, x, weight=None, dsum=None, ids=None, eps: float = 1e-6,
                  want_dx: bool = True, want_dweight: bool | None = None, stream=None):
    """(dx, dweight) of rms_norm (hg_rms_norm_grad).  x: the rows that were normalised,
    the forward call's sum (or its x, with the same ids, when it had no residual); dsum:
    the gradient of sum.  dx is the gradient of x and of residual; dweight is float32 (by
    default wanted when there is a weight).  What is not wanted is None."""
    return _call("rms_norm_grad", stream, dy, x, weight, dsum, ids, eps, want_dx, want_dweight)


def linear(x, w, bias=None, act=None, residual=None, x_scale=None, w_scale=None, out_dtype=None,
           keep_pre: bool = False, stream=None):
    """(y, pre): y = act(x w^T + bias) + residual (hg_linear); pre: the values before the
    activation, with keep_pre (else None).  x [m, k], w [n, k]; act None, "relu", "gelu" (tanh
    form) or "silu".  With torch.float8_e4m3fn x and w, x_scale [m] and w_scale [n] (float32)
    are needed, and out_dtype (default bfloat16) is the type of y, pre and residual."""
    return _call("linear", stream, x, w, bias, _act(act), residual, x_scale, w_scale, out_dtype,
                 keep_pre)


def linear_grad(dy, x, w, pre=None, act=None, want_dx: bool = True, want_dw: bool = True,
                want_dbias: bool = True, dw_dtype=None, stream=None):
    """(dx, dw, dbias) of linear (hg_linear_grad).  pre: the forward call's, needed with an
    activation.  dw is in dw_dtype (default w's, or float32), dbias in float32.  The gradient
    of residual is dy.  What is not wanted is None."""
    return _call("linear_grad", stream, dy, x, w, pre, _act(act), want_dx, want_dw, want_dbias,
                 dw_dtype)


def distill(logits, ids, teacher, temperature: float = 1.0, row_weight=None,
            want_loss: bool = True, want_grad: bool = False, stream=None):
    """(loss, grad): per row the divergence of softmax(logits / temperature) from the softmax of
    the teacher's top logits (hg_distill).  ids (int64) and teacher [rows, top]: the listed
    classes and the teacher's logits, -1 where a list ends early.  loss is float32 [rows]; grad,
    of sum(row_weight loss) by the logits, has their dtype.  What is not wanted is None."""
    return _call("distill", stream, logits, ids, teacher, temperature, row_weight, want_loss,
                 want_grad)
