"""Dense operators on gathered rows (include/hg.h, last section): root-mean-square norm, layer norm,
matrix product with an epilogue (also of 8-bit rows), embedding, distillation from a teacher's top
logits, forward and backward, and rows kept in 8-bit integers.

Argument marshalling only, in the native module.  Matrices are 2-D tensors; rows may have any stride, and
a tensor whose columns are not contiguous is copied first.  Outputs and workspaces
are made on `stream` (default: the current stream), where the work runs; as with any
torch call, tensors made on another stream have to be ready, and kept until it is done.

Nothing is recorded for autograd: embed, the norms, linear, quantize, dequantize, and distill without
its gradient refuse (ValueError) tensors that require one, unless gradients are off (torch.no_grad(),
or the forward of a torch.autograd.Function); so does embed_grad of a table that it adds to.  The
backward passes are calls of their own; distill's gradient can be given to logits.backward(grad).

    x = embed(table, ids, out_dtype=torch.bfloat16)
    y, h, scale = rms_norm(x, weight, residual=r)            # h = x + r; layer_norm the same way
    z, pre = linear(y, w, bias=b, act="gelu", residual=h, keep_pre=True)
    loss, grad = distill(logits, top_ids, top_logits, temperature=2.0, want_grad=True)
    dx, dw, db = linear_grad(dz, y, w, pre=pre, act="gelu")
    dx, dweight = rms_norm_grad(dy, h, weight, dsum=dh)
    embed_grad(dx, ids, nodes, scale=-rate, into=table)

In 8-bit integers, and with activations that are kept in 8 bits:

    q, h, c = layer_norm(x, weight, bias, residual=r, out_dtype=torch.int8)
    z, pre = linear(q, wq, bias=b, x_scale=c, w_scale=wc)
    y8, yc = quantize(y, group=128)
    pre8, prec = quantize(pre, group=128)
    dx, dw, db = linear_grad(dz, y8, w, pre=pre8, act="gelu", x_scale=yc, pre_scale=prec, group=128)
"""
from __future__ import annotations

import ctypes

import torch

from . import HG_DT_BF16, HG_DT_F16, HG_DT_F32, HG_DT_NONE, _check, load_library  # noqa: F401

HG_DT_E4M3, HG_DT_I8 = 4, 6
HG_MAX_TOP = 1024
HG_KEPT_GROUP = 128
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


class LayerNormArgs(ctypes.Structure):
    _fields_ = [("rows", _I64), ("dim", _I64), ("dtype", _I32), ("out_dtype", _I32),
                ("weight_dtype", _I32), ("bias_dtype", _I32), ("eps", _F), ("x", _P),
                ("x_stride", _I64), ("x_rows", _I64), ("ids", _P), ("residual", _P),
                ("residual_stride", _I64), ("weight", _P), ("bias", _P), ("y", _P),
                ("y_stride", _I64), ("scale", _P), ("sum", _P), ("sum_stride", _I64)]


class LayerNormGradArgs(ctypes.Structure):
    _fields_ = [("rows", _I64), ("dim", _I64), ("dtype", _I32), ("weight_dtype", _I32),
                ("eps", _F), ("x", _P), ("x_stride", _I64), ("x_rows", _I64), ("ids", _P),
                ("weight", _P), ("dy", _P), ("dy_stride", _I64), ("dsum", _P),
                ("dsum_stride", _I64), ("dx", _P), ("dx_stride", _I64), ("dweight", _P),
                ("dbias", _P), ("workspace", _P), ("workspace_bytes", _I64)]


class EmbedArgs(ctypes.Structure):
    _fields_ = [("n", _I64), ("nodes", _I64), ("dim", _I64), ("table_dtype", _I32),
                ("out_dtype", _I32), ("scale", _F), ("table", _P), ("table_stride", _I64),
                ("ids", _P), ("y", _P), ("y_stride", _I64)]


class EmbedGradArgs(ctypes.Structure):
    _fields_ = [("n", _I64), ("nodes", _I64), ("dim", _I64), ("dtype", _I32), ("out_dtype", _I32),
                ("add", _I32), ("scale", _F), ("dy", _P), ("dy_stride", _I64), ("ids", _P),
                ("dtable", _P), ("dtable_stride", _I64), ("workspace", _P),
                ("workspace_bytes", _I64)]


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


class QuantizeArgs(ctypes.Structure):
    _fields_ = [("rows", _I64), ("dim", _I64), ("dtype", _I32), ("group", _I32), ("x", _P),
                ("x_stride", _I64), ("q", _P), ("q_stride", _I64), ("scale", _P)]


class DequantizeArgs(ctypes.Structure):
    _fields_ = [("rows", _I64), ("dim", _I64), ("dtype", _I32), ("group", _I32), ("q", _P),
                ("q_stride", _I64), ("scale", _P), ("x", _P), ("x_stride", _I64)]


class LinearGradKeptArgs(ctypes.Structure):
    _fields_ = [("grad", LinearGradArgs), ("group", _I32), ("x_scale", _P), ("pre_scale", _P)]


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


def layer_norm(x, weight=None, bias=None, residual=None, ids=None, eps: float = 1e-5,
               out_dtype=None, stream=None):
    """(y, sum, scale): y = (h - mean(h)) weight / sqrt(var(h) + eps) + bias per row, h = x +
    residual (hg_layer_norm).  ids: int64 [rows], row i is x[ids[i]] (out of range: a row of NaN).
    out_dtype: x's dtype, or torch.float8_e4m3fn or torch.int8, with scale [rows] (else None).
    sum: h, when there is a residual (else None)."""
    return _call("layer_norm", stream, x, weight, bias, residual, ids, eps, out_dtype)


def layer_norm_grad(dy, x, weight=None, dsum=None, ids=None, eps: float = 1e-5,
                    want_dx: bool = True, want_dweight: bool | None = None,
                    want_dbias: bool = True, stream=None):
    """(dx, dweight, dbias) of layer_norm (hg_layer_norm_grad).  x: the rows that were normalised,
    the forward call's sum (or its x, with the same ids, when it had no residual); dsum: the
    gradient of sum.  dx is the gradient of x and of residual; dweight (by default wanted when
    there is a weight) and dbias are float32.  What is not wanted is None."""
    return _call("layer_norm_grad", stream, dy, x, weight, dsum, ids, eps, want_dx, want_dweight,
                 want_dbias)


def embed(table, ids, scale: float = 1.0, out_dtype=None, stream=None):
    """scale table[ids] (hg_embed), in out_dtype (default: the table's).  ids: int64 [n]; -1
    (padding) is a row of zeros, any other out of range a row of NaN."""
    return _call("embed", stream, table, ids, scale, out_dtype)[0]


def embed_grad(dy, ids, nodes: int, scale: float = 1.0, out_dtype=None, into=None, stream=None):
    """The gradient of embed's table [nodes, dim] (hg_embed_grad), summed in a fixed order:
    scale times the sum of dy's rows over the positions of each id, in out_dtype (float32 by
    default, or dy's).  Ids out of range count for nothing.  into: a float32 table that it is
    added to in place, and that is returned; rows that no id names are not touched (with scale
    = -rate a step of descent).  dy shares no memory with it."""
    return _call("embed_grad", stream, dy, ids, nodes, scale, out_dtype, into)[0]


def linear(x, w, bias=None, act=None, residual=None, x_scale=None, w_scale=None, out_dtype=None,
           keep_pre: bool = False, stream=None):
    """(y, pre): y = act(x w^T + bias) + residual (hg_linear); pre: the values before the
    activation, with keep_pre (else None).  x [m, k], w [n, k]; act None, "relu", "gelu" (tanh
    form) or "silu".  With torch.float8_e4m3fn or torch.int8 x and w, x_scale [m] and w_scale [n]
    (float32) are needed, and out_dtype (default bfloat16) is the type of y, pre and residual."""
    return _call("linear", stream, x, w, bias, _act(act), residual, x_scale, w_scale, out_dtype,
                 keep_pre)


def linear_grad(dy, x, w, pre=None, act=None, want_dx: bool = True, want_dw: bool = True,
                want_dbias: bool = True, dw_dtype=None, stream=None, x_scale=None, pre_scale=None,
                group: int = 0):
    """(dx, dw, dbias) of linear (hg_linear_grad).  pre: the forward call's, needed with an
    activation.  dw is in dw_dtype (default w's, or float32), dbias in float32.  The gradient
    of residual is dy.  What is not wanted is None.
    x or pre may be what quantize kept of it, with its x_scale or pre_scale, and the group of
    both (hg_linear_grad_kept); x and w need not have the same type then."""
    return _call("linear_grad", stream, dy, x, w, pre, _act(act), want_dx, want_dw, want_dbias,
                 dw_dtype, x_scale, pre_scale, group)


def quantize(x, group: int = 0, stream=None):
    """(q, scale): x's rows in torch.int8, and what to multiply them with (hg_quantize): scale is
    [rows], for linear's x_scale or w_scale, or with group 128 (a scale for every 128 columns, for
    activations that are kept) [rows, ceil(dim / 128)].  A row (or group) that is not finite is
    zeros with a scale of NaN."""
    return _call("quantize", stream, x, group)


def dequantize(q, scale, group: int = 0, out_dtype=torch.bfloat16, stream=None):
    """q times scale, as quantize made them, rounded once to out_dtype (hg_dequantize)."""
    return _call("dequantize", stream, q, scale, group, out_dtype)[0]


def distill(logits, ids, teacher, temperature: float = 1.0, row_weight=None,
            want_loss: bool = True, want_grad: bool = False, stream=None):
    """(loss, grad): per row the divergence of softmax(logits / temperature) from the softmax of
    the teacher's top logits (hg_distill).  ids (int64) and teacher [rows, top]: the listed
    classes and the teacher's logits, -1 where a list ends early.  loss is float32 [rows]; grad,
    of sum(row_weight loss) by the logits, has their dtype.  What is not wanted is None."""
    return _call("distill", stream, logits, ids, teacher, temperature, row_weight, want_loss,
                 want_grad)
