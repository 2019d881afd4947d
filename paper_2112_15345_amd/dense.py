"""Dense operators on gathered rows (include/hg.h, last section): root-mean-square
norm, matrix product with an epilogue, distillation from a teacher's top logits,
forward and backward.

Argument marshalling only.  Matrices are 2-D tensors; rows may have any stride, and
a tensor whose columns are not contiguous is copied first.  Outputs and workspaces
are made on `stream` (default: the current stream), where the work runs.

    y, h, scale = rms_norm(x, weight, residual=r)            # h = x + r
    z, pre = linear(y, w, bias=b, act="gelu", residual=h, keep_pre=True)
    loss, grad = distill(logits, top_ids, top_logits, temperature=2.0, want_grad=True)
    dx, dw, db = linear_grad(dz, y, w, pre=pre, act="gelu")
    dx, dweight = rms_norm_grad(dy, h, weight, dsum=dh)
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from . import HG_DT_BF16, HG_DT_F16, HG_DT_F32, HG_DT_NONE, _check, load_library

HG_DT_E4M3 = 4
HG_MAX_TOP = 1024
HG_ACT_NONE, HG_ACT_RELU, HG_ACT_GELU, HG_ACT_SILU = 0, 1, 2, 3
_ACTS = {None: HG_ACT_NONE, "none": HG_ACT_NONE, "relu": HG_ACT_RELU, "gelu": HG_ACT_GELU,
         "silu": HG_ACT_SILU}
_CODE = {torch.float32: HG_DT_F32, torch.float16: HG_DT_F16, torch.bfloat16: HG_DT_BF16,
         torch.float8_e4m3fn: HG_DT_E4M3}

_P, _I64, _I32, _F = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float


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


def _matrix(name, t, device=None, rows=None, cols=None, dtypes=None) -> torch.Tensor:
    """A 2-D tensor with contiguous columns, checked."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name}: a 2-D tensor is wanted")
    if t.device.type != "cuda" or (device is not None and t.device != device):
        raise ValueError(f"{name}: on {t.device}, not on {device or 'a GPU'}")
    if dtypes is not None and t.dtype not in dtypes:
        raise ValueError(f"{name}: unsupported dtype {t.dtype}")
    if (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, not {(rows, cols)}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        t = t.contiguous()
    return t


def _vector(name, t, device, n, dtypes) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or t.dim() != 1 or t.shape[0] != n:
        raise ValueError(f"{name}: a 1-D tensor of {n} is wanted")
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, not on {device}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: unsupported dtype {t.dtype}")
    return t.contiguous()


def _ptr(t):
    return t.data_ptr() if t is not None and t.numel() else None


def _stride(t):
    """Elements between rows (a matrix of one row may report any)."""
    return 0 if t is None else (t.stride(0) if t.shape[0] > 1 else t.shape[1])


@contextlib.contextmanager
def _on(device, stream):
    """The device, and the stream that outputs are made on and the work runs on."""
    with torch.cuda.device(device):
        if stream is None:
            yield int(torch.cuda.current_stream().cuda_stream)
        else:
            with torch.cuda.stream(stream):
                yield int(stream.cuda_stream)


def _workspace(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


_FLOATS = (torch.float32, torch.float16, torch.bfloat16)


def _taken(x, ids):
    """x, ids and the number of rows they stand for."""
    x = _matrix("x", x, dtypes=_FLOATS)
    if ids is None:
        return x, None, x.shape[0]
    if not isinstance(ids, torch.Tensor) or ids.dim() != 1:
        raise ValueError("ids: a 1-D tensor is wanted")
    ids = _vector("ids", ids, x.device, ids.shape[0], (torch.int64,))
    return x, ids, ids.shape[0]


def rms_norm(x, weight=None, residual=None, ids=None, eps: float = 1e-6, out_dtype=None,
             stream=None):
    """(y, sum, scale): y = h weight / sqrt(mean(h^2) + eps) per row, h = x + residual
    (hg_rms_norm).  ids: int64 [rows], row i is x[ids[i]] (out of range: a row of NaN).
    out_dtype: x's dtype, or torch.float8_e4m3fn, with scale [rows] (else None).  sum: h,
    when there is a residual (else None)."""
    x, ids, rows = _taken(x, ids)
    dim, dev = x.shape[1], x.device
    if residual is not None:
        residual = _matrix("residual", residual, dev, rows, dim, (x.dtype,))
    if weight is not None:
        weight = _vector("weight", weight, dev, dim, (torch.float32, x.dtype))
    out_dtype = out_dtype or x.dtype
    if out_dtype not in (x.dtype, torch.float8_e4m3fn):
        raise ValueError(f"out_dtype: {out_dtype} is neither x's nor torch.float8_e4m3fn")
    with _on(dev, stream) as s:
        y = torch.empty((rows, dim), dtype=out_dtype, device=dev)
        total = torch.empty((rows, dim), dtype=x.dtype, device=dev) if residual is not None else None
        scale = (torch.empty(rows, dtype=torch.float32, device=dev)
                 if out_dtype != x.dtype else None)
        a = NormArgs(rows, dim, _CODE[x.dtype], _CODE[out_dtype],
                     HG_DT_NONE if weight is None else _CODE[weight.dtype], eps, _ptr(x),
                     _stride(x), x.shape[0], _ptr(ids), _ptr(residual), _stride(residual),
                     _ptr(weight), _ptr(y), dim, _ptr(scale), _ptr(total), dim)
        _check(load_library().hg_rms_norm(ctypes.byref(a), s))
    return y, total, scale


def rms_norm_grad(dy, x, weight=None, dsum=None, ids=None, eps: float = 1e-6,
                  want_dx: bool = True, want_dweight: bool | None = None, stream=None):
    """(dx, dweight) of rms_norm (hg_rms_norm_grad).  x: the rows that were normalised,
    the forward call's sum (or its x, with the same ids, when it had no residual); dsum:
    the gradient of sum.  dx is the gradient of x and of residual; dweight is float32 (by
    default wanted when there is a weight).  What is not wanted is None."""
    x, ids, rows = _taken(x, ids)
    dim, dev = x.shape[1], x.device
    dy = _matrix("dy", dy, dev, rows, dim, (x.dtype,))
    if dsum is not None:
        dsum = _matrix("dsum", dsum, dev, rows, dim, (x.dtype,))
    if weight is not None:
        weight = _vector("weight", weight, dev, dim, (torch.float32, x.dtype))
    if want_dweight is None:
        want_dweight = weight is not None
    lib = load_library()
    with _on(dev, stream) as s:
        dx = torch.empty((rows, dim), dtype=x.dtype, device=dev) if want_dx else None
        dw = torch.empty(dim, dtype=torch.float32, device=dev) if want_dweight else None
        ws = _workspace(lib.hg_rms_norm_grad_workspace(rows, dim) if want_dweight else 0, dev)
        a = NormGradArgs(rows, dim, _CODE[x.dtype],
                         HG_DT_NONE if weight is None else _CODE[weight.dtype], eps, _ptr(x),
                         _stride(x), x.shape[0], _ptr(ids), _ptr(weight), _ptr(dy), _stride(dy),
                         _ptr(dsum), _stride(dsum), _ptr(dx), dim, _ptr(dw), _ptr(ws),
                         ws.numel() if ws is not None else 0)
        _check(lib.hg_rms_norm_grad(ctypes.byref(a), s))
    return dx, dw


def linear(x, w, bias=None, act=None, residual=None, x_scale=None, w_scale=None, out_dtype=None,
           keep_pre: bool = False, stream=None):
    """(y, pre): y = act(x w^T + bias) + residual (hg_linear); pre: the values before the
    activation, with keep_pre (else None).  x [m, k], w [n, k]; act None, "relu", "gelu" (tanh
    form) or "silu".  With torch.float8_e4m3fn x and w, x_scale [m] and w_scale [n] (float32)
    are needed, and out_dtype (default bfloat16) is the type of y, pre and residual."""
    x = _matrix("x", x, dtypes=(*_FLOATS, torch.float8_e4m3fn))
    dev = x.device
    m, k = x.shape
    w = _matrix("w", w, dev, None, k, (x.dtype,))
    n = w.shape[0]
    if act not in _ACTS:
        raise ValueError(f"act: {act!r} is none of None, relu, gelu, silu")
    if x.dtype == torch.float8_e4m3fn:
        out_dtype = out_dtype or torch.bfloat16
        if x_scale is None or w_scale is None:
            raise ValueError("8-bit operands need x_scale and w_scale")
        x_scale = _vector("x_scale", x_scale, dev, m, (torch.float32,))
        w_scale = _vector("w_scale", w_scale, dev, n, (torch.float32,))
        if out_dtype not in _FLOATS:
            raise ValueError(f"out_dtype: unsupported {out_dtype}")
    else:
        if x_scale is not None or w_scale is not None:
            raise ValueError("scales are for 8-bit operands")
        if out_dtype not in (None, x.dtype):
            raise ValueError(f"out_dtype: {out_dtype} is not x's {x.dtype}")
        out_dtype = x.dtype
    if bias is not None:
        bias = _vector("bias", bias, dev, n, _FLOATS)
    if residual is not None:
        residual = _matrix("residual", residual, dev, m, n, (out_dtype,))
    lib = load_library()
    with _on(dev, stream) as s:
        y = torch.empty((m, n), dtype=out_dtype, device=dev)
        pre = torch.empty((m, n), dtype=out_dtype, device=dev) if keep_pre else None
        ws = _workspace(lib.hg_linear_workspace(m, k, n, _CODE[x.dtype]), dev)
        a = LinearArgs(m, k, n, _CODE[x.dtype], _CODE[out_dtype],
                       HG_DT_NONE if bias is None else _CODE[bias.dtype], _ACTS[act], _ptr(x),
                       _stride(x), _ptr(x_scale), _ptr(w), _stride(w), _ptr(w_scale), _ptr(bias),
                       _ptr(residual), _stride(residual), _ptr(y), n, _ptr(pre), n, _ptr(ws),
                       ws.numel() if ws is not None else 0)
        _check(lib.hg_linear(ctypes.byref(a), s))
    return y, pre


def linear_grad(dy, x, w, pre=None, act=None, want_dx: bool = True, want_dw: bool = True,
                want_dbias: bool = True, dw_dtype=None, stream=None):
    """(dx, dw, dbias) of linear (hg_linear_grad).  pre: the forward call's, needed with an
    activation.  dw is in dw_dtype (default w's, or float32), dbias in float32.  The gradient
    of residual is dy.  What is not wanted is None."""
    x = _matrix("x", x, dtypes=_FLOATS)
    dev = x.device
    m, k = x.shape
    w = _matrix("w", w, dev, None, k, (x.dtype,))
    n = w.shape[0]
    dy = _matrix("dy", dy, dev, m, n, (x.dtype,))
    if act not in _ACTS:
        raise ValueError(f"act: {act!r} is none of None, relu, gelu, silu")
    if _ACTS[act] == HG_ACT_NONE:
        pre = None
    elif pre is None:
        raise ValueError("an activation needs pre")
    else:
        pre = _matrix("pre", pre, dev, m, n, (x.dtype,))
    dw_dtype = dw_dtype or w.dtype
    if dw_dtype not in (w.dtype, torch.float32):
        raise ValueError(f"dw_dtype: {dw_dtype} is neither w's nor float32")
    lib = load_library()
    with _on(dev, stream) as s:
        dx = torch.empty((m, k), dtype=x.dtype, device=dev) if want_dx else None
        dw = torch.empty((n, k), dtype=dw_dtype, device=dev) if want_dw else None
        db = torch.empty(n, dtype=torch.float32, device=dev) if want_dbias else None
        ws = _workspace(lib.hg_linear_grad_workspace(m, k, n, _CODE[x.dtype], _ACTS[act]), dev)
        a = LinearGradArgs(m, k, n, _CODE[x.dtype], _CODE[dw_dtype], _ACTS[act], _ptr(dy),
                           _stride(dy), _ptr(pre), _stride(pre), _ptr(x), _stride(x), _ptr(w),
                           _stride(w), _ptr(dx), k, _ptr(dw), k, _ptr(db), _ptr(ws),
                           ws.numel() if ws is not None else 0)
        _check(lib.hg_linear_grad(ctypes.byref(a), s))
    return dx, dw, db


def distill(logits, ids, teacher, temperature: float = 1.0, row_weight=None,
            want_loss: bool = True, want_grad: bool = False, stream=None):
    """(loss, grad): per row the divergence of softmax(logits / temperature) from the softmax of
    the teacher's top logits (hg_distill).  ids (int64) and teacher [rows, top]: the listed
    classes and the teacher's logits, -1 where a list ends early.  loss is float32 [rows]; grad,
    of sum(row_weight loss) by the logits, has their dtype.  What is not wanted is None."""
    logits = _matrix("logits", logits, dtypes=_FLOATS)
    dev = logits.device
    rows, classes = logits.shape
    ids = _matrix("ids", ids, dev, rows, None, (torch.int64,))
    top = ids.shape[1]
    teacher = _matrix("teacher", teacher, dev, rows, top, _FLOATS)
    if row_weight is not None:
        row_weight = _vector("row_weight", row_weight, dev, rows, (torch.float32,))
    with _on(dev, stream) as s:
        loss = torch.empty(rows, dtype=torch.float32, device=dev) if want_loss else None
        grad = torch.empty_like(logits, memory_format=torch.contiguous_format) if want_grad else None
        a = DistillArgs(rows, classes, top, _CODE[logits.dtype], _CODE[teacher.dtype],
                        temperature, _ptr(logits), _stride(logits), _ptr(ids), _stride(ids),
                        _ptr(teacher), _stride(teacher), _ptr(row_weight), _ptr(loss), _ptr(grad),
                        classes)
        _check(load_library().hg_distill(ctypes.byref(a), s))
    return loss, grad
