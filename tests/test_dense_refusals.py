"""The dense operators' C entry points refuse bad arguments on the host, before any device work
(no GPU needed; the pointers are never read)."""
import ctypes

import pytest

import paper_2112_15345_amd as hg
from paper_2112_15345_amd import dense

P = 0x1000  # never dereferenced
LIB = hg.load_library()


def norm(**kw):
    v = dict(rows=2, dim=8, dtype=1, out_dtype=1, weight_dtype=0, eps=1e-6, x=P, x_stride=8, x_rows=2,
             y=P, y_stride=8)
    return LIB.hg_rms_norm(ctypes.byref(dense.NormArgs(**{**v, **kw})), None)


def norm_grad(**kw):
    v = dict(rows=2, dim=8, dtype=1, weight_dtype=0, eps=1e-6, x=P, x_stride=8, x_rows=2, dy=P,
             dy_stride=8, dx=P, dx_stride=8)
    return LIB.hg_rms_norm_grad(ctypes.byref(dense.NormGradArgs(**{**v, **kw})), None)


def linear(**kw):
    v = dict(m=2, k=8, n=4, dtype=3, out_dtype=3, bias_dtype=1, act=0, x=P, x_stride=8, w=P,
             w_stride=8, y=P, y_stride=4, workspace=P, workspace_bytes=1 << 40)
    return LIB.hg_linear(ctypes.byref(dense.LinearArgs(**{**v, **kw})), None)


def linear_grad(**kw):
    v = dict(m=2, k=8, n=4, dtype=3, dw_dtype=3, act=0, dy=P, dy_stride=4, x=P, x_stride=8, w=P,
             w_stride=8, dx=P, dx_stride=8, dw=P, dw_stride=8, dbias=P, workspace=P,
             workspace_bytes=1 << 40)
    return LIB.hg_linear_grad(ctypes.byref(dense.LinearGradArgs(**{**v, **kw})), None)


def distill(**kw):
    v = dict(rows=2, classes=8, top=2, dtype=1, teacher_dtype=1, temperature=1.0, logits=P,
             logits_stride=8, ids=P, ids_stride=2, teacher=P, teacher_stride=2, loss=P, grad=P,
             grad_stride=8)
    return LIB.hg_distill(ctypes.byref(dense.DistillArgs(**{**v, **kw})), None)


BIG = 1 << 31
CASES = [
    (norm, hg.HG_EINVAL, [dict(rows=-1), dict(dim=0), dict(dtype=0), dict(dtype=4), dict(out_dtype=2),
                          dict(weight_dtype=2), dict(weight_dtype=1), dict(eps=-1.0),
                          dict(eps=float("nan")), dict(x=None), dict(x_stride=-1), dict(y=None),
                          dict(y_stride=7), dict(sum=P, sum_stride=7), dict(out_dtype=4),
                          dict(ids=P, x_rows=-1), dict(residual=P, residual_stride=-8)]),
    (norm, hg.HG_EUNSUPPORTED, [dict(rows=BIG), dict(dim=BIG)]),
    (norm_grad, hg.HG_EINVAL, [dict(rows=-1), dict(dim=0), dict(dtype=4), dict(weight_dtype=3),
                               dict(weight_dtype=1), dict(dy=None), dict(x=None), dict(dx_stride=7),
                               dict(dsum=P, dsum_stride=-1), dict(eps=float("inf")),
                               dict(dweight=P), dict(dweight=P, workspace=P, workspace_bytes=63)]),
    (norm_grad, hg.HG_EUNSUPPORTED, [dict(rows=BIG), dict(dim=BIG)]),
    (linear, hg.HG_EINVAL, [dict(m=-1), dict(k=-1), dict(n=-1), dict(dtype=0), dict(dtype=5),
                            dict(out_dtype=1), dict(dtype=4), dict(dtype=4, out_dtype=4, x_scale=P,
                                                                   w_scale=P),
                            dict(bias=P, bias_dtype=0), dict(bias=P, bias_dtype=4), dict(act=4),
                            dict(act=-1), dict(x=None), dict(w=None), dict(x_stride=-1),
                            dict(y=None), dict(y_stride=3), dict(pre=P, pre_stride=3),
                            dict(residual=P, residual_stride=-1),
                            dict(m=1, k=1 << 20, n=4, x_stride=1 << 20, w_stride=1 << 20,
                                 workspace=None, workspace_bytes=0)]),
    (linear, hg.HG_EUNSUPPORTED, [dict(m=BIG), dict(k=BIG), dict(n=BIG)]),
    (linear_grad, hg.HG_EINVAL, [dict(m=-1), dict(dtype=4), dict(dw_dtype=2), dict(act=7),
                                 dict(act=1), dict(dy=None), dict(w=None), dict(x=None),
                                 dict(dx_stride=7), dict(dw_stride=7), dict(dy_stride=-1),
                                 dict(workspace=None), dict(workspace_bytes=1)]),
    (linear_grad, hg.HG_EUNSUPPORTED, [dict(m=BIG), dict(k=BIG), dict(n=BIG)]),
    (distill, hg.HG_EINVAL, [dict(rows=-1), dict(classes=0), dict(top=-1), dict(dtype=4),
                             dict(teacher_dtype=0), dict(temperature=0.0),
                             dict(temperature=float("inf")), dict(temperature=float("nan")),
                             dict(logits=None), dict(ids=None), dict(teacher=None),
                             dict(grad_stride=7), dict(logits_stride=-1), dict(ids_stride=-1)]),
    (distill, hg.HG_EUNSUPPORTED, [dict(rows=BIG), dict(classes=BIG), dict(top=1025)]),
]


@pytest.mark.parametrize("call,status,kw", [(c, s, k) for c, s, ks in CASES for k in ks])
def test_refused(call, status, kw):
    assert call(**kw) == status
    assert len(LIB.hg_last_error()) > 10


def test_null_and_empty():
    for f in (LIB.hg_rms_norm, LIB.hg_rms_norm_grad, LIB.hg_linear, LIB.hg_linear_grad,
              LIB.hg_distill):
        assert f(None, None) == hg.HG_EINVAL
    # nothing to do: no array is needed
    assert norm(rows=0, x=None, y=None) == hg.HG_OK
    assert linear(m=0, x=None, y=None) == hg.HG_OK
    assert linear(n=0, w=None, y=None) == hg.HG_OK
    assert distill(rows=0, logits=None) == hg.HG_OK
    assert distill(loss=None, grad=None) == hg.HG_OK
    assert norm_grad(dx=None) == hg.HG_OK


def test_workspaces():
    assert LIB.hg_rms_norm_grad_workspace(0, 8) == 0
    assert LIB.hg_rms_norm_grad_workspace(100, 8) >= 4 * 8
    assert LIB.hg_linear_workspace(0, 8, 8, 3) == 0
    # an activation's dz is held there
    assert (LIB.hg_linear_grad_workspace(1000, 64, 64, 3, 2)
            >= LIB.hg_linear_grad_workspace(1000, 64, 64, 3, 0) + 1000 * 64 * 2)


def test_feature_tables_are_not_in_8_bits():
    """The 8-bit type is for the dense operators only."""
    out = ctypes.c_void_p()
    nt = (hg.NTypeDesc * 1)(hg.NTypeDesc(10, ctypes.c_void_p(P), hg.HG_DT_E4M3, 4))
    assert LIB.hg_create(nt, 1, None, 0, None, None, ctypes.byref(out)) == hg.HG_EINVAL
