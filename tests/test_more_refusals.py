"""The C entry points of layer norms, embeddings, integers and kept rows refuse bad arguments on the
host, before any device work, and the binding refuses unfit tensors (no GPU needed; the pointers are
never read)."""
import ctypes
import types

import pytest
import torch

import paper_2112_15345_amd as hg
from paper_2112_15345_amd import dense

P = 0x1000  # never dereferenced
BIG = 1 << 31
NAN, INF = float("nan"), float("inf")
LIB = hg.load_library()


def layer_norm(**kw):
    v = dict(rows=2, dim=8, dtype=1, out_dtype=1, eps=1e-6, x=P, x_stride=8, x_rows=2, y=P, y_stride=8)
    return LIB.hg_layer_norm(ctypes.byref(dense.LayerNormArgs(**{**v, **kw})), None)


def layer_norm_grad(**kw):
    v = dict(rows=2, dim=8, dtype=1, eps=1e-6, x=P, x_stride=8, x_rows=2, dy=P, dy_stride=8, dx=P,
             dx_stride=8)
    return LIB.hg_layer_norm_grad(ctypes.byref(dense.LayerNormGradArgs(**{**v, **kw})), None)


def embed(**kw):
    v = dict(n=2, nodes=5, dim=8, table_dtype=1, out_dtype=3, scale=1.0, table=P, table_stride=8, ids=P,
             y=P, y_stride=8)
    return LIB.hg_embed(ctypes.byref(dense.EmbedArgs(**{**v, **kw})), None)


def embed_grad(**kw):
    v = dict(n=2, nodes=5, dim=8, dtype=3, out_dtype=1, scale=1.0, dy=P, dy_stride=8, ids=P, dtable=P,
             dtable_stride=8, workspace=P, workspace_bytes=1 << 40)
    return LIB.hg_embed_grad(ctypes.byref(dense.EmbedGradArgs(**{**v, **kw})), None)


def quantize(**kw):
    v = dict(rows=2, dim=300, dtype=3, group=128, x=P, x_stride=300, q=P, q_stride=300, scale=P)
    return LIB.hg_quantize(ctypes.byref(dense.QuantizeArgs(**{**v, **kw})), None)


def dequantize(**kw):
    v = dict(rows=2, dim=300, dtype=3, group=128, q=P, q_stride=300, scale=P, x=P, x_stride=300)
    return LIB.hg_dequantize(ctypes.byref(dense.DequantizeArgs(**{**v, **kw})), None)


def integers(**kw):
    v = dict(m=2, k=8, n=4, dtype=6, out_dtype=3, bias_dtype=1, act=0, x=P, x_stride=8, w=P,
             w_stride=8, x_scale=P, w_scale=P, y=P, y_stride=4, workspace=P, workspace_bytes=1 << 40)
    return LIB.hg_linear(ctypes.byref(dense.LinearArgs(**{**v, **kw})), None)


def grad_kept(group=0, x_scale=P, pre_scale=P, **kw):
    v = dict(m=2, k=8, n=4, dtype=3, dw_dtype=3, act=1, dy=P, dy_stride=4, pre=P, pre_stride=4, x=P,
             x_stride=8, w=P, w_stride=8, dx=P, dx_stride=8, dw=P, dw_stride=8, dbias=P, workspace=P,
             workspace_bytes=1 << 40)
    args = dense.LinearGradKeptArgs(dense.LinearGradArgs(**{**v, **kw}), group, x_scale, pre_scale)
    return LIB.hg_linear_grad_kept(ctypes.byref(args), None)


CASES = [
    (layer_norm, hg.HG_EINVAL,
     [dict(rows=-1), dict(dim=0), dict(dtype=0), dict(dtype=4), dict(dtype=6), dict(out_dtype=2),
      dict(out_dtype=5), dict(weight_dtype=2), dict(weight_dtype=1), dict(bias_dtype=3),
      dict(bias_dtype=1), dict(eps=-1.0), dict(eps=NAN), dict(x=None), dict(x_stride=-1),
      dict(y=None), dict(y_stride=7), dict(sum=P, sum_stride=7), dict(out_dtype=4),
      dict(out_dtype=6), dict(ids=P, x_rows=-1), dict(residual=P, residual_stride=-8)]),
    (layer_norm, hg.HG_EUNSUPPORTED, [dict(rows=BIG), dict(dim=BIG)]),
    (layer_norm_grad, hg.HG_EINVAL,
     [dict(rows=-1), dict(dim=0), dict(dtype=6), dict(weight_dtype=3), dict(weight_dtype=1),
      dict(dy=None), dict(x=None), dict(dx_stride=7), dict(dsum=P, dsum_stride=-1), dict(eps=INF),
      dict(dweight=P), dict(dbias=P), dict(dbias=P, workspace=P, workspace_bytes=127)]),
    (layer_norm_grad, hg.HG_EUNSUPPORTED, [dict(rows=BIG), dict(dim=BIG)]),
    (embed, hg.HG_EINVAL,
     [dict(n=-1), dict(nodes=-1), dict(dim=0), dict(table_dtype=0), dict(table_dtype=4),
      dict(out_dtype=6), dict(scale=NAN), dict(scale=INF), dict(table=None), dict(table_stride=-1),
      dict(ids=None), dict(y=None), dict(y_stride=7)]),
    (embed, hg.HG_EUNSUPPORTED, [dict(n=BIG), dict(nodes=BIG), dict(dim=BIG)]),
    (embed_grad, hg.HG_EINVAL,
     [dict(n=-1), dict(nodes=-1), dict(dim=0), dict(dtype=0), dict(dtype=4), dict(out_dtype=2),
      dict(add=2), dict(add=-1), dict(add=1, out_dtype=3), dict(scale=-INF), dict(dy=None),
      dict(dy_stride=-1), dict(ids=None), dict(dtable=None), dict(dtable_stride=7),
      dict(workspace=None), dict(workspace_bytes=15)]),
    (embed_grad, hg.HG_EUNSUPPORTED, [dict(n=BIG), dict(nodes=BIG), dict(dim=BIG)]),
    (quantize, hg.HG_EINVAL,
     [dict(rows=-1), dict(dim=0), dict(dtype=0), dict(dtype=4), dict(dtype=6), dict(group=64),
      dict(group=-1), dict(x=None), dict(x_stride=-1), dict(q=None), dict(q_stride=299),
      dict(scale=None)]),
    (quantize, hg.HG_EUNSUPPORTED, [dict(rows=BIG), dict(dim=BIG)]),
    (dequantize, hg.HG_EINVAL,
     [dict(rows=-1), dict(dim=0), dict(dtype=6), dict(group=127), dict(x=None), dict(x_stride=299),
      dict(q=None), dict(q_stride=-1), dict(scale=None)]),
    (dequantize, hg.HG_EUNSUPPORTED, [dict(rows=BIG), dict(dim=BIG)]),
    (integers, hg.HG_EINVAL,
     [dict(m=-1), dict(out_dtype=0), dict(out_dtype=4), dict(out_dtype=6), dict(x_scale=None),
      dict(w_scale=None), dict(x=None), dict(w=None), dict(y_stride=3), dict(act=4),
      dict(m=1, k=1 << 16, n=4, x_stride=1 << 16, w_stride=1 << 16, workspace=None)]),
    (integers, hg.HG_EUNSUPPORTED, [dict(m=BIG), dict(k=1 << 17), dict(n=BIG)]),
    (grad_kept, hg.HG_EINVAL,
     [dict(group=64), dict(m=-1), dict(dtype=6), dict(dw_dtype=6), dict(dy=None), dict(pre=None),
      dict(pre_stride=-1), dict(x=None), dict(x_stride=-1), dict(w=None), dict(dx_stride=7),
      dict(dw_stride=7), dict(workspace=None), dict(workspace_bytes=31)]),
    (grad_kept, hg.HG_EUNSUPPORTED, [dict(m=BIG), dict(k=BIG), dict(n=BIG)]),
]


@pytest.mark.parametrize("call,status,kw", [(c, s, k) for c, s, ks in CASES for k in ks])
def test_refused(call, status, kw):
    assert call(**kw) == status
    assert len(LIB.hg_last_error()) > 10


def test_null_and_empty():
    for f in (LIB.hg_layer_norm, LIB.hg_layer_norm_grad, LIB.hg_embed, LIB.hg_embed_grad,
              LIB.hg_quantize, LIB.hg_dequantize, LIB.hg_linear_grad_kept):
        assert f(None, None) == hg.HG_EINVAL
    assert layer_norm(rows=0, x=None, y=None) == hg.HG_OK
    assert layer_norm_grad(dx=None) == hg.HG_OK
    assert embed(n=0, table=None, ids=None, y=None) == hg.HG_OK
    assert embed_grad(n=0, add=1, dtable=None) == hg.HG_OK
    assert embed_grad(nodes=0, dtable=None) == hg.HG_OK
    assert LIB.hg_layer_norm_grad_workspace(0, 8) == 0
    assert quantize(rows=0, x=None, q=None, scale=None) == hg.HG_OK
    assert dequantize(rows=0, x=None, q=None, scale=None) == hg.HG_OK
    # the rows that x stands for are made there
    assert (LIB.hg_linear_grad_kept_workspace(1000, 64, 64, 3, 2)
            >= LIB.hg_linear_grad_workspace(1000, 64, 64, 3, 2) + 1000 * 64 * 2)
    assert LIB.hg_embed_grad_workspace(0, 9, 8) == 0
    for n in (1, 4096, 4097, 1 << 18, (1 << 31) - 1):
        for nodes in (1, 1000, (1 << 31) - 1):
            assert LIB.hg_embed_grad_workspace(n, nodes, 24) >= 8 * n  # (the sorted pairs)
    assert LIB.hg_layer_norm_grad_workspace(100, 8) >= 2 * 4 * 8


def test_tensors_that_do_not_fit():
    x, g = torch.zeros(4, 8), torch.zeros(4, 8, requires_grad=True)
    for call in (lambda: hg.layer_norm(g), lambda: hg.layer_norm(x, torch.zeros(8, requires_grad=True)),
                 lambda: hg.layer_norm(x, bias=torch.zeros(8, requires_grad=True)),
                 lambda: hg.layer_norm(x, residual=g), lambda: hg.embed(g, torch.zeros(2).long()),
                 lambda: hg.embed_grad(x, torch.zeros(4).long(), 4, into=g),
                 lambda: hg.quantize(g),
                 lambda: hg.dequantize(x.to(torch.int8), torch.zeros(4, requires_grad=True))):
        with pytest.raises(ValueError, match="gradient"):
            call()
    for call in (lambda: hg.layer_norm(x), lambda: hg.layer_norm_grad(g, g),
                 lambda: hg.embed(x, torch.zeros(2).long()),
                 lambda: hg.embed_grad(g, torch.zeros(4).long(), 4), lambda: hg.quantize(x),
                 lambda: hg.dequantize(x.to(torch.int8), x[0])):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_stream_by_position():
    """linear_grad's tenth argument is the stream, as it was before rows could be kept."""
    t = torch.zeros(2, 2)
    stream = types.SimpleNamespace(device=torch.device("cuda", 0))
    with pytest.raises(ValueError, match="a stream of cuda:0"):
        hg.linear_grad(t, t, t, None, None, True, True, True, None, stream)


# (each is refused before any work on a device: dy's rows in the table's, or the table's in dy's)
@pytest.mark.parametrize("kw", [
    dict(), dict(add=1, dtype=1), dict(dtable=P + 16, dtable_stride=8), dict(dtable=P - 4 * 8 * 4),
    dict(dtype=1, dy_stride=0, dtable=P - 60), dict(n=1, dy_stride=1 << 62),
    dict(dtype=1, dy_stride=24, dtable_stride=16, dtable=P + 32),
    dict(dtype=1, dy_stride=32, dtable_stride=16, dtable=P + 4 * 7),
    dict(dtype=1, dy_stride=32, dtable_stride=16, dtable=P + 4 * 25 - 4 * 64),
])
def test_gradient_in_the_rows_that_it_is_made_of(kw):
    assert embed_grad(**kw) == hg.HG_EINVAL
    assert b"memory" in LIB.hg_last_error()
