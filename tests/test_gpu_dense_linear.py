"""linear and linear_grad against their definition in 64 bits: types, one row to many, odd sizes,
strides, lengths of zero, split depths, activations, infinities, other streams, capture."""
import ctypes

import pytest
import torch

import dense_ref as R
import paper_2112_15345_amd as hg
from paper_2112_15345_amd import dense

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
ACTS = ["none", "relu", "gelu", "silu"]


def rand(*shape, dtype=F32, seed=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def to_8_bits(x):
    c = torch.clamp(x.abs().amax(1) / 448.0, min=2.0 ** -126) if x.numel() else \
        torch.ones(x.shape[0], device="cuda")
    return (x / c[:, None]).to(E4M3), c


def check(x, w, got, bias=None, act="none", residual=None, xs=None, ws=None, out=None):
    """A product's error: its sum of k terms, held to k 2^-23 of the terms' sizes, and the scales'
    and the bias's roundings; an activation's slope is at most 1.13, its own error 16 units of
    2^-24 of its argument."""
    y, pre = got
    out = out or x.dtype
    k = x.shape[1]
    a, b = x.double(), w.double()
    if xs is not None:
        a, b = a * xs.double()[:, None], b * ws.double()[:, None]
    z = a @ b.t()
    size = (a.abs() @ b.abs().t()) * ((2 * k + 8) * R.E)
    if bias is not None:
        z = z + bias.double()
        size = size + R.E * z.abs()
    v = R.act(z, act)
    vsize = 1.13 * size + 16 * R.E * z.abs() if act != "none" else size
    if residual is not None:
        v = v + residual.double()
        vsize = vsize + R.E * v.abs()
    assert y.dtype == out and y.shape == z.shape
    R.assert_close(y, v, R.rounding(v, out) + vsize, "y")
    if pre is not None:
        R.assert_close(pre, z, R.rounding(z, out) + size, "pre")


# m, k, n: one row, a few, a tile and its neighbours, odd everything, short and long depths
SIZES = [(1, 1, 1), (1, 64, 128), (1, 2048, 1000), (3, 100, 47), (7, 4096, 256), (16, 512, 512),
         (17, 33, 65), (31, 96, 40), (33, 130, 129), (64, 768, 64), (65, 1000, 100),
         (127, 129, 255), (128, 128, 128), (129, 64, 257), (200, 8, 300), (257, 4099, 130),
         (300, 2000, 16), (513, 200, 511), (1000, 64, 24), (2050, 72, 136), (5000, 136, 260)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16, E4M3])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_forward(m, k, n, dtype):
    outs = [BF16, F32, F16] if dtype == E4M3 else [dtype]
    for i, act in enumerate(ACTS):
        out = outs[i % len(outs)]
        x, w = rand(m, k, seed=m + k), rand(n, k, seed=n, scale=k ** -0.5)
        xs = ws = None
        if dtype == E4M3:
            (x, xs), (w, ws) = to_8_bits(x), to_8_bits(w)
        else:
            x, w = x.to(dtype), w.to(dtype)
        bias = [None, rand(n, seed=4), rand(n, seed=4, dtype=BF16), rand(n, seed=4)][i]
        res = rand(m, n, dtype=out, seed=5) if i in (1, 3) else None
        got = hg.linear(x, w, bias=bias, act=act, residual=res, x_scale=xs, w_scale=ws,
                        out_dtype=out, keep_pre=i >= 2)
        assert (got[1] is not None) == (i >= 2)
        check(x, w, got, bias, act, res, xs, ws, out)


def check_grad(dy, x, w, pre, act, got, dw_dtype=None):
    dx, dw, db = got
    dtype = x.dtype
    slope = torch.ones_like(dy, dtype=torch.float64) if act == "none" else \
        R.act_slope(pre.double(), act)
    dz = dy.double() * slope
    # dz in 32 bits, then rounded to the type before the products (with an activation)
    dz_size = torch.zeros_like(dz)
    if act != "none":
        dz_size = dy.double().abs() * 32 * R.E * (1 + pre.double().abs())
    dz_rounded = dz_size + (R.rounding(dz, dtype) if act != "none" else 0)
    for what, got_, want, size, terms, depth in (
            ("dx", dx, dz @ w.double(), dz_rounded @ w.double().abs(),
             dz.abs() @ w.double().abs(), dy.shape[1]),
            ("dw", dw, dz.t() @ x.double(), dz_rounded.t() @ x.double().abs(),
             dz.abs().t() @ x.double().abs(), dy.shape[0])):
        if got_ is None:
            continue
        out = dtype if what == "dx" else (dw_dtype or dtype)
        assert got_.dtype == out, what
        R.assert_close(got_, want, R.rounding(want, out) + size * 1.01 + terms * (2 * depth + 8) * R.E,
                       what)
    if db is not None:
        assert db.dtype == F32
        R.assert_close(db, dz.sum(0), dz_size.sum(0)
                       + dz.abs().sum(0) * (2 * dy.shape[0] + 8) * R.E + 1e-37, "dbias")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_backward(m, k, n, dtype):
    for i, act in enumerate(ACTS):
        x, w = rand(m, k, dtype=dtype, seed=1), rand(n, k, dtype=dtype, seed=2, scale=k ** -0.5)
        dy = rand(m, n, dtype=dtype, seed=3)
        pre = rand(m, n, dtype=dtype, seed=4, scale=2.0) if act != "none" else None
        dw_dtype = F32 if i % 2 == 0 else None
        got = hg.linear_grad(dy, x, w, pre=pre, act=act, dw_dtype=dw_dtype)
        check_grad(dy, x, w, pre, act, got, dw_dtype)
        again = hg.linear_grad(dy, x, w, pre=pre, act=act, dw_dtype=dw_dtype)
        assert all(torch.equal(a, b) for a, b in zip(got, again))
        for keep in range(3):
            want = [j == keep for j in range(3)]
            some = hg.linear_grad(dy, x, w, pre=pre, act=act, want_dx=want[0], want_dw=want[1],
                                  want_dbias=want[2], dw_dtype=dw_dtype)
            for j in range(3):
                assert (some[j] is not None) == want[j]
                if want[j]:
                    assert torch.equal(some[j], got[j])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,k,n", [(70_000, 40, 72), (20_011, 300, 17), (9, 70_000, 24),
                                   (40, 24, 50_000), (4096, 1024, 512)])
def test_long_axes(m, k, n, dtype):
    x, w = rand(m, k, dtype=dtype, seed=1), rand(n, k, dtype=dtype, seed=2, scale=k ** -0.5)
    check(x, w, hg.linear(x, w))
    dy = rand(m, n, dtype=dtype, seed=3)
    check_grad(dy, x, w, None, "none", hg.linear_grad(dy, x, w, dw_dtype=F32), F32)


@pytest.mark.parametrize("act", ACTS)
def test_gradient_by_differences(act):
    """The gradient of a weighted sum of y by central differences in 64 bits, of the definition
    that the forward test holds the kernel to."""
    m, k, n = 4, 21, 13
    x, w, b = rand(m, k, seed=1), rand(n, k, seed=2, scale=0.3), rand(n, seed=3)
    dy = rand(m, n, seed=4)
    pre = hg.linear(x, w, bias=b, act=act, keep_pre=True)[1]
    dx, dw, db = hg.linear_grad(dy, x, w, pre=pre, act=act)

    def value(x64, w64, b64):
        return (R.act(x64 @ w64.t() + b64, act) * dy.double()).sum()

    base = [x.double(), w.double(), b.double()]
    step = 1e-5
    for which, got, places in ((0, dx, [(0, 0), (3, 20), (2, 7)]), (1, dw, [(0, 0), (12, 20), (5, 3)]),
                               (2, db, [(0,), (12,)])):
        for at in places:
            up, down = [t.clone() for t in base], [t.clone() for t in base]
            up[which][at] += step
            down[which][at] -= step
            num = float((value(*up) - value(*down)) / (2 * step))
            assert abs(num - float(got[at])) <= 2e-5 * (1 + abs(num))


def test_lengths_of_zero():
    for dtype in (F32, BF16):
        b, r = rand(5, seed=1), rand(3, 5, dtype=dtype, seed=2)
        y, pre = hg.linear(rand(3, 0, dtype=dtype), rand(5, 0, dtype=dtype), bias=b, act="silu",
                           residual=r, keep_pre=True)
        check(rand(3, 0, dtype=dtype), rand(5, 0, dtype=dtype), (y, pre), b, "silu", r)
        assert hg.linear(rand(0, 4, dtype=dtype), rand(5, 4, dtype=dtype))[0].shape == (0, 5)
        assert hg.linear(rand(3, 4, dtype=dtype), rand(0, 4, dtype=dtype))[0].shape == (3, 0)
        dx, dw, db = hg.linear_grad(rand(0, 5, dtype=dtype), rand(0, 4, dtype=dtype),
                                    rand(5, 4, dtype=dtype))
        assert dx.shape == (0, 4) and dw.shape == (5, 4) and not dw.any() and not db.any()
        dx, dw, db = hg.linear_grad(rand(3, 0, dtype=dtype), rand(3, 4, dtype=dtype),
                                    rand(0, 4, dtype=dtype))
        assert dx.shape == (3, 4) and not dx.any() and dw.shape == (0, 4)
        dx, dw, db = hg.linear_grad(rand(3, 5, dtype=dtype), rand(3, 0, dtype=dtype),
                                    rand(5, 0, dtype=dtype))
        assert dx.shape == (3, 0) and dw.shape == (5, 0) and db.any()
    y, _ = hg.linear(torch.empty(2, 0, dtype=E4M3, device="cuda"),
                     torch.empty(4, 0, dtype=E4M3, device="cuda"), bias=rand(4, seed=1),
                     x_scale=torch.ones(2, device="cuda"), w_scale=torch.ones(4, device="cuda"))
    assert torch.equal(y, rand(4, seed=1).to(BF16).expand(2, 4))


@pytest.mark.parametrize("dtype", [F32, F16, BF16, E4M3])
def test_strides_and_layouts(dtype):
    """Odd starts and strides, broadcast rows, columns that are not contiguous: the results of
    packed copies, bit for bit where the same kernel runs, else within its bounds."""
    for m, k, n in ((6, 64, 40), (150, 99, 133), (150, 128, 128)):
        xb, wb = rand(m * 2 + 1, k + 5, seed=1), rand(n + 2, k + 9, seed=2, scale=k ** -0.5)
        kw = {}
        if dtype == E4M3:
            (xb, xs), (wb, ws) = to_8_bits(xb), to_8_bits(wb)
            x, w = xb[1::2, 3:3 + k], wb[2:, 1:1 + k]
            kw = dict(x_scale=xs[1::2], w_scale=ws[2:])
            out = BF16
        else:
            xb, wb = xb.to(dtype), wb.to(dtype)
            x, w = xb[1::2, 3:3 + k], wb[2:, 1:1 + k]
            out = dtype
        res = rand(1, n, dtype=out, seed=3).expand(m, n)
        got = hg.linear(x, w, residual=res, **kw)
        check(x, w, got, residual=res, xs=kw.get("x_scale"), ws=kw.get("w_scale"), out=out)
        xt = x.t().contiguous().t()
        got = hg.linear(xt, w, **kw)
        check(x, w, got, xs=kw.get("x_scale"), ws=kw.get("w_scale"), out=out)
        if dtype != E4M3:
            dy = rand(m, 2 * n + 1, dtype=dtype, seed=4)[:, 1:1 + n]
            pre = rand(m, n + 3, dtype=dtype, seed=5)[:, 2:2 + n]
            for act in ("none", "gelu"):
                p = None if act == "none" else pre
                check_grad(dy, x, w, p, act, hg.linear_grad(dy, x, w, pre=p, act=act))
            wide = rand(1, n, dtype=dtype, seed=6).expand(m, n)
            check_grad(wide, x, w, None, "none", hg.linear_grad(wide, x, w))


def test_offsets_past_32_bits():
    m, k, n, stride = 66_001, 64, 72, 65_536
    buf = torch.empty(m * stride, dtype=BF16, device="cuda")
    x = buf.as_strided((m, k), (stride, 1))
    x.copy_(rand(m, k, dtype=BF16, seed=1))
    w = rand(n, k, dtype=BF16, seed=2, scale=0.1)
    assert torch.equal(hg.linear(x, w)[0], hg.linear(x.contiguous(), w)[0])
    assert torch.equal(hg.linear(x[-3:], w)[0], hg.linear(x[-3:].contiguous(), w)[0])
    dy = rand(m, n, dtype=BF16, seed=3)
    a, b = hg.linear_grad(dy, x, w), hg.linear_grad(dy, x.contiguous(), w)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("m", [2, 40, 300])
def test_values_that_are_not_finite(m, dtype):
    """NaN and infinities stay in their rows and columns; rows past the end add nothing."""
    k, n = 72, 50
    x, w = rand(m, k, dtype=dtype, seed=1), rand(n, k, dtype=dtype, seed=2, scale=0.1)
    clean = hg.linear(x, w, act="gelu")[0]
    x[0, 5] = float("nan")
    x[1, 70] = float("inf")
    w[7] = 0
    w[9, 3] = float("-inf")
    for act in ACTS:
        y = hg.linear(x, w, act=act)[0]
        z = x.double() @ w.double().t()
        cols = [j for j in range(n) if j not in (7, 9)]
        if m > 2 and act == "gelu":
            assert torch.equal(y[2:, cols], clean[2:, cols])
        assert torch.isnan(y[0]).all() and torch.isnan(y[1, 7])
        want = R.act(z, act)[1, cols]
        pos = z[1, cols] > 0
        assert (y[1, cols][pos] == float("inf")).all()
        if act == "none":
            assert (y[1, cols][~pos] == float("-inf")).all()
        else:
            assert not y[1, cols][~pos].any()
        del want


def test_residual_in_place():
    x, w = rand(200, 96, dtype=BF16, seed=1), rand(130, 96, dtype=BF16, seed=2)
    r = rand(200, 130, dtype=BF16, seed=3)
    want = hg.linear(x, w, residual=r)[0]
    lib = hg.load_library()
    need = lib.hg_linear_workspace(200, 96, 130, dense.HG_DT_BF16)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    a = dense.LinearArgs(200, 96, 130, dense.HG_DT_BF16, dense.HG_DT_BF16, 0, 0, x.data_ptr(), 96,
                         None, w.data_ptr(), 96, None, None, r.data_ptr(), 130, r.data_ptr(), 130,
                         None, 0, ws.data_ptr(), ws.numel())
    assert lib.hg_linear(ctypes.byref(a), ctypes.c_void_p(
        torch.cuda.current_stream().cuda_stream)) == hg.HG_OK
    assert torch.equal(r, want)


def test_other_stream_and_capture():
    """(300 rows of a deep product: one that is split and joined.)"""
    x, w, b = rand(300, 4096, dtype=BF16, seed=1), rand(136, 4096, dtype=BF16, seed=2), rand(136)
    dy, pre = rand(300, 136, dtype=BF16, seed=3), rand(300, 136, dtype=BF16, seed=4)

    def calls(**kw):
        return (hg.linear(x, w, bias=b, act="silu", **kw)[0],
                *hg.linear_grad(dy, x, w, pre=pre, act="silu", **kw),
                hg.linear(x[:1], w, bias=b, **kw)[0])

    want = calls()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = calls(stream=s)
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    for seed in (5, 6, 7):
        x.copy_(rand(300, 4096, dtype=BF16, seed=seed))
        graph.replay()
        want = calls()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_binding_refuses():
    x, w = rand(4, 8, dtype=BF16), rand(5, 8, dtype=BF16)
    x8, xs = to_8_bits(rand(4, 8))
    w8, ws = to_8_bits(rand(5, 8))
    for kw in (dict(x=x[0], w=w), dict(x=x, w=rand(5, 7, dtype=BF16)), dict(x=x, w=w.float()),
               dict(x=x, w=w, act="tanh"), dict(x=x, w=w, bias=rand(4)),
               dict(x=x, w=w, residual=rand(4, 5)), dict(x=x, w=w, x_scale=xs),
               dict(x=x, w=w, out_dtype=F32), dict(x=x8, w=w8), dict(x=x8, w=w8, x_scale=xs),
               dict(x=x8, w=w8, x_scale=xs[:3], w_scale=ws),
               dict(x=x8, w=w8, x_scale=xs, w_scale=ws, out_dtype=E4M3), dict(x=x.cpu(), w=w)):
        with pytest.raises(ValueError):
            hg.linear(**kw)
    dy = rand(4, 5, dtype=BF16)
    for kw in (dict(dy=dy[:3], x=x, w=w), dict(dy=dy, x=x, w=w, act="gelu"),
               dict(dy=dy, x=x, w=w, dw_dtype=F16), dict(dy=dy, x=x8, w=w8)):
        with pytest.raises(ValueError):
            hg.linear_grad(**kw)
