"""rms_norm and rms_norm_grad against their definition in 64 bits: every way a row is shared out
(by its length), types, odd lengths and strides, ids, rows that break, other streams, capture."""
import ctypes

import pytest
import torch

import dense_ref as R
import paper_2112_15345_amd as hg
from paper_2112_15345_amd import dense

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
# one length per way of sharing a row (in 16-byte vectors: 8, 16, 32, 64, 128, 256, 512, 1024 and
# past it), and odd ones
DIMS = [1, 3, 16, 33, 64, 100, 127, 128, 250, 512, 1000, 1024, 1999, 2048, 4095, 8192, 8200, 20_001]
ROWS = [0, 1, 5, 130]


def rand(*shape, dtype=F32, seed=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def check_forward(x, weight, residual, ids, eps, out, got):
    y, total, scale = got
    taken = x if ids is None else x[ids]
    h, want, _, rel = R.norm(taken, weight, residual, eps)
    # h is rounded to 32 bits before it is used: relative to the terms of the sum
    cancel = 0.0
    if residual is not None:
        assert total.dtype == x.dtype
        R.assert_close(total, h, R.rounding(h, x.dtype) + h.abs() * R.E, "sum")
    else:
        assert total is None
    size = want.abs() * rel + cancel
    if out == E4M3:
        assert y.dtype == E4M3 and scale.dtype == F32
        c = torch.clamp(want.abs().amax(1) / 448.0, min=2.0 ** -126)
        R.assert_close(scale, c, c * (rel + 4 * R.E) + 2.0 ** -149, "scale")
        value = y.double() * scale.double()[:, None]
        # half a step of e4m3: 2^-4 of the value, or 2^-10 scales below its smallest normal
        # (a value that its own error carries over a step's middle is the same distance off)
        R.assert_close(value, want, size * 2 + want.abs() * (2.0 ** -4) * 1.001
                       + scale.double()[:, None] * 2.0 ** -10 * 1.001, "y")
        assert float(y.float().abs().amax()) <= 448
    else:
        assert y.dtype == x.dtype and scale is None
        R.assert_close(y, want, R.rounding(want, x.dtype) + size, "y")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", DIMS)
def test_forward(dim, dtype):
    for rows in ROWS:
        for out in (dtype, E4M3):
            for weight, residual in ((None, None), (F32, None), (dtype, 1), (F32, 1)):
                x = rand(rows, dim, dtype=dtype, seed=rows + dim)
                w = None if weight is None else (1 + rand(dim, seed=7, scale=0.2)).to(weight)
                r = rand(rows, dim, dtype=dtype, seed=3) if residual else None
                got = hg.rms_norm(x, w, residual=r, eps=1e-5, out_dtype=out)
                if rows:
                    check_forward(x, w, r, None, 1e-5, out, got)
                else:
                    assert got[0].shape == (0, dim)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", DIMS)
def test_backward(dim, dtype):
    for rows in ROWS:
        for weight, dsum in ((None, None), (F32, 1), (dtype, None)):
            x = rand(rows, dim, dtype=dtype, seed=rows + dim)
            dy = rand(rows, dim, dtype=dtype, seed=11)
            w = None if weight is None else (1 + rand(dim, seed=7, scale=0.2)).to(weight)
            ds = rand(rows, dim, dtype=dtype, seed=5) if dsum else None
            dx, dw = hg.rms_norm_grad(dy, x, w, dsum=ds, eps=1e-5, want_dweight=True)
            assert dx.dtype == dtype and dw.dtype == F32
            if rows == 0:
                assert dx.shape == (0, dim) and not dw.any()
                continue
            h, _, s, rel = R.norm(x, w, None, 1e-5)
            g = dy.double() * (1.0 if w is None else w.double())
            mean = (g * h).mean(1, keepdim=True)
            want = s * (g - h * s * s * mean)
            # every factor is off by rel; mean(g h) by that of the terms' sizes
            size = rel * s * (g.abs() + h.abs() * s * s * 4 * (g * h).abs().mean(1, keepdim=True))
            if ds is not None:
                want = want + ds.double()
                size = size + R.E * (want.abs() + ds.double().abs())
            R.assert_close(dx, want, R.rounding(want, dtype) + 2 * size, "dx")
            terms = dy.double() * h * s
            R.assert_close(dw, terms.sum(0),
                           terms.abs().sum(0) * (rel + (rows + 8) * 2 * R.E) + 1e-30, "dweight")
            only = hg.rms_norm_grad(dy, x, w, dsum=ds, eps=1e-5, want_dx=False, want_dweight=True)
            assert only[0] is None and torch.equal(only[1], dw)
            only = hg.rms_norm_grad(dy, x, w, dsum=ds, eps=1e-5, want_dweight=False)
            assert only[1] is None and torch.equal(only[0], dx)


def test_gradient_by_differences():
    """The gradient of a weighted sum of y and sum by central differences in 64 bits, of the
    definition that the forward test holds the kernel to."""
    rows, dim, eps = 3, 37, 1e-5
    x, w = rand(rows, dim, seed=1), 1 + rand(dim, seed=2, scale=0.2)
    dy, ds = rand(rows, dim, seed=3), rand(rows, dim, seed=4)

    def value(x64, w64):
        y = R.norm(x64, w64, None, eps)[1]
        return (y * dy.double()).sum() + (x64 * ds.double()).sum()

    dx, dw = hg.rms_norm_grad(dy, x, w, dsum=ds, eps=eps)
    step = 1e-5
    for i, j in ((0, 0), (1, 5), (2, 36), (1, 20)):
        d = torch.zeros(rows, dim, dtype=torch.float64, device="cuda")
        d[i, j] = step
        num = (value(x.double() + d, w.double()) - value(x.double() - d, w.double())) / (2 * step)
        assert abs(float(num) - float(dx[i, j])) <= 1e-5 * (1 + abs(float(num)))
    for j in (0, 17, 36):
        d = torch.zeros(dim, dtype=torch.float64, device="cuda")
        d[j] = step
        num = (value(x.double(), w.double() + d) - value(x.double(), w.double() - d)) / (2 * step)
        assert abs(float(num) - float(dw[j])) <= 1e-5 * (1 + abs(float(num)))


@pytest.mark.parametrize("dtype,dim", [(F32, 128), (F32, 30), (BF16, 100), (F16, 3000), (BF16, 9000)])
def test_rows_by_id(dtype, dim):
    table = rand(50, dim, dtype=dtype, seed=1)
    ids = torch.tensor([3, 49, 0, 3, 17], device="cuda")
    r = rand(5, dim, dtype=dtype, seed=2)
    for residual in (None, r):
        check_forward(table, None, residual, ids, 1e-6, dtype,
                      hg.rms_norm(table, residual=residual, ids=ids))
    check_forward(table, None, None, ids, 1e-6, E4M3, hg.rms_norm(table, ids=ids, out_dtype=E4M3))
    dy = rand(5, dim, dtype=dtype, seed=4)
    by_id = hg.rms_norm_grad(dy, table, ids=ids, want_dweight=True)
    plain = hg.rms_norm_grad(dy, table[ids], want_dweight=True)
    assert torch.equal(by_id[0], plain[0]) and torch.equal(by_id[1], plain[1])
    # ids out of range: NaN rows, the others as they are
    wild = torch.tensor([3, 50, -1, 17, 1 << 40], device="cuda")
    y, _, _ = hg.rms_norm(table, ids=wild)
    y8, _, sc = hg.rms_norm(table, ids=wild, out_dtype=E4M3)
    good = hg.rms_norm(table[[3, 17]])[0]
    assert torch.equal(y[[0, 3]], good) and torch.isnan(y[[1, 2, 4]].float()).all()
    assert torch.isnan(y8[[1, 2, 4]].float()).all() and torch.isnan(sc[[1, 2, 4]]).all()
    assert not torch.isnan(sc[[0, 3]]).any()


def test_strides_and_layouts():
    big = rand(40, 300, dtype=BF16, seed=1)
    x = big[3:25:2, 5:106]                       # odd offset and stride, 101 columns
    r = rand(1, 101, dtype=BF16, seed=2).expand(11, 101)   # a broadcast residual: stride 0
    check_forward(x, None, r, None, 1e-6, BF16, hg.rms_norm(x, residual=r))
    t = rand(101, 11, dtype=BF16, seed=3).t()    # columns that are not contiguous
    check_forward(t, None, None, None, 1e-6, BF16, hg.rms_norm(t))
    dy = rand(1, 1, dtype=BF16, seed=4).expand(11, 101)
    a = hg.rms_norm_grad(dy, x, want_dweight=True)
    b = hg.rms_norm_grad(dy.contiguous(), x.contiguous(), want_dweight=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_offsets_past_32_bits():
    """Rows whose offset is past 2^31 and 2^32 elements."""
    rows, dim, stride = 70_001, 64, 65_536
    buf = torch.empty(rows * stride, dtype=BF16, device="cuda")
    x = buf.as_strided((rows, dim), (stride, 1))
    x.copy_(rand(rows, dim, dtype=BF16, seed=1))
    y, _, _ = hg.rms_norm(x)
    assert torch.equal(y, hg.rms_norm(x.contiguous())[0])
    ids = torch.tensor([rows - 1, 40_000, 0], device="cuda")
    assert torch.equal(hg.rms_norm(x, ids=ids)[0], y[ids])
    dx, dw = hg.rms_norm_grad(x, x, want_dweight=True)
    dx2, dw2 = hg.rms_norm_grad(x.contiguous(), x.contiguous(), want_dweight=True)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


@pytest.mark.parametrize("dim", [40, 256, 2000, 10_000])
def test_rows_that_break(dim):
    """NaN takes its row, an infinity its place; zero and tiny rows; the neighbours are unhurt."""
    x = rand(6, dim, seed=1)
    clean = hg.rms_norm(x)[0]
    x[1, dim // 2] = float("nan")
    x[2, 3] = float("inf")
    x[3] = 0
    x[4] *= 1e-30
    y, _, _ = hg.rms_norm(x, eps=1e-6)
    y8, _, sc = hg.rms_norm(x, eps=1e-6, out_dtype=E4M3)
    assert torch.isnan(y[1]).all() and torch.isnan(y8[1].float()).all() and torch.isnan(sc[1])
    assert torch.isnan(y[2, 3]) and not y[2, torch.arange(dim) != 3].any() and torch.isnan(sc[2])
    assert not y[3].any() and not y8[3].float().any() and float(sc[3]) == 2.0 ** -126
    assert torch.equal(y[[0, 5]], clean[[0, 5]])
    check_forward(x[4:5], None, None, None, 1e-6, F32, hg.rms_norm(x[4:5]))
    zero = hg.rms_norm(x[3:4], eps=0.0)[0]  # 0 times an infinite 1 / rms
    assert torch.isnan(zero).all()
    dx, dw = hg.rms_norm_grad(torch.ones_like(x), x, want_dweight=True)
    assert torch.isnan(dx[1]).all() and not torch.isnan(dx[[0, 4, 5]]).any()


def test_in_place_outputs():
    """sum over the residual and y over x, as the C entry allows, for a row in registers and one
    that is read twice."""
    for dim in (96, 9000):
        x, r = rand(7, dim, dtype=BF16, seed=1), rand(7, dim, dtype=BF16, seed=2)
        y, h, _ = hg.rms_norm(x, residual=r)
        a = dense.NormArgs(7, dim, dense.HG_DT_BF16, dense.HG_DT_BF16, dense.HG_DT_NONE, 1e-6,
                           x.data_ptr(), dim, 7, None, r.data_ptr(), dim, None, x.data_ptr(), dim,
                           None, r.data_ptr(), dim)
        assert hg.load_library().hg_rms_norm(
            ctypes.byref(a), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == hg.HG_OK
        assert torch.equal(x, y) and torch.equal(r, h)


def test_other_stream_and_capture():
    x, w = rand(300, 512, dtype=BF16, seed=1), 1 + rand(512, seed=2, scale=0.1)
    dy = rand(300, 512, dtype=BF16, seed=3)
    want, grads = hg.rms_norm(x, w, residual=x), hg.rms_norm_grad(dy, x, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = hg.rms_norm(x, w, residual=x, stream=s)
    back = hg.rms_norm_grad(dy, x, w, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(back[0], grads[0]) and torch.equal(back[1], grads[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = hg.rms_norm(x, w, residual=x)
        back = hg.rms_norm_grad(dy, x, w)
    for seed in (5, 6, 7):
        x.copy_(rand(300, 512, dtype=BF16, seed=seed))
        graph.replay()
        want, grads = hg.rms_norm(x, w, residual=x), hg.rms_norm_grad(dy, x, w)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(back[0], grads[0]) and torch.equal(back[1], grads[1])


def test_binding_refuses():
    x = rand(4, 8)
    for bad in (dict(x=x[0]), dict(x=x.double()), dict(x=x, weight=rand(7)),
                dict(x=x, weight=rand(8).to(F16)), dict(x=x, residual=rand(3, 8)),
                dict(x=x, residual=rand(4, 8, dtype=BF16)), dict(x=x, out_dtype=F16),
                dict(x=x, ids=torch.zeros(2, dtype=torch.int32, device="cuda")),
                dict(x=x.cpu())):
        with pytest.raises(ValueError):
            hg.rms_norm(**bad)
    with pytest.raises(hg.HGError):
        hg.rms_norm(x, eps=-1.0)
    with pytest.raises(ValueError):
        hg.rms_norm_grad(rand(4, 7), x)
