"""layer_norm and layer_norm_grad against their definition in 64 bits: every way a row is shared out
(by its length), types, odd lengths and strides, ids, 8-bit results, rows that break, rows far from 0,
other streams, capture."""
import ctypes

import pytest
import torch

import dense_ref as R
import paper_2112_15345_amd as hg
from paper_2112_15345_amd import dense

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
E4M3, I8 = torch.float8_e4m3fn, torch.int8
# one length per way of sharing a row (in 16-byte vectors: 8 .. 1024 and past it), and odd ones
DIMS = [1, 2, 3, 16, 33, 64, 100, 127, 250, 512, 1000, 1024, 1999, 2048, 4095, 8192, 8200, 20_001]
E = R.E


def rand(*shape, dtype=F32, seed=0, scale=1.0, shift=0.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale + shift).to(dtype)


class Ref:
    """The definition, and how far each of its steps may be off in 32 bits: dd for d = h - mean(h)
    (a sum of D terms, the subtraction, the rounding of x + residual), rel for s (the sum of
    squares of d's that are dd off, rsqrt)."""

    def __init__(self, x, residual, eps):
        self.h = h = x.double() if residual is None else x.double() + residual.double()
        D = h.shape[1]
        self.d = d = h - h.mean(1, keepdim=True)
        var = d.square().mean(1, keepdim=True)
        self.s = 1 / torch.sqrt(var + eps)
        self.sum_off = (2 * D + 4) * E  # of a mean over the row, in parts of its terms' sizes
        self.dd = self.sum_off * h.abs().mean(1, keepdim=True) + E * (d.abs() + h.abs())
        off = 2 * (d.abs() * self.dd).mean(1, keepdim=True) + self.dd.square().mean(1, keepdim=True)
        self.rel = 0.55 * (off / (var + eps) + self.sum_off) + 8 * E

    def forward(self, weight, bias):
        w = 1.0 if weight is None else weight.double()
        b = 0.0 if bias is None else bias.double()
        n = self.d * self.s * w
        size = (self.s * w * self.dd).abs() * (1 + self.rel) + n.abs() * (self.rel + 4 * E)
        return n + b, size + (n + b).abs() * 2 * E

    def backward(self, dy, weight):
        """(dx, its bound, the terms of dweight, their bound)"""
        s, d, rel = self.s, self.d, self.rel
        dy = dy.double()
        g = dy * (1.0 if weight is None else weight.double())
        mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
        k = mean(g * d) * s * s
        gm_off = self.sum_off * mean(g.abs())
        k_off = s * s * (self.sum_off * mean((g * d).abs()) + mean(g.abs() * self.dd)) \
            + k.abs() * (2 * rel + 4 * E)
        inner = g - mean(g) - d * k
        size = s * (4 * E * (g.abs() + mean(g).abs() + (d * k).abs()) + gm_off
                    + self.dd * k.abs() + d.abs() * k_off) + s * inner.abs() * rel
        n_off = s * self.dd + (s * d).abs() * (rel + 4 * E)
        return s * inner, 1.1 * size, dy * d * s, dy.abs() * n_off


def check_forward(x, weight, bias, residual, eps, out, got):
    y, total, scale = got
    ref = Ref(x, residual, eps)
    want, size = ref.forward(weight, bias)
    if residual is not None:
        assert total.dtype == x.dtype
        R.assert_close(total, ref.h, R.rounding(ref.h, x.dtype) + ref.h.abs() * E, "sum")
    else:
        assert total is None
    if out not in (E4M3, I8):
        assert y.dtype == x.dtype and scale is None
        R.assert_close(y, want, R.rounding(want, x.dtype) + size, "y")
        return
    top = 448.0 if out == E4M3 else 127.0
    assert y.dtype == out and scale.dtype == F32
    c = torch.clamp(want.abs().amax(1) / top, min=2.0 ** -126)
    R.assert_close(scale, c, size.amax(1) / top + c * 4 * E + 2.0 ** -149, "scale")
    value = y.double() * scale.double()[:, None]
    # half a step: 2^-4 of the value (or 2^-10 scales below the smallest normal) in e4m3, half a
    # scale in integers; an error that carries a value over a step's middle is as far off
    step = want.abs() * 2.0 ** -4 + scale.double()[:, None] * 2.0 ** -10 if out == E4M3 \
        else scale.double()[:, None] * 0.5
    R.assert_close(value, want, size * 2 + step * 1.001, "y")
    assert float(y.float().abs().amax()) <= top


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", DIMS)
def test_forward(dim, dtype):
    for rows in (0, 1, 5, 130):
        for out, weight, bias, residual in ((dtype, None, None, 0), (dtype, F32, dtype, 1),
                                            (dtype, dtype, F32, 0), (E4M3, F32, F32, 1),
                                            (I8, None, F32, 0), (I8, F32, F32, 1)):
            x = rand(rows, dim, dtype=dtype, seed=rows + dim, shift=0.5)
            w = None if weight is None else (1 + rand(dim, seed=7, scale=0.2)).to(weight)
            b = None if bias is None else rand(dim, dtype=bias, seed=8, scale=0.3)
            r = rand(rows, dim, dtype=dtype, seed=3) if residual else None
            got = hg.layer_norm(x, w, b, residual=r, out_dtype=out)
            if rows:
                check_forward(x, w, b, r, 1e-5, out, got)
            else:
                assert got[0].shape == (0, dim)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", DIMS)
def test_backward(dim, dtype):
    for rows in (0, 1, 5, 130):
        for weight, dsum in ((None, None), (F32, 1), (dtype, None)):
            x = rand(rows, dim, dtype=dtype, seed=rows + dim, shift=0.5)
            dy = rand(rows, dim, dtype=dtype, seed=11)
            w = None if weight is None else (1 + rand(dim, seed=7, scale=0.2)).to(weight)
            ds = rand(rows, dim, dtype=dtype, seed=5) if dsum else None
            dx, dw, db = hg.layer_norm_grad(dy, x, w, dsum=ds, want_dweight=True)
            assert dx.dtype == dtype and dw.dtype == F32 and db.dtype == F32
            if rows == 0:
                assert dx.shape == (0, dim) and not dw.any() and not db.any()
                continue
            want, size, terms, terms_off = Ref(x, None, 1e-5).backward(dy, w)
            if ds is not None:
                want = want + ds.double()
                size = size + E * (want.abs() + ds.double().abs())
            R.assert_close(dx, want, R.rounding(want, dtype) + size, "dx")
            many = (rows + 8) * 2 * E
            R.assert_close(dw, terms.sum(0), terms_off.sum(0) + terms.abs().sum(0) * many + 1e-30,
                           "dweight")
            R.assert_close(db, dy.double().sum(0), dy.double().abs().sum(0) * many + 1e-30, "dbias")
            # each by itself is the same
            for k in range(3):
                only = hg.layer_norm_grad(dy, x, w, dsum=ds, want_dx=k == 0, want_dweight=k == 1,
                                          want_dbias=k == 2)
                for j, v in enumerate((dx, dw, db)):
                    assert (only[j] is None) if j != k else torch.equal(only[j], v)


def test_gradient_by_differences():
    rows, dim, eps = 3, 37, 1e-5
    x, w = rand(rows, dim, seed=1, shift=2.0), 1 + rand(dim, seed=2, scale=0.2)
    b, dy, ds = rand(dim, seed=6), rand(rows, dim, seed=3), rand(rows, dim, seed=4)

    def value(x64, w64, b64):
        y = Ref(x64, None, eps).forward(w64, b64)[0]
        return (y * dy.double()).sum() + (x64 * ds.double()).sum()

    dx, dw, db = hg.layer_norm_grad(dy, x, w, dsum=ds, eps=eps)
    step, args = 1e-5, (x.double(), w.double(), b.double())
    for k, got, places in ((0, dx, ((0, 0), (1, 5), (2, 36), (1, 20))), (1, dw, ((0,), (17,), (36,))),
                           (2, db, ((0,), (17,), (36,)))):
        for at in places:
            d = torch.zeros_like(args[k])
            d[at] = step
            up, down = (value(*(a + sign * d if j == k else a for j, a in enumerate(args)))
                        for sign in (1, -1))
            num = float(up - down) / (2 * step)
            assert abs(num - float(got[at])) <= 1e-5 * (1 + abs(num))


@pytest.mark.parametrize("dtype,dim", [(F32, 128), (F32, 30), (BF16, 100), (F16, 3000), (BF16, 9000)])
def test_rows_by_id(dtype, dim):
    table = rand(50, dim, dtype=dtype, seed=1)
    ids = torch.tensor([3, 49, 0, 3, 17], device="cuda")
    r = rand(5, dim, dtype=dtype, seed=2)
    for residual in (None, r):
        for out in (dtype, E4M3, I8):
            check_forward(table[ids], None, None, residual, 1e-5, out,
                          hg.layer_norm(table, residual=residual, ids=ids, out_dtype=out))
    dy = rand(5, dim, dtype=dtype, seed=4)
    by_id = hg.layer_norm_grad(dy, table, ids=ids, want_dweight=True)
    plain = hg.layer_norm_grad(dy, table[ids], want_dweight=True)
    assert all(torch.equal(a, b) for a, b in zip(by_id, plain))
    # ids out of range: broken rows, the others as they are
    wild = torch.tensor([3, 50, -1, 17, 1 << 40], device="cuda")
    good, bad = [0, 3], [1, 2, 4]
    y = hg.layer_norm(table, ids=wild)[0]
    assert torch.equal(y[good], hg.layer_norm(table[[3, 17]])[0])
    assert torch.isnan(y[bad].float()).all()
    for out in (E4M3, I8):
        q, _, sc = hg.layer_norm(table, ids=wild, out_dtype=out)
        w, _, wsc = hg.layer_norm(table[[3, 17]], out_dtype=out)
        assert torch.equal(q[good].view(torch.uint8), w.view(torch.uint8))
        assert torch.equal(sc[good], wsc) and torch.isnan(sc[bad]).all()
        assert (q[bad] == 0).all() if out == I8 else torch.isnan(q[bad].float()).all()


@pytest.mark.parametrize("dim", [64, 1000, 2048, 9000])
def test_rows_that_break(dim):
    """A NaN or an infinity in a row is that row's alone; zeros and equal elements are rows too."""
    x = rand(7, dim, seed=1)
    x[1, dim // 2] = float("nan")
    x[2, dim - 1] = float("inf")
    x[3, 0] = -float("inf")
    x[4] = 0
    x[5] = 3.0
    b = rand(dim, seed=2)
    y, _, _ = hg.layer_norm(x, bias=b)
    assert torch.isnan(y[1:4]).all() and torch.equal(y[4:6], b.expand(2, dim))
    rest = hg.layer_norm(x[[0, 6]], bias=b)[0]
    assert torch.equal(y[[0, 6]], rest)
    q, _, sc = hg.layer_norm(x, bias=b, out_dtype=I8)
    assert torch.isnan(sc[1:4]).all() and not q[1:4].any() and not torch.isnan(sc[4:]).any()
    q, _, sc = hg.layer_norm(x, out_dtype=I8)  # nothing but zeros has the least scale
    assert (sc[4:6] == 2.0 ** -126).all() and not q[4:6].any()
    q, _, sc = hg.layer_norm(x, bias=b, out_dtype=E4M3)
    assert torch.isnan(sc[1:4]).all() and torch.isnan(q[1:4].float()).all()
    # with eps 0, equal elements have no variance to divide by
    assert torch.isnan(hg.layer_norm(x[5:6], eps=0.0)[0]).all()


@pytest.mark.parametrize("dtype,dim", [(F32, 256), (F32, 1000), (F32, 9000)])
def test_rows_far_from_zero(dtype, dim):
    """A mean 1000 times the spread: the squares are summed around the mean."""
    x = rand(16, dim, dtype=dtype, seed=3, shift=1000.0)
    y = hg.layer_norm(x)[0].double()
    want = Ref(x, None, 1e-5).forward(None, None)[0]
    # by x^2's sum alone the variance of 1 would be lost in 1e6 (2^-24 of which is 0.06); here
    # the mean is off by some 2^-24 x 1000 a level of the sum's tree (12 levels), 7e-4
    assert float((y - want).abs().max()) <= 2e-3


def test_strides_and_copies():
    big = rand(40, 700, dtype=BF16, seed=1)
    x, r = big[:, 3:303], big[:, 350:650]
    check_forward(x, None, None, r, 1e-5, BF16, hg.layer_norm(x, residual=r))
    row = big[:1, :300].expand(40, 300)  # one row for all: stride 0
    check_forward(x, None, None, row, 1e-5, BF16, hg.layer_norm(x, residual=row))
    t = rand(300, 40, dtype=F32, seed=2).t()  # columns that are not contiguous: copied
    check_forward(t, None, None, None, 1e-5, F32, hg.layer_norm(t))
    dy = big[:, 11:311]
    for a, b in zip(hg.layer_norm_grad(dy, x, dsum=r, want_dweight=True),
                    hg.layer_norm_grad(dy.contiguous(), x.contiguous(), dsum=r.contiguous(),
                                       want_dweight=True)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dim", [40, 1024, 3000, 9000])
def test_in_place(dim):
    """sum over x, y over residual; dx over dy: what the header allows."""
    rows = 33
    x, r = rand(rows, dim, dtype=BF16, seed=1), rand(rows, dim, dtype=BF16, seed=2)
    want = hg.layer_norm(x, residual=r)
    a, b = x.clone(), r.clone()
    args = dense.LayerNormArgs(rows=rows, dim=dim, dtype=3, out_dtype=3, eps=1e-5, x=a.data_ptr(),
                               x_stride=dim, residual=b.data_ptr(), residual_stride=dim,
                               y=b.data_ptr(), y_stride=dim, sum=a.data_ptr(), sum_stride=dim)
    stream = torch.cuda.current_stream().cuda_stream
    assert hg.load_library().hg_layer_norm(ctypes.byref(args), stream) == 0
    assert torch.equal(b, want[0]) and torch.equal(a, want[1])
    dy = rand(rows, dim, dtype=BF16, seed=3)
    want = hg.layer_norm_grad(dy, x, want_dbias=False)[0]
    args = dense.LayerNormGradArgs(rows=rows, dim=dim, dtype=3, eps=1e-5, x=x.data_ptr(),
                                   x_stride=dim, dy=dy.data_ptr(), dy_stride=dim,
                                   dx=dy.data_ptr(), dx_stride=dim)
    assert hg.load_library().hg_layer_norm_grad(ctypes.byref(args), stream) == 0
    assert torch.equal(dy, want)


def test_many_rows_repeat_and_stream():
    """More rows than the blocks walk over at once; the same bits again, and on another stream."""
    for dim, dtype in ((64, F32), (1024, BF16)):
        x, dy = rand(20_011, dim, dtype=dtype, seed=1), rand(20_011, dim, dtype=dtype, seed=2)
        w = 1 + rand(dim, seed=3, scale=0.1)
        check_forward(x, w, None, None, 1e-5, dtype, hg.layer_norm(x, w))
        first = hg.layer_norm_grad(dy, x, w)
        terms, off = Ref(x, None, 1e-5).backward(dy, w)[2:]
        # (each of up to 1024 parts sums 20 rows by itself; the tree adds 42 levels at most)
        R.assert_close(first[1], terms.sum(0), off.sum(0) + terms.abs().sum(0) * 160 * E, "dweight")
        other = torch.cuda.Stream()
        torch.cuda.synchronize()
        for again in (hg.layer_norm_grad(dy, x, w), hg.layer_norm_grad(dy, x, w, stream=other)):
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_capture():
    x, r = rand(300, 512, dtype=BF16, seed=1), rand(300, 512, dtype=BF16, seed=2)
    dy, w, b = rand(300, 512, dtype=BF16, seed=3), 1 + rand(512, seed=4), rand(512, seed=5)

    def work():
        q, h, sc = hg.layer_norm(x, w, b, residual=r, out_dtype=I8)
        return (q, h, sc, *hg.layer_norm_grad(dy, h, w))

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for seed in (11, 12, 13):
        x.copy_(rand(300, 512, dtype=BF16, seed=seed))
        want = work()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("dtype,dim", [(F32, 64), (F32, 1000), (F32, 9000), (BF16, 40), (BF16, 2048),
                                       (BF16, 20_001)])
def test_squares_past_the_range(dtype, dim):
    """A finite row whose squares (or their sum) pass float32's range is NaN, whatever the bias and the
    result's type, and so is what its gradient reaches; the other rows are as they are by themselves."""
    x, r, dy = (rand(7, dim, dtype=dtype, seed=s) for s in (1, 2, 3))
    x[1] = 1e20
    x[1, ::2] = -1e20
    x[2] *= 3e19
    x[4, dim // 3] = 2e19  # (one square alone)
    x[6] *= 1e15           # (squares that stay in it)
    bad, good = [1, 2, 4], [0, 3, 5, 6]
    w, b = 1 + rand(dim, seed=4, scale=0.1), rand(dim, seed=5)
    for residual in (None, r):
        part = None if residual is None else r[good]
        for out in (dtype, E4M3, I8):
            y, total, scale = hg.layer_norm(x, w, b, residual=residual, out_dtype=out)
            want = hg.layer_norm(x[good], w, b, residual=part, out_dtype=out)
            check_forward(x[good], w, b, part, 1e-5, out, want)
            assert torch.equal(y[good].float(), want[0].float())
            if out == I8:
                assert not y[bad].any()
            else:
                assert torch.isnan(y[bad].float()).all()
            if out != dtype:
                assert torch.isnan(scale[bad]).all() and torch.equal(scale[good], want[2])
            if residual is not None:
                assert torch.isfinite(total.float()).all()
    for ds in (None, r):
        dx, dw, db = hg.layer_norm_grad(dy, x, w, dsum=ds)
        want = hg.layer_norm_grad(dy[good], x[good], w, dsum=None if ds is None else ds[good])
        assert torch.isnan(dx[bad].float()).all() and torch.equal(dx[good], want[0])
        assert torch.isnan(dw).all() and torch.isfinite(db).all()


@pytest.mark.parametrize("dim", [32, 250, 1000, 2048, 9000])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -95, 2.0 ** -112, 2.0 ** -119, 2.0 ** 120])
def test_8_bits_are_the_quotients(dim, size):
    """The integer (or e4m3 value) is that of y / scale as float32 rounds it: bit for bit what quantize
    makes of the same rows.  (53 bits round to 24 as the quotient itself does: 53 >= 2 x 24 + 2.)"""
    rows = (1 << 21) // dim
    x = rand(rows, dim, seed=dim, shift=0.3)
    w, b = (1 + rand(dim, seed=1, scale=0.2)) * size, rand(dim, seed=2, scale=0.3) * size
    y = hg.layer_norm(x, w, b)[0]
    q, _, c = hg.layer_norm(x, w, b, out_dtype=I8)
    want, wc = hg.quantize(y)
    assert torch.equal(c, wc)
    assert torch.equal(q, want), f"{int((q != want).sum())} of {q.numel()} integers"
    q, _, c = hg.layer_norm(x, w, b, out_dtype=E4M3)
    assert torch.equal(c, (y.abs().amax(1).double() / 448).float().clamp(min=2.0 ** -126))
    want = (y.double() / c.double()[:, None]).float().to(E4M3)
    off = q.view(torch.uint8) != want.view(torch.uint8)
    assert not off.any(), f"{int(off.sum())} of {q.numel()} values"
