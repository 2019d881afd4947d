"""quantize, dequantize, and linear_grad from kept rows.  The integers are the definition's bit for bit:
in float32, the quotients by division, on the CPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

import dense_ref as R
import paper_2112_15345_amd as hg
from paper_2112_15345_amd import dense
from test_gpu_dense_linear import ACTS, rand

pytestmark = pytest.mark.gpu

F32, F16, BF16, I8 = torch.float32, torch.float16, torch.bfloat16, torch.int8
GROUP = hg.HG_KEPT_GROUP
DIMS = [1, 2, 3, 16, 33, 64, 100, 127, 128, 129, 250, 512, 1000, 1024, 1999, 2048, 4095, 8192, 8200,
        20_001]


def define(x, group):
    """q and scale of rows in numpy's float32."""
    x = x.float().cpu().numpy()
    rows, dim = x.shape
    width = group or dim
    q, scale = np.zeros((rows, dim), np.int8), np.zeros((rows, -(-dim // width)), np.float32)
    for g in range(scale.shape[1]):
        part = x[:, g * width:(g + 1) * width]
        top = np.abs(part).max(1)
        c = top * (np.float32(1) / np.float32(127))
        c = np.maximum(c, np.float32(2.0 ** -126)).astype(np.float32)
        c[~np.isfinite(top)] = np.nan
        fine = np.isfinite(c)
        q[fine, g * width:(g + 1) * width] = np.rint(part[fine] / c[fine, None]).astype(np.int8)
        scale[:, g] = c
    return q, scale if group else scale[:, 0]


def check(x, group, got):
    q, scale = got
    assert q.dtype == I8 and scale.dtype == F32 and q.shape == x.shape
    want_q, want_scale = define(x, group)
    assert np.array_equal(scale.cpu().numpy(), want_scale, equal_nan=True)
    assert np.array_equal(q.cpu().numpy(), want_q)


@pytest.mark.parametrize("group", [0, GROUP])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", DIMS)
def test_quantize(dim, dtype, group):
    for rows in (0, 1, 5, 67):
        x = rand(rows, dim, dtype=dtype, seed=rows + dim, scale=3.0)
        got = hg.quantize(x, group=group)
        if rows == 0:
            assert got[0].shape == (0, dim) and got[1].shape[0] == 0
            continue
        check(x, group, got)
        for out in (F32, F16, BF16):
            back = hg.dequantize(*got, group=group, out_dtype=out)
            c = got[1].repeat_interleave(GROUP, 1)[:, :dim] if group else got[1][:, None]
            # one rounding to the type, or one to float32 before it
            want = got[0].double() * c.double()
            assert back.dtype == out
            R.assert_close(back, want, R.rounding(want, out) + R.E * want.abs(), "back")


def test_many_rows():
    x = rand(40_003, 300, dtype=BF16, seed=1)
    for group in (0, GROUP):
        check(x, group, hg.quantize(x, group=group))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_middles(dtype):
    """Quotients that lie between two integers, exactly and next to it: to the even one."""
    step = (torch.arange(-254, 255, device="cuda") / 2.0)
    for scale in (1.0, 0.125, 2.0 ** -10):
        check((step * scale)[None].to(dtype), 0, hg.quantize((step * scale)[None].to(dtype)))
    # scales that are no powers of two, elements as near to the middles as float32 has them
    for top in (1.0, 3.7, 100.1, 5e-30, 1e30):
        c = torch.tensor(top, dtype=F32) * (torch.ones(()) / 127)
        mid = (torch.arange(-126, 126, dtype=F32) + 0.5) * c
        row = torch.cat([torch.tensor([top]), mid, torch.nextafter(mid, mid + 1e38),
                         torch.nextafter(mid, mid - 1e38)])[None].cuda()
        check(row, 0, hg.quantize(row))


@pytest.mark.parametrize("group", [0, GROUP])
@pytest.mark.parametrize("dim", [40, 300, 9000])
def test_rows_at_the_ends(dim, group):
    x = rand(9, dim, seed=1)
    x[1] = 0
    x[2] *= 1e-39  # below the smallest normal number
    x[3] *= 1e37
    x[4, 5] = math.nan
    x[5, dim - 1] = math.inf
    x[6, 0] = -math.inf
    x[7] = 3.4e38
    q, scale = hg.quantize(x, group=group)
    check(x, group, (q, scale))
    back = hg.dequantize(q, scale, group=group, out_dtype=F32)
    broken = torch.isnan(back)
    width = group or dim
    for row, col in ((4, 5), (5, dim - 1), (6, 0)):
        g = col // width
        assert broken[row, g * width:(g + 1) * width].all()
        broken[row, g * width:(g + 1) * width] = False
    assert not broken.any()


def test_strides_streams_and_capture():
    big = rand(50, 800, dtype=BF16, seed=1)
    for x in (big[:, 3:403], big[::2, :300], big[:1].expand(50, 800), big.t()):
        for group in (0, GROUP):
            check(x, group, hg.quantize(x, group=group))
    q, scale = hg.quantize(big, group=GROUP)
    part = hg.dequantize(q[:, 128:400], scale[:, 1:4], group=GROUP)
    assert torch.equal(part, hg.dequantize(q, scale, group=GROUP)[:, 128:400])
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    again = hg.quantize(big, group=GROUP, stream=other)
    torch.cuda.synchronize()
    assert torch.equal(q, again[0]) and torch.equal(scale, again[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = hg.quantize(big)
        back = hg.dequantize(*out)
    for seed in (3, 4, 5):
        big.copy_(rand(50, 800, dtype=BF16, seed=seed))
        graph.replay()
        torch.cuda.synchronize()
        check(big, 0, out)
        assert torch.equal(back, hg.dequantize(*out))


def test_offsets_past_32_bits():
    rows, dim = 2_200_003, 1024
    x = torch.zeros(rows, dim, dtype=BF16, device="cuda")
    x[-2:] = rand(2, dim, dtype=BF16, seed=1)
    for group in (0, GROUP):
        q, scale = hg.quantize(x, group=group)
        check(x[-3:], group, (q[-3:], scale[-3:]))
        assert torch.equal(hg.dequantize(q, scale, group=group)[-3:],
                           hg.dequantize(q[-3:], scale[-3:], group=group))


def stands_for(q, scale, group):
    c = scale.double().repeat_interleave(GROUP, 1)[:, :q.shape[1]] if group else \
        scale.double()[:, None]
    return q.double() * c


SIZES = [(1, 1, 1), (1, 64, 128), (3, 100, 47), (17, 33, 65), (33, 130, 129), (64, 768, 64),
         (65, 1000, 100), (129, 64, 257), (257, 4099, 130), (513, 200, 511), (5000, 136, 260)]


def check_grad(dy, x, w, pre, act, got, x_off, dw_dtype):
    """As in linear_grad: dz in 32 bits is rounded to the type before the products; x (in double, as
    the integers stand for it) is rounded to the type before its one."""
    dx, dw, db = got
    dtype = w.dtype
    dy = dy.double()
    slope = torch.ones_like(dy) if act == "none" else R.act_slope(pre, act)
    if act == "relu":  # (its slope at 0 is 0, and integers are often 0)
        slope = torch.where(pre == 0, 0.0, slope)
    dz = dy * slope
    dz_size = torch.zeros_like(dz) if act == "none" else dy.abs() * 32 * R.E * (1 + pre.abs())
    dz_off = dz_size + (R.rounding(dz, dtype) if act != "none" else 0)
    terms = dz.abs() @ w.double().abs()
    want = dz @ w.double()
    R.assert_close(dx, want, R.rounding(want, dtype) + 1.01 * (dz_off @ w.double().abs())
                   + terms * (2 * dy.shape[1] + 8) * R.E, "dx")
    terms = dz.abs().t() @ x.abs()
    want = dz.t() @ x
    off = dz_off.t() @ x.abs() + (dz.abs() + dz_off).t() @ x_off
    assert dw.dtype == (dw_dtype or dtype)
    R.assert_close(dw, want, R.rounding(want, dw.dtype) + 1.01 * off
                   + terms * (2 * dy.shape[0] + 8) * R.E, "dw")
    R.assert_close(db, dz.sum(0), dz_size.sum(0) + dz.abs().sum(0) * (2 * dy.shape[0] + 8) * R.E
                   + 1e-37, "dbias")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_backward(m, k, n, dtype):
    for i, act in enumerate(ACTS):
        group = (0, GROUP)[i % 2]
        w = rand(n, k, dtype=dtype, seed=2, scale=k ** -0.5)
        dy = rand(m, n, dtype=dtype, seed=3)
        x, xs = hg.quantize(rand(m, k, seed=1), group=group)
        kw = dict(act=act, dw_dtype=F32 if i < 2 else None, x_scale=xs, group=group)
        pre64 = None
        if act != "none":
            kw["pre"], kw["pre_scale"] = hg.quantize(rand(m, n, seed=4, scale=2.0), group=group)
            pre64 = stands_for(kw["pre"], kw["pre_scale"], group)
        x64 = stands_for(x, xs, group)
        x_off = R.rounding(x64, dtype) + R.E * x64.abs()
        got = hg.linear_grad(dy, x, w, **kw)
        check_grad(dy, x64, w, pre64, act, got, x_off, kw["dw_dtype"])
        for j, want in enumerate(("want_dx", "want_dw", "want_dbias")):
            only = hg.linear_grad(dy, x, w, **kw, **{f: f == want for f in ("want_dx", "want_dw",
                                                                            "want_dbias")})
            assert torch.equal(only[j], got[j]) and sum(t is None for t in only) == 2


@pytest.mark.parametrize("m,k,n", [(300, 256, 136), (2100, 1024, 512), (16_400, 128, 256)])
def test_one_of_the_two_kept(m, k, n):
    """x alone or pre alone: bit for bit what linear_grad gives for the rows that they stand for."""
    dy, w = rand(m, n, dtype=F32, seed=1), rand(n, k, seed=2)
    x, pre = rand(m, k, seed=3), rand(m, n, seed=4)
    for group in (0, GROUP):
        x8, pre8 = hg.quantize(x, group=group), hg.quantize(pre, group=group)
        xd = hg.dequantize(*x8, group=group, out_dtype=F32)
        pred = hg.dequantize(*pre8, group=group, out_dtype=F32)
        for got, want in (
                (hg.linear_grad(dy, x8[0], w, pre=pre, act="gelu", x_scale=x8[1], group=group),
                 hg.linear_grad(dy, xd, w, pre=pre, act="gelu")),
                (hg.linear_grad(dy, x, w, pre=pre8[0], act="silu", pre_scale=pre8[1], group=group),
                 hg.linear_grad(dy, x, w, pre=pred, act="silu")),
                (hg.linear_grad(dy, x8[0], w, x_scale=x8[1], group=group),
                 hg.linear_grad(dy, xd, w))):
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_empty_and_strided():
    w, one = rand(6, 40, dtype=BF16), torch.ones(0, device="cuda")
    x = torch.zeros(0, 40, dtype=I8, device="cuda")
    dx, dw, db = hg.linear_grad(rand(0, 6, dtype=BF16), x, w, x_scale=one)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()
    x, xs = hg.quantize(rand(70, 300, seed=1))
    pre, ps = hg.quantize(rand(70, 300, seed=2))
    dy, w = rand(70, 140, dtype=BF16, seed=3), rand(140, 120, dtype=BF16, seed=4)
    got = hg.linear_grad(dy, x[:, 5:125], w, pre=pre[:, 7:147], act="silu", x_scale=xs, pre_scale=ps)
    want = hg.linear_grad(dy, x[:, 5:125].contiguous(), w, pre=pre[:, 7:147].contiguous(), act="silu",
                          x_scale=xs, pre_scale=ps)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_binding_refuses():
    x, xs = hg.quantize(rand(4, 8))
    g, gs = hg.quantize(rand(4, 8), group=GROUP)
    w, dy = rand(6, 8, dtype=BF16), rand(4, 6, dtype=BF16)
    for call in (lambda: hg.quantize(x), lambda: hg.quantize(rand(4, 8), group=64),
                 lambda: hg.dequantize(x, xs, group=GROUP), lambda: hg.dequantize(g, gs),
                 lambda: hg.dequantize(x, xs, out_dtype=I8), lambda: hg.dequantize(w, xs),
                 lambda: hg.linear_grad(dy, x, w), lambda: hg.linear_grad(dy, w[:4], w, x_scale=xs),
                 lambda: hg.linear_grad(dy, x, w, x_scale=xs, group=GROUP),
                 lambda: hg.linear_grad(dy, x, w, x_scale=xs[:3]),
                 lambda: hg.linear_grad(dy, x, w, x_scale=xs, act="gelu"),
                 lambda: hg.linear_grad(dy, x, w, x_scale=xs, pre_scale=xs),
                 lambda: hg.linear_grad(dy, x, w, x_scale=xs, act="gelu", pre=dy, pre_scale=xs)):
        with pytest.raises(ValueError):
            call()


def test_backward_in_a_graph():
    m, k, n = 300, 128, 256
    dy, w = rand(m, n, dtype=BF16, seed=1), rand(n, k, dtype=BF16, seed=2)
    x, pre = rand(m, k, dtype=BF16, seed=3), rand(m, n, dtype=BF16, seed=4)

    def work():
        x8, xs = hg.quantize(x, group=GROUP)
        pre8, ps = hg.quantize(pre, group=GROUP)
        return hg.linear_grad(dy, x8, w, pre=pre8, act="gelu", x_scale=xs, pre_scale=ps, group=GROUP)

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for seed in (5, 6, 7):
        x.copy_(rand(m, k, dtype=BF16, seed=seed))
        dy.copy_(rand(m, n, dtype=BF16, seed=seed + 10))
        want = work()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_workspace_is_what_the_call_needs():
    """Rows that stand for x are made where x is kept and dw is wanted, and nowhere else."""
    m, k, n = 4096, 4096, 128
    widened = m * k * 2
    dy, w = rand(m, n, dtype=BF16, seed=1), rand(n, k, dtype=BF16, seed=2)
    x, pre = rand(m, k, dtype=BF16, seed=3), rand(m, n, dtype=BF16, seed=4)
    x8, xs = hg.quantize(x, group=GROUP)
    pre8, ps = hg.quantize(pre, group=GROUP)

    def taken(**kw):
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        got = hg.linear_grad(dy, pre=pre8, act="gelu", pre_scale=ps, group=GROUP, w=w, **kw)
        peak = torch.cuda.max_memory_allocated() - before
        return peak - sum(t.numel() * t.element_size() for t in got if t is not None)

    both = taken(x=x8, x_scale=xs)
    assert widened <= both
    assert taken(x=x8, x_scale=xs, want_dw=False) <= both - widened
    assert taken(x=x) <= both - widened


def test_least_workspace_is_enough():
    """By the C entry point: hg_linear_grad_workspace's size where x is not kept, or dw not wanted."""
    m, k, n = 300, 250, 140
    lib = hg.load_library()
    dy, w = rand(m, n, dtype=BF16, seed=1), rand(n, k, dtype=BF16, seed=2)
    x, pre = rand(m, k, dtype=BF16, seed=3), rand(m, n, dtype=BF16, seed=4)
    x8, xs = hg.quantize(x)
    pre8, ps = hg.quantize(pre)
    need = lib.hg_linear_grad_workspace(m, k, n, 3, 2)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for kept in (True, False):
        rows = x8 if kept else x
        dx = torch.empty(m, k, dtype=BF16, device="cuda")
        dw = None if kept else torch.empty(n, k, dtype=BF16, device="cuda")
        db = torch.empty(n, device="cuda")
        grad = dense.LinearGradArgs(
            m=m, k=k, n=n, dtype=3, dw_dtype=3, act=2, dy=dy.data_ptr(), dy_stride=n,
            pre=pre8.data_ptr(), pre_stride=n, x=rows.data_ptr(), x_stride=k, w=w.data_ptr(), w_stride=k,
            dx=dx.data_ptr(), dx_stride=k, dw=None if kept else dw.data_ptr(), dw_stride=k,
            dbias=db.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=need)
        args = dense.LinearGradKeptArgs(grad, 0, xs.data_ptr() if kept else None, ps.data_ptr())
        stream = torch.cuda.current_stream().cuda_stream
        assert lib.hg_linear_grad_kept(ctypes.byref(args), stream) == hg.HG_OK
        want = hg.linear_grad(dy, rows, w, pre=pre8, act="gelu", x_scale=xs if kept else None,
                              pre_scale=ps, want_dw=not kept)
        assert torch.equal(dx, want[0]) and torch.equal(db, want[2])
        assert kept or torch.equal(dw, want[1])
