"""Products large enough that operands whose rows are not whole 16-byte pieces are copied into rows
that are, and products whose tiles fill half of the units and whose depth is cut."""
import ctypes

import pytest
import torch

import paper_2112_15345_amd as hg
from paper_2112_15345_amd import dense
from test_gpu_dense_linear import BF16, E4M3, F16, F32, check, check_grad, rand, to_8_bits

pytestmark = pytest.mark.gpu

# every one of m k n is at least 4e9: odd rows of x and w, of dz, of both, and odd heights
SIZES = [(2500, 1301, 1303), (2401, 1304, 1303), (2403, 1301, 1304), (251, 4097, 4001)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16, E4M3])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_forward(m, k, n, dtype):
    out = BF16 if dtype == E4M3 else dtype
    x, w = rand(m, k, seed=1), rand(n, k, seed=2, scale=k ** -0.5)
    kw = {}
    if dtype == E4M3:
        (x, xs), (w, ws) = to_8_bits(x), to_8_bits(w)
        kw = dict(x_scale=xs, w_scale=ws)
    else:
        x, w = x.to(dtype), w.to(dtype)
    bias, res = rand(n, seed=3), rand(m, n, dtype=out, seed=4)
    got = hg.linear(x, w, bias=bias, act="silu", residual=res, out_dtype=out, keep_pre=True, **kw)
    check(x, w, got, bias, "silu", res, kw.get("x_scale"), kw.get("w_scale"), out)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_backward(m, k, n, dtype):
    x, w = rand(m, k, dtype=dtype, seed=1), rand(n, k, dtype=dtype, seed=2, scale=k ** -0.5)
    dy = rand(m, n, dtype=dtype, seed=3)
    for act in ("none", "gelu"):
        pre = rand(m, n, dtype=dtype, seed=4, scale=2.0) if act != "none" else None
        got = hg.linear_grad(dy, x, w, pre=pre, act=act)
        check_grad(dy, x, w, pre, act, got)
        for keep in range(3):
            want = [j == keep for j in range(3)]
            some = hg.linear_grad(dy, x, w, pre=pre, act=act, want_dx=want[0], want_dw=want[1],
                                  want_dbias=want[2])
            assert all(torch.equal(some[j], got[j]) for j in range(3) if want[j])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_views(dtype):
    """Odd starts and strides, a broadcast row of gradients."""
    m, k, n = SIZES[0]
    x = rand(m, k + 6, dtype=dtype, seed=1)[:, 3:3 + k]
    w = rand(n, k + 3, dtype=dtype, seed=2, scale=k ** -0.5)[:, 1:1 + k]
    check(x, w, hg.linear(x, w))
    dy = rand(m, n + 3, dtype=dtype, seed=3)[:, 2:2 + n]
    check_grad(dy, x, w, None, "none", hg.linear_grad(dy, x, w))
    wide = rand(1, n, dtype=dtype, seed=4).expand(m, n)
    check_grad(wide, x, w, None, "none", hg.linear_grad(wide, x, w))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_values_that_are_not_finite(dtype):
    """They stay in their rows and columns: the zeros that rows end in meet no infinity."""
    m, k, n = SIZES[0]
    x, w = rand(m, k, dtype=dtype, seed=1), rand(n, k, dtype=dtype, seed=2, scale=0.1)
    dy = rand(m, n, dtype=dtype, seed=3)
    clean, grads = hg.linear(x, w)[0], hg.linear_grad(dy, x, w)
    x[5, k - 1], w[9, k - 1], dy[7, n - 1] = float("inf"), float("nan"), float("-inf")
    y, (dx, dw, db) = hg.linear(x, w)[0], hg.linear_grad(dy, x, w)
    rows, cols = torch.arange(m) != 5, torch.arange(n) != 9
    assert torch.equal(y[rows][:, cols], clean[rows][:, cols])
    assert torch.isinf(y[5, cols]).all() and torch.isnan(y[:, 9]).all()
    rows, cols = torch.arange(m) != 7, torch.arange(k) != k - 1
    assert torch.equal(dx[rows][:, cols], grads[0][rows][:, cols])
    assert torch.isinf(dx[7, cols]).all() and torch.isnan(dx[:, k - 1]).all()
    rows = torch.arange(n) != n - 1
    assert torch.equal(dw[rows][:, cols], grads[1][rows][:, cols])
    assert torch.isinf(dw[n - 1, cols]).all() and torch.isinf(dw[rows][:, k - 1]).all()
    assert torch.equal(db[rows], grads[2][rows]) and db[n - 1] == float("-inf")


def test_workspaces_of_the_size_asked_for():
    lib = hg.load_library()
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    for m, k, n in SIZES[:3]:
        for act in (0, 2):
            x, w = rand(m, k, dtype=BF16, seed=1), rand(n, k, dtype=BF16, seed=2)
            dy, y = rand(m, n, dtype=BF16, seed=3), torch.empty(m, n, dtype=BF16, device="cuda")
            need = lib.hg_linear_workspace(m, k, n, dense.HG_DT_BF16)
            ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
            a = dense.LinearArgs(m, k, n, 3, 3, 0, act, x.data_ptr(), k, None, w.data_ptr(), k,
                                 None, None, None, 0, y.data_ptr(), n, None, 0, ws.data_ptr(), need)
            assert lib.hg_linear(ctypes.byref(a), stream) == hg.HG_OK
            assert (ws[need:] == 0x5a).all()
            need = lib.hg_linear_grad_workspace(m, k, n, dense.HG_DT_BF16, act)
            ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
            dx, dw = torch.empty_like(x), torch.empty_like(w)
            db = torch.empty(n, device="cuda")
            g = dense.LinearGradArgs(m, k, n, 3, 3, act, dy.data_ptr(), n, y.data_ptr(), n,
                                     x.data_ptr(), k, w.data_ptr(), k, dx.data_ptr(), k,
                                     dw.data_ptr(), k, db.data_ptr(), ws.data_ptr(), need)
            assert lib.hg_linear_grad(ctypes.byref(g), stream) == hg.HG_OK
            assert (ws[need:] == 0x5a).all()


def test_capture():
    m, k, n = SIZES[0]
    x, w = rand(m, k, dtype=BF16, seed=1), rand(n, k, dtype=BF16, seed=2)
    dy = rand(m, n, dtype=BF16, seed=3)

    def calls():
        return (hg.linear(x, w)[0], *hg.linear_grad(dy, x, w))

    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    for seed in (4, 5):
        x.copy_(rand(m, k, dtype=BF16, seed=seed))
        graph.replay()
        want = calls()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,k,n", [(8200, 2000, 2700), (8201, 2001, 2701)])
def test_deep_products_of_few_rounds(m, k, n, dtype):
    """(352 tiles of 128 x 128, and 176 of 256 x 128, in the weight gradient.)"""
    x, w = rand(m, k, dtype=dtype, seed=1), rand(n, k, dtype=dtype, seed=2, scale=k ** -0.5)
    dy = rand(m, n, dtype=dtype, seed=3)
    got = hg.linear_grad(dy, x, w, want_dx=False, dw_dtype=F32)
    check_grad(dy, x, w, None, "none", got, F32)
    again = hg.linear_grad(dy, x, w, want_dx=False, dw_dtype=F32)
    assert torch.equal(got[1], again[1])
