"""The dense operators where their kernels change hands or values leave the ordinary: more rows than a
grid has groups, rows on both sides of the few-rows kernel and of whole rounds of tiles, float32
values at the ends of their range (whose products run on 16-bit pieces), workspaces of exactly the
size asked for, and two streams at once."""
import ctypes

import pytest
import torch

import dense_ref as R
import paper_2112_15345_amd as hg
from paper_2112_15345_amd import dense

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn


def rand(*shape, dtype=F32, seed=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def product(x, w, y, dtype):
    """y against x w^T: a sum of k terms held to k 2^-23 of their sizes, then one rounding."""
    z = x.double() @ w.double().t()
    size = (x.double().abs() @ w.double().abs().t()) * ((2 * x.shape[1] + 8) * R.E)
    R.assert_close(y, z, R.rounding(z, dtype) + size, "y")


@pytest.mark.parametrize("classes", [3, 2100])
def test_distill_of_more_rows_than_a_grid(classes):
    """(65536 blocks of 4 rows, or of 1.)"""
    rows = 300_000 if classes < 512 else 70_000
    z = rand(rows, classes, dtype=BF16, seed=1)
    ids, t = torch.randint(classes, (rows, 2), device="cuda"), rand(rows, 2, seed=2)
    loss, grad = hg.distill(z, ids, t, want_grad=True)
    alone = hg.distill(z, ids, t)[0]
    want, wgrad, size, _, _ = R.distill(z, ids, t, 1.0, None)
    bound = (size + 1) * (2 * classes + 128) * R.E
    R.assert_close(loss, want, bound, "loss")
    R.assert_close(alone, want, bound, "loss alone")
    R.assert_close(grad[-1000:], wgrad[-1000:], R.rounding(wgrad[-1000:], BF16)
                   + (2 * classes + 256) * R.E, "grad")


def test_norm_of_more_long_rows_than_a_grid():
    rows, dim = 65_600, 8_200
    x = rand(64, dim, dtype=BF16, seed=1)
    ids = torch.arange(rows, device="cuda") % 64
    y, _, _ = hg.rms_norm(x, ids=ids)
    want = hg.rms_norm(x)[0]
    assert torch.equal(y[-64:], want) and torch.equal(y[:64], want)
    assert torch.equal(y[65_536 - 64:65_536], want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m", [31, 32, 33, 255, 256, 257, 16_384, 16_385, 16_640])
def test_rows_at_the_borders(m, dtype):
    """Rows about the few-rows kernel's limit, a tile's height, and whole rounds of tiles; the
    same rows in any of them stay within the bounds, and the last row is there."""
    k, n = 520, 1032
    x, w = rand(m, k, dtype=dtype, seed=1), rand(n, k, dtype=dtype, seed=2, scale=k ** -0.5)
    y = hg.linear(x, w)[0]
    at = torch.tensor([0, m // 2, m - 2, m - 1], device="cuda")
    product(x[at], w, y[at], dtype)
    dy = rand(m, n, dtype=dtype, seed=3)
    dx = hg.linear_grad(dy, x, w, want_dw=False, want_dbias=False)[0]
    product(dy[at], w.t().contiguous(), dx[at], dtype)


@pytest.mark.parametrize("m", [300, 5000])
def test_float32_ends_of_the_range(m):
    """Values that round past the largest bfloat16, and small ones down to 2^-100."""
    k, n = 72, 136
    x, w = rand(m, k, seed=1), rand(n, k, seed=2, scale=1e-3)
    x[0, 3] = 3.4028e38
    x[1, 4] = -3.4028e38
    w[5, 7] = 0.0
    y = hg.linear(x, w)[0]
    product(x, w, y, F32)
    tiny = rand(m, k, seed=3, scale=2.0 ** -98)
    tiny = torch.where(tiny.abs() < 2.0 ** -100, 2.0 ** -100, tiny)
    y = hg.linear(tiny, rand(n, k, seed=4))[0]
    product(tiny, rand(n, k, seed=4), y, F32)


def test_float32_infinities_backward():
    """Infinities in dz, w and x, through both products of the backward pass."""
    m, k, n = 400, 136, 264
    x, w, dy = rand(m, k, seed=1), rand(n, k, seed=2), rand(m, n, seed=3)
    clean = hg.linear_grad(dy, x, w)
    x[:, 0] = 1.0
    clean = hg.linear_grad(dy, x, w)
    dy[7, 9] = float("inf")
    dx, dw, db = hg.linear_grad(dy, x, w)
    assert torch.isinf(dx[7]).all() and torch.equal(dx[7] > 0, w[9] > 0)
    rows = torch.arange(m) != 7
    assert torch.equal(dx[rows], clean[0][rows])
    assert torch.isinf(dw[9]).all() and torch.equal(dw[9] > 0, x[7] > 0)
    cols = torch.arange(n) != 9
    assert torch.equal(dw[cols], clean[1][cols])
    assert torch.isinf(db[9]) and torch.equal(db[cols], clean[2][cols])


def test_workspaces_of_the_size_asked_for():
    """Calls with workspaces whose neighbours are watched: nothing is written past the end."""
    lib = hg.load_library()
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    for m, k, n, act in ((300, 4096, 136, 0), (8, 70_000, 24, 0), (5000, 264, 520, 2),
                         (16_385, 520, 1032, 0)):
        x, w = rand(m, k, dtype=BF16, seed=1), rand(n, k, dtype=BF16, seed=2)
        dy, y = rand(m, n, dtype=BF16, seed=3), torch.empty(m, n, dtype=BF16, device="cuda")
        need = lib.hg_linear_workspace(m, k, n, dense.HG_DT_BF16)
        ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
        a = dense.LinearArgs(m, k, n, 3, 3, 0, act, x.data_ptr(), k, None, w.data_ptr(), k, None,
                             None, None, 0, y.data_ptr(), n, None, 0, ws.data_ptr(), need)
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
    rows, dim = 700, 520
    x, dy = rand(rows, dim, seed=1), rand(rows, dim, seed=2)
    need = lib.hg_rms_norm_grad_workspace(rows, dim)
    ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty(dim, device="cuda")
    g = dense.NormGradArgs(rows, dim, 1, 0, 1e-6, x.data_ptr(), dim, rows, None, None,
                           dy.data_ptr(), dim, None, 0, dx.data_ptr(), dim, dw.data_ptr(),
                           ws.data_ptr(), need)
    assert lib.hg_rms_norm_grad(ctypes.byref(g), stream) == hg.HG_OK
    assert (ws[need:] == 0x5a).all()


def test_two_streams_at_once():
    """The same operators on two streams, again and again: each call has its own workspace."""
    args = []
    for seed in (1, 2):
        x, w = rand(400, 4096, dtype=BF16, seed=seed), rand(136, 4096, dtype=BF16, seed=seed + 2)
        z = rand(64, 5000, dtype=BF16, seed=seed + 4)
        args.append((x, w, z, torch.randint(5000, (64, 9), device="cuda"), rand(64, 9, seed=6)))

    def calls(x, w, z, ids, t, stream=None):
        return (hg.linear(x, w, stream=stream)[0],
                *hg.rms_norm_grad(x, x, want_dweight=True, stream=stream),
                *hg.distill(z, ids, t, want_grad=True, stream=stream))

    want = [calls(*a) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(5):
        for i in (0, 1):
            got[i].append(calls(*args[i], stream=streams[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[i]))
