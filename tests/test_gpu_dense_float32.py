"""float32 products on 128 x 128 tiles, whose elements are multiplied as three 16-bit pieces: products
past the largest float32 and just below it, elements that round past the largest bfloat16, and
depths so short that a product without the third pieces would not stay within the bound.

(More than 128 tiles of 128 x 128, or a depth of at least 32 slabs of 32 for half of them, are not
made of 64 x 64 tiles, which use the 32-bit instructions.)"""
import pytest
import torch

import dense_ref as R
import paper_2112_15345_amd as hg

pytestmark = pytest.mark.gpu

F32 = torch.float32
TWO64 = 2.0 ** 64 - 2.0 ** 40  # the largest float32 below 2^64; its square is 2^128 - 2^105, finite
BIG, FACTOR = 1.0037e30, 1.0037e12  # (their pieces' products overflow with either sign)


def rand(*shape, seed=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda") * scale


def signs(n):
    return 1.0 - 2.0 * (torch.arange(n, device="cuda") % 2)


def check(got, a, b, what):
    """got against a b^T: a sum of k terms held to k 2^-23 of their sizes; past the largest float32
    it is an infinity."""
    want = a.double() @ b.double().t()
    size = (a.double().abs() @ b.double().abs().t()) * ((2 * a.shape[1] + 8) * R.E)
    want = want.float().double()
    size = torch.nan_to_num(size, posinf=0.0) + R.rounding(torch.nan_to_num(want, posinf=0.0, neginf=0.0), F32)
    R.assert_close(got, want, size, what)


def test_forward_overflow():
    m, k, n = 2100, 72, 1032
    x, w = rand(m, k, seed=1), rand(n, k, seed=2)
    w[:, 5] = FACTOR * signs(n)
    w[4, 5] = 7e12
    w[11], w[11, 6] = 0.0, TWO64
    base = hg.linear(torch.where(torch.arange(m, device="cuda")[:, None] < 32, 0.0, x), w)[0]
    x[3, 5], x[8, 5] = BIG, 3e37
    x[9], x[9, 6] = 0.0, TWO64
    y = hg.linear(x, w)[0]
    check(y, x, w, "y")
    assert torch.isinf(y[3, :11]).all() and torch.isinf(y[8, :11]).all()
    assert float(y[9, 11]) == 2.0 ** 128 - 2.0 ** 105
    # the other rows are what they are without these; the same rows in a call of few
    assert torch.equal(y[32:], base[32:])
    few = hg.linear(x[:32], w)[0]
    assert torch.equal(torch.isinf(few), torch.isinf(y[:32])) and not torch.isnan(few).any()
    cut = hg.linear(x, w, act="relu")[0]
    assert not cut[y == -float("inf")].any() and (cut[y == float("inf")] == float("inf")).all()


def test_forward_past_bfloat16():
    """Elements that a bfloat16 would round to an infinity, and infinities and NaN beside them."""
    m, k, n = 2100, 72, 1032
    x, w = rand(m, k, seed=1), rand(n, k, seed=2, scale=1e-3)
    x[0, 3], x[1, 4] = 3.4028e38, -3.4028e38
    w[5, 7] = 0.0
    check(hg.linear(x, w)[0], x, w, "y")
    clean = hg.linear(x, w)[0]
    x[130, 7], x[131, 7], x[132, 9] = float("inf"), -float("inf"), float("nan")
    y = hg.linear(x, w)[0]
    check(y, x, w, "y")
    rows = (torch.arange(m) < 130) | (torch.arange(m) > 132)
    assert torch.equal(y[rows], clean[rows]) and torch.isnan(y[130:133, 5]).all()


def test_backward_overflow():
    m, k, n = 2100, 1100, 1032
    x, w, dy = rand(m, k, seed=1), rand(n, k, seed=2), rand(m, n, seed=3)
    x[3], w[5] = FACTOR * signs(k), -FACTOR * signs(k)
    dy[3, 5] = BIG
    dy[40], dy[:, 40] = 0.0, 0.0
    dy[40, 40] = TWO64
    w[40, :7], x[40, :7] = TWO64, -TWO64
    dx, dw, db = hg.linear_grad(dy, x, w)
    check(dx, dy, w.t().contiguous(), "dx")
    check(dw, dy.t().contiguous(), x.t().contiguous(), "dw")
    assert torch.isinf(dx[3]).all() and torch.isinf(dw[5]).all()
    assert (dx[40, :7] == 2.0 ** 128 - 2.0 ** 105).all()
    assert (dw[40, :7] == -(2.0 ** 128 - 2.0 ** 105)).all()


def test_short_depths():
    """At a depth of 8 the bound is 24 units of 2^-24 of the terms' sizes; without the third pieces
    a product is off by up to 2^-15 of its own size."""
    x, w = rand(20_000, 8, seed=1), rand(520, 8, seed=2)
    check(hg.linear(x, w)[0], x, w, "y")
    dy, w = rand(20_000, 8, seed=3), rand(8, 520, seed=4)
    x = rand(20_000, 520, seed=5)
    check(hg.linear_grad(dy, x, w, want_dw=False, want_dbias=False)[0], dy, w.t().contiguous(), "dx")
    dy, x, w = rand(8, 2100, seed=6), rand(8, 1100, seed=7), rand(2100, 1100, seed=8)
    check(hg.linear_grad(dy, x, w, want_dx=False, want_dbias=False)[1], dy.t().contiguous(),
          x.t().contiguous(), "dw")
