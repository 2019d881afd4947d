"""Scales of 8-bit rows at the ends of float32's range: z = x_scale w_scale sum as long as it is a float32,
whatever the product of the two scales is."""
import pytest
import torch

import paper_2112_15345_amd as hg
from test_gpu_dense_linear import BF16, E4M3, F32, check, rand, to_8_bits

pytestmark = pytest.mark.gpu


# few rows, and few with their depth in parts; 64 x 64, 128 x 128 and 256 x 256 tiles; rows that are
# not whole 16-byte pieces
@pytest.mark.parametrize("m,k,n", [(9, 64, 300), (9, 8192, 40), (300, 96, 136), (2100, 64, 1032),
                                   (8200, 1024, 4104), (300, 97, 137)])
def test_scales_at_the_ends(m, k, n):
    x, w = to_8_bits(rand(m, k, seed=1))[0], to_8_bits(rand(n, k, seed=2))[0]
    x[5] = torch.full((k,), 2.0 ** -9, device="cuda").to(E4M3)
    x[6] = 0
    w[9] = torch.full((k,), 2.0 ** -9, device="cuda").to(E4M3)
    w[:, 1] = torch.tensor(2.0 ** -9).to(E4M3)
    xs = torch.full((m,), 2.0 ** -10, device="cuda")
    ws = torch.full((n,), 2.0 ** -12, device="cuda")
    xs[:8] = torch.tensor([2.0 ** -126, 1.7 * 2.0 ** -80, 2.0 ** 90, 1.0, 1e-45, 2.0 ** 70, 2.0 ** 100, 3e38])
    ws[:12] = torch.tensor([2.0 ** -126, 1.3 * 2.0 ** -60, 2.0 ** -100, 1.0, 2.0 ** 100, 2.0 ** 20, 1e-45,
                            3e38, 2.0 ** -30, 2.0 ** 60, 2.0 ** 126, 5.0])
    y = hg.linear(x, w, x_scale=xs, w_scale=ws, out_dtype=F32)[0]
    # what passes the largest float32 is an infinity; the rest is held to the bound
    a = x.double() * xs.double()[:, None]
    z = a @ (w.double() * ws.double()[:, None]).t()
    past = z.abs() > 3.4e38
    assert (torch.isinf(y) == past).all() and (y[past] > 0).equal(z[past] > 0)
    assert not y[6].any()
    assert torch.isfinite(y[5, 9]) and float(y[5, 9]) == k * 2.0 ** 112
    near = ~past.any(1)
    check(x[near], w, (y[near], None), xs=xs[near], ws=ws, out=F32)
    near = ~past.any(0)
    check(x, w[near], (y[:, near], None), xs=xs, ws=ws[near], out=F32)


def test_scales_that_are_not_finite():
    x, w = to_8_bits(rand(40, 64, seed=1))[0], to_8_bits(rand(50, 64, seed=2))[0]
    xs, ws = torch.ones(40, device="cuda"), torch.ones(50, device="cuda")
    clean = hg.linear(x, w, x_scale=xs, w_scale=ws, out_dtype=F32)[0]
    xs[3], xs[4], ws[7] = float("inf"), float("nan"), float("nan")
    y = hg.linear(x, w, x_scale=xs, w_scale=ws, out_dtype=F32)[0]
    rows, cols = torch.tensor([i for i in range(40) if i not in (3, 4)]), torch.arange(50) != 7
    assert torch.equal(y[rows][:, cols], clean[rows][:, cols])
    assert torch.isinf(y[3, cols]).all() and torch.isnan(y[4]).all() and torch.isnan(y[:, 7]).all()
    b = hg.linear(x, w, x_scale=xs, w_scale=ws, bias=rand(50, seed=3), act="relu")[0]
    assert b.dtype == BF16 and (torch.isinf(b[3, cols]) == (clean[3, cols] > 0)).all()
