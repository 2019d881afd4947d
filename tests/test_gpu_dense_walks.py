"""The norms over more rows than a grid has groups, so that every group takes several: forward and
backward against the definition in 64 bits, for each way a row is shared."""
import pytest
import torch

import dense_ref as R
import paper_2112_15345_amd as hg

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn


def rand(*shape, dtype=F32, seed=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


# (rows of a block at a time: 32, 16, 8, 4 and 1; at most 2048 blocks going forward and 1024
# backward)
WALKS = [(150_001, 40), (80_003, 100), (40_001, 250), (20_011, 500), (9001, 1999), (5003, 4090), (4097, 8001),
         (2500, 9001)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", WALKS)
def test_forward(rows, dim, dtype):
    x, r = rand(rows, dim, dtype=dtype, seed=1), rand(rows, dim, dtype=dtype, seed=2)
    w = 1 + rand(dim, seed=3, scale=0.2)
    y, total, _ = hg.rms_norm(x, w, residual=r, eps=1e-5)
    h, want, _, rel = R.norm(x, w, r, 1e-5)
    R.assert_close(total, h, R.rounding(h, dtype) + h.abs() * R.E, "sum")
    R.assert_close(y, want, R.rounding(want, dtype) + want.abs() * rel, "y")
    ids = torch.randint(rows, (rows,), device="cuda")
    y8, _, scale = hg.rms_norm(x, w, ids=ids, eps=1e-5, out_dtype=E4M3)
    _, want, _, rel = R.norm(x[ids], w, None, 1e-5)
    value = y8.double() * scale.double()[:, None]
    R.assert_close(value, want, want.abs() * (2 * rel + 2.0 ** -4 * 1.001)
                   + scale.double()[:, None] * 2.0 ** -10 * 1.001, "y8")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,dim", WALKS)
def test_backward(rows, dim, dtype):
    x, dy = rand(rows, dim, dtype=dtype, seed=1), rand(rows, dim, dtype=dtype, seed=2)
    w, ds = 1 + rand(dim, seed=3, scale=0.2), rand(rows, dim, dtype=dtype, seed=4)
    dx, dw = hg.rms_norm_grad(dy, x, w, dsum=ds, eps=1e-5)
    h, _, s, rel = R.norm(x, w, None, 1e-5)
    g = dy.double() * w.double()
    want = s * (g - h * s * s * (g * h).mean(1, keepdim=True))
    size = rel * s * (g.abs() + h.abs() * s * s * 4 * (g * h).abs().mean(1, keepdim=True))
    want = want + ds.double()
    size = size + R.E * (want.abs() + ds.double().abs())
    R.assert_close(dx, want, R.rounding(want, dtype) + 2 * size, "dx")
    terms = dy.double() * h * s
    # a sum of `rows` terms in some order, and no wider: a row left out or taken twice is a term of
    # some 1 among sums of sizes of the root of their number
    R.assert_close(dw, terms.sum(0),
                   terms.abs().sum(0) * (rel + (rows + 8) * 2 * R.E), "dweight")
    near = (dw.double() - terms.sum(0)).abs().max()
    assert float(near) < 0.02 * rows ** 0.5
