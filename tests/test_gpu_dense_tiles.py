"""Products on 256 x 256 and 256 x 128 tiles, and products whose rows are cut into whole rounds of tiles and
a rest with tiles of its own: every type and direction, with all that an epilogue reads and writes.
(Which tiles a size gets is pinned by the tests of the plans.)"""
import pytest
import torch

import paper_2112_15345_amd as hg
from test_gpu_dense_linear import BF16, E4M3, F16, F32, check, check_grad, rand, to_8_bits

pytestmark = pytest.mark.gpu

# 33 x 17 tiles of 256 x 256 at depths of 8 slabs of 64 elements, and of 8 and a piece
LARGE = [(8201, 512, 4104), (8193, 520, 4112)]
# rounds of 256 x 256 tiles and a rest (1057 = 4 rounds and 33; 517 = 2 rounds and 5 of 8), of
# 128 x 128 (float32), and a rest of one row
ROUNDS = [(8201, 1032, 8200), (12_001, 1160, 2816)]


def forward(m, k, n, dtype, act, out=None):
    out = out or dtype
    x, w = rand(m, k, seed=1), rand(n, k, seed=2, scale=k ** -0.5)
    kw = {}
    if dtype == E4M3:
        (x, xs), (w, ws) = to_8_bits(x), to_8_bits(w)
        # (a scale of its own for each row: a shift by a row would show)
        kw = dict(x_scale=xs, w_scale=ws)
    else:
        x, w = x.to(dtype), w.to(dtype)
    bias = rand(n, seed=3)
    residual = rand(m, n + 3, dtype=out, seed=4)[:, 1:1 + n]
    got = hg.linear(x, w, bias=bias, act=act, residual=residual, out_dtype=out, keep_pre=True, **kw)
    check(x, w, got, bias, act, residual, kw.get("x_scale"), kw.get("w_scale"), out)
    bare = hg.linear(x, w, out_dtype=out, **kw)
    check(x, w, bare, xs=kw.get("x_scale"), ws=kw.get("w_scale"), out=out)


@pytest.mark.parametrize("dtype", [F16, BF16, E4M3])
@pytest.mark.parametrize("m,k,n", LARGE)
def test_forward(m, k, n, dtype):
    forward(m, k, n, dtype, "gelu", BF16 if dtype == E4M3 else None)


def test_forward_8_bits_to_float32():
    forward(*LARGE[1], E4M3, "silu", F32)


@pytest.mark.parametrize("dtype", [F32, F16, BF16, E4M3])
@pytest.mark.parametrize("m,k,n", ROUNDS)
def test_forward_in_rounds(m, k, n, dtype):
    forward(m, k, n, dtype, "relu", F16 if dtype == E4M3 else None)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("m,k,n", [(8201, 4104, 520), (8201, 4104, 1032), (8193, 8200, 1040)])
def test_backward(m, k, n, dtype):
    """dx on 256 x 256 tiles (in whole rounds and a rest from a depth of 16 slabs on), dw on 256 x 128."""
    x, w = rand(m, k, dtype=dtype, seed=1), rand(n, k, dtype=dtype, seed=2, scale=k ** -0.5)
    dy = rand(m, n, dtype=dtype, seed=3)
    pre = rand(m, n, dtype=dtype, seed=4, scale=2.0)
    for act in ("none", "silu"):
        p = None if act == "none" else pre
        got = hg.linear_grad(dy, x, w, pre=p, act=act, dw_dtype=F32 if act == "none" else None)
        check_grad(dy, x, w, p, act, got, F32 if act == "none" else None)


@pytest.mark.parametrize("dtype", [F16, BF16, E4M3])
def test_values_that_are_not_finite(dtype):
    """On 256 x 256 tiles: they stay in their rows and columns."""
    m, k, n = LARGE[1]
    x, w = rand(m, k, seed=1), rand(n, k, seed=2, scale=0.1)
    kw = {}
    if dtype == E4M3:
        (x, xs), (w, ws) = to_8_bits(x), to_8_bits(w)
        kw = dict(x_scale=xs, w_scale=ws)
    else:
        x, w = x.to(dtype), w.to(dtype)
    clean = hg.linear(x, w, **kw)[0]
    x[8192, k - 1], w[4111, 3] = float("nan"), float("nan")
    y = hg.linear(x, w, **kw)[0]
    assert torch.equal(y[:8192, :4111], clean[:8192, :4111])
    assert torch.isnan(y[8192]).all() and torch.isnan(y[:, 4111]).all()
