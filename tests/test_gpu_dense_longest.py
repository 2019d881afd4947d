"""Rows about as long as the dense operators take them (2^31 - 1 elements): their counters pass neither
the row's end nor their own range.  Of ones and zeros, whose sums over a thread's part of the row
(2^23 elements) and over the row are exact in 32 bits."""
import math

import pytest
import torch

import paper_2112_15345_amd as hg

pytestmark = pytest.mark.gpu

BF16, E4M3 = torch.bfloat16, torch.float8_e4m3fn
LENGTHS = [(1 << 31) - 1, (1 << 31) - 2043]


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dim", LENGTHS)
def test_norm(dim):
    x = torch.ones(1, dim, dtype=BF16, device="cuda")
    x[0, -1] = 0
    y = hg.rms_norm(x)[0]
    assert int((y == 1).sum()) == dim - 1 and float(y[0, -1]) == 0
    y, _, scale = hg.rms_norm(x, eps=0.0, out_dtype=E4M3)
    q = y.view(torch.uint8)
    assert int((q == 0x7e).sum()) == dim - 1 and int(q[0, -1]) == 0  # (0x7e: 448)
    assert abs(float(scale[0]) * 448 - 1) <= 2.0 ** -21


@pytest.mark.parametrize("dim", LENGTHS)
def test_norm_gradient(dim):
    """Of a row of ones and a gradient of ones nothing is left but what s and the mean are off by
    (some units of 2^-24); dsum is added to it."""
    x = torch.ones(1, dim, dtype=BF16, device="cuda")
    dx, none = hg.rms_norm_grad(x, x, eps=0.0)
    assert none is None and float(dx.abs().amax()) <= 2.0 ** -20
    dx = hg.rms_norm_grad(x, x, dsum=x, eps=0.0)[0]
    assert int((dx == 1).sum()) == dim


@pytest.mark.parametrize("classes", LENGTHS)
def test_distill(classes):
    """All classes alike: q is 1 / classes, and the listed one's entry is q - 1."""
    z = torch.zeros(1, classes, dtype=BF16, device="cuda")
    ids = torch.full((1, 1), classes - 1, device="cuda")
    t = torch.zeros(1, 1, device="cuda")
    want = math.log(classes)
    loss, none = hg.distill(z, ids, t)
    assert none is None and abs(float(loss[0]) - want) <= 8 * 2.0 ** -24 * want
    loss, grad = hg.distill(z, ids, t, want_grad=True)
    assert abs(float(loss[0]) - want) <= 8 * 2.0 ** -24 * want
    assert int((grad == 2.0 ** -31).sum()) == classes - 1 and float(grad[0, -1]) == -1
