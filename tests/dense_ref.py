"""The dense operators' definitions in 64 bits, and the bounds that their results are held to.

Unit roundoffs: a result in float32, float16 or bfloat16 is rounded once, to nearest (2^-24, 2^-11
and 2^-8 of its size; below the smallest normal number half a step of the subnormals).  A sum of n
terms in float32, in any order, is within n 2^-23 of the sum of the terms' sizes (2^-24 by
rounding; matrix instructions may cut instead of rounding).  exp2, log, rsqrt and a division are
within a few units of 2^-24, taken as 8."""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SUB = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}
E = 2.0 ** -24


def assert_close(got, want, size, what):
    """|got - want| <= size elementwise, with the same NaN and infinities; the bound's overflow
    cases (a want past the type's range) are not meant to occur in finite tests."""
    got, want, size = got.double(), want.double(), size.double()
    assert got.shape == want.shape, what
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), f"{what}: NaN at other places"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]) and not torch.isinf(got[~inf]).any(), f"{what}: inf"
    fine = ~(nan | inf)
    over = ((got - want).abs() - size)[fine]
    if over.numel():
        assert float(over.max()) <= 0, (
            f"{what}: {int((over > 0).sum())} of {over.numel()} out of bounds, worst by "
            f"{float(over.max()):.3g} of a bound of {float(size[fine][over.argmax()]):.3g}")


def rounding(want, dtype):
    return want.abs() * U[dtype] * 1.0001 + SUB[dtype]


def norm(x, weight, residual, eps):
    """(h, y, 1 / rms, relative error of y before rounding) of rows in double."""
    h = x.double() if residual is None else x.double() + residual.double()
    D = h.shape[1]
    s = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    y = h * s * (1.0 if weight is None else weight.double())
    # the mean of squares is a sum of positive terms (half its error reaches s), h itself is
    # rounded to 32 bits once, then two products
    return h, y, s, (0.5 * D * 2 + 24) * E


def act(z, name):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def act_slope(z, name):
    """The derivative, by autograd."""
    with torch.enable_grad():
        z = z.detach().clone().requires_grad_(True)
        (g,) = torch.autograd.grad(act(z, name).sum(), z)
    return g


def distill(logits, ids, teacher, T, row_weight):
    """(loss, grad, entropy-like size of the loss) in double, row by row rules included."""
    z = logits.double() / T
    n = z.shape[1]
    a = torch.ones(z.shape[0], dtype=torch.float64, device=z.device) if row_weight is None \
        else row_weight.double()
    bad = ((ids < -1) | (ids >= n)).any(1)
    t = teacher.double() / T
    off = (ids < 0) | (ids >= n) | (t == -math.inf)
    t = torch.where(off, -math.inf, t)
    some = (~off).any(1)
    p = torch.softmax(torch.where(some[:, None], t, 0.0), 1) if ids.shape[1] else t
    p = torch.where(off | ~some[:, None], 0.0, p)
    lq = torch.log_softmax(z, 1)
    at = ids.clamp(0, n - 1)
    each = torch.where(p == 0, 0.0, p * (torch.log(p) - lq.gather(1, at)))
    size = torch.where(p == 0, 0.0, p * (torch.log(p).abs() + lq.gather(1, at).abs() + 1)).sum(1)
    loss = each.sum(1)
    grad = torch.exp(lq).scatter_add(1, at, -p) * (a / T)[:, None]
    nan = torch.isnan(p).any(1) | torch.isnan(lq).any(1)
    loss = torch.where(nan, math.nan, loss)
    grad = torch.where(nan[:, None], math.nan, grad)
    empty = ~some & ~bad
    loss = torch.where(bad, math.nan, torch.where(empty, 0.0, loss))
    grad = torch.where(bad[:, None], math.nan, torch.where(empty[:, None], 0.0, grad))
    grad = torch.where((a == 0)[:, None], 0.0, grad)
    return loss, grad, size, p, torch.exp(lq)
