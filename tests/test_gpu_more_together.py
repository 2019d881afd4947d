"""Embedding, layer norm, products, kept activations and the table's step as a training step runs them,
on the rows of a mini-batch; and the same layer served in 8-bit integers.  Every stage is held to its
definition in 64 bits on the inputs that it had."""
import pytest
import torch

import dense_ref as R
import paper_2112_15345_amd as hg
from test_gpu_dense_linear import rand
from test_gpu_layer_norm import Ref

pytestmark = pytest.mark.gpu

F32, BF16, I8 = torch.float32, torch.bfloat16, torch.int8
GROUP = hg.HG_KEPT_GROUP
NODES, DIM, HIDDEN = 3000, 192, 640


def graph():
    """A graph whose vertices have no features, and a mini-batch of it."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    deg = torch.bincount(torch.randint(NODES, (20_000,), generator=g, device="cuda"), minlength=NODES)
    indptr = torch.zeros(NODES + 1, dtype=torch.int64, device="cuda")
    indptr[1:] = torch.cumsum(deg, 0)
    indices = torch.randint(NODES, (20_000,), generator=g, device="cuda")
    gr = hg.Graph([(NODES, None)], [(0, 0, indptr, indices)], device="cuda")
    seeds = torch.randperm(NODES, generator=g, device="cuda")[:100]
    return gr.sample_blocks([seeds], [[5], [5]], rng_seed=1)


def stands_for(q, scale):
    return q.double() * scale.double().repeat_interleave(GROUP, 1)[:, :q.shape[1]]


class Layer:
    """h = embed(ids); n = layer_norm(h); u = gelu(n W1 + b1); y = u W2 + h, in float32."""

    def __init__(self):
        self.table = rand(NODES, DIM, seed=1, scale=DIM ** -0.5)
        self.norm, self.shift = 1 + rand(DIM, seed=2, scale=0.1), rand(DIM, seed=3, scale=0.1)
        self.w1, self.b1 = rand(HIDDEN, DIM, seed=4, scale=DIM ** -0.5), rand(HIDDEN, seed=5)
        self.w2 = rand(DIM, HIDDEN, seed=6, scale=HIDDEN ** -0.5)

    def forward(self, ids):
        """y, and what the backward pass reads: the rows that products took, in 8 bits."""
        h = hg.embed(self.table, ids, scale=DIM ** 0.5)
        n = hg.layer_norm(h, self.norm, self.shift)[0]
        u, pre = hg.linear(n, self.w1, bias=self.b1, act="gelu", keep_pre=True)
        y = hg.linear(u, self.w2, residual=h)[0]
        return y, (h, *(hg.quantize(t, group=GROUP) for t in (n, pre, u)))

    def backward(self, dy, kept, ids):
        h, n8, pre8, u8 = kept
        du, dw2, _ = hg.linear_grad(dy, u8[0], self.w2, x_scale=u8[1], group=GROUP, want_dbias=False)
        dn, dw1, db1 = hg.linear_grad(du, n8[0], self.w1, pre=pre8[0], act="gelu", x_scale=n8[1],
                                      pre_scale=pre8[1], group=GROUP)
        dh, dnorm, dshift = hg.layer_norm_grad(dn, h, self.norm, dsum=dy)
        return dict(du=du, w2=dw2, dn=dn, w1=dw1, b1=db1, dh=dh, norm=dnorm, shift=dshift,
                    table=hg.embed_grad(dh, ids, NODES, scale=DIM ** 0.5))


def test_training_step():
    ids = graph().input_nodes(0)
    assert 100 < ids.numel() < NODES
    L = Layer()
    y, kept = L.forward(ids)
    h, n8, pre8, u8 = kept
    # forward: each stage from the definition of the one before
    h64 = L.table.double()[ids] * DIM ** 0.5
    n64, n_off = Ref(h64, None, 1e-5).forward(L.norm, L.shift)
    pre64 = n64 @ L.w1.double().t() + L.b1.double()
    u64 = R.act(pre64, "gelu")
    y64 = u64 @ L.w2.double().t() + h64
    # by 32 bits alone, (2 terms + 8) 2^-24 of a product's terms: 392 of 9 for pre (2.2e-4), which go
    # on through 20 of |w2|, and 1288 of 10 for y: 6e-3
    assert float((y.double() - y64).abs().max()) < 6e-3
    # kept within half a step (0.01 and more, next to which 2.5e-4 is 0.025)
    for (q, c), want in ((n8, n64), (pre8, pre64), (u8, u64)):
        step = c.double().repeat_interleave(GROUP, 1)[:, :q.shape[1]]
        assert float(((stands_for(q, c) - want).abs() / step).max()) < 0.53
    # backward, from what was kept
    dy = rand(*y.shape, seed=9)
    g = L.backward(dy, kept, ids)
    n, pre, u = (stands_for(*t) for t in (n8, pre8, u8))
    du = dy.double() @ L.w2.double()
    dz = du * R.act_slope(pre, "gelu")
    dn = dz @ L.w1.double()
    dh, _, terms, _ = Ref(h, None, 1e-5).backward(dn, L.norm)
    dh = dh + dy.double()
    table = torch.zeros(NODES, DIM, dtype=torch.float64, device="cuda")
    table.index_add_(0, ids, dh * DIM ** 0.5)
    for name, want in dict(du=du, w2=dy.double().t() @ u, dn=dn, w1=dz.t() @ n, b1=dz.sum(0), dh=dh,
                           norm=terms.sum(0), shift=dn.sum(0), table=table).items():
        got = g[name].double()
        # four products in a row at most, whose roundings fall independently: 2^-24 sqrt(2 terms) of
        # the terms' root mean square each, some 4 x 37 x 2^-24 = 1e-5 of the result for 700 terms
        assert float((got - want).norm() / want.norm()) < 1e-4, name
    # the table's step in place is the same gradient's
    table = L.table.clone()
    hg.embed_grad(g["dh"], ids, NODES, scale=-0.1 * DIM ** 0.5, into=L.table)
    want = table.double() - 0.1 * g["table"].double()
    assert float((L.table.double() - want).abs().max()) < 1e-5
    rest = torch.ones(NODES, dtype=torch.bool, device="cuda")
    rest[ids] = False
    assert torch.equal(L.table[rest], table[rest])


def test_step_is_repeated_bit_for_bit_and_captured():
    ids = graph().input_nodes(0)
    L = Layer()
    y, kept = L.forward(ids)
    dy = rand(*y.shape, seed=9)
    first = L.backward(dy, kept, ids)
    torch.cuda.synchronize()
    c = torch.cuda.CUDAGraph()
    with torch.cuda.graph(c):
        y2, kept2 = L.forward(ids)
        again = L.backward(dy, kept2, ids)
    for seed in (11, 12, 13):
        dy.copy_(rand(*y.shape, seed=seed))
        y, kept = L.forward(ids)
        first = L.backward(dy, kept, ids)
        c.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and all(torch.equal(first[k], again[k]) for k in first)


@pytest.mark.parametrize("rows", [1, 7, 300])
def test_served_in_integers(rows):
    """The layer with weights and rows in 8-bit integers: off by what half a step of each element makes."""
    L = Layer()
    ids = torch.arange(rows, device="cuda") * 5
    h = hg.embed(L.table, ids, scale=DIM ** 0.5)
    w1, c1 = hg.quantize(L.w1)
    w2, c2 = hg.quantize(L.w2)
    q, _, c = hg.layer_norm(h, L.norm, L.shift, out_dtype=I8)
    u = hg.linear(q, w1, bias=L.b1, act="gelu", x_scale=c, w_scale=c1, out_dtype=F32)[0]
    uq, uc = hg.quantize(u)
    y = hg.linear(uq, w2, residual=h, x_scale=uc, w_scale=c2, out_dtype=F32)[0]
    n64 = Ref(h, None, 1e-5).forward(L.norm, L.shift)[0]

    def product(x, x_step, w, w_step):
        """A product of values that are each within their step: the result and its bound."""
        off = x_step @ (w.abs() + w_step).t() + x.abs() @ w_step.t()
        return x @ w.t(), off

    half = lambda s, like: (0.501 * s.double()[:, None]).expand_as(like)  # noqa: E731
    z, off = product(n64, half(c, n64), L.w1.double(), half(c1, L.w1))
    z = z + L.b1.double()
    R.assert_close(u, R.act(z, "gelu"), 1.13 * off + 1e-4 * (1 + z.abs()), "hidden")
    z, off = product(u.double(), half(uc, u), L.w2.double(), half(c2, L.w2))
    R.assert_close(y, z + h.double(), off + 1e-4 * (1 + z.abs() + h.double().abs()), "y")
