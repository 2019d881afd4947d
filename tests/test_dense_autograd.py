"""The dense operators record nothing for autograd, and say so: a forward call refuses tensors that require a
gradient (checked first, so that no GPU is needed), unless gradients are off."""
import pytest
import torch

import paper_2112_15345_amd as hg


def refused(call):
    with pytest.raises(ValueError, match="gradient"):
        call()
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):  # (the next thing checked)
        call()


def test_forward_calls_refuse():
    x, g = torch.zeros(4, 8), torch.zeros(4, 8, requires_grad=True)
    w, b = torch.zeros(8), torch.zeros(4, requires_grad=True)
    for call in (lambda: hg.rms_norm(g), lambda: hg.rms_norm(x, w.clone().requires_grad_()),
                 lambda: hg.rms_norm(x, residual=g), lambda: hg.linear(g, x), lambda: hg.linear(x, g),
                 lambda: hg.linear(x, x, bias=b), lambda: hg.linear(x, x, residual=g * 2),
                 lambda: hg.distill(g, torch.zeros(4, 2, dtype=torch.int64), x[:, :2])):
        refused(call)


def test_calls_that_give_the_gradient_do_not():
    g = torch.zeros(4, 8, requires_grad=True)
    for call in (lambda: hg.distill(g, torch.zeros(4, 2, dtype=torch.int64), g[:, :2], want_grad=True),
                 lambda: hg.linear_grad(g, g, g), lambda: hg.rms_norm_grad(g, g)):
        with pytest.raises(ValueError, match="GPU"):
            call()


@pytest.mark.gpu
def test_inside_autograd():
    """A layer of one's own over the calls, and distill's gradient given back to autograd's logits."""
    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            ctx.save_for_backward(x, w)
            return hg.linear(x, w)[0]

        @staticmethod
        def backward(ctx, dy):
            x, w = ctx.saved_tensors
            return hg.linear_grad(dy, x, w, want_dbias=False)[:2]

    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.randn(40, 24, generator=gen, device="cuda")
    w = torch.randn(16, 24, generator=gen, device="cuda", requires_grad=True)
    ids = torch.randint(16, (40, 3), generator=gen, device="cuda")
    t = torch.randn(40, 3, generator=gen, device="cuda")
    logits = Layer.apply(x, w)
    loss, grad = hg.distill(logits, ids, t, want_grad=True)
    assert not loss.requires_grad and not grad.requires_grad
    logits.backward(grad)
    want = hg.linear_grad(grad, x, w, want_dx=False, want_dbias=False)[1]
    assert torch.equal(w.grad, want)
