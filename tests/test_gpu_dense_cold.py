"""distill at the lowest temperature: softmax picks the largest logit."""
import pytest
import torch

import paper_2112_15345_amd as hg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("classes", [50, 3000, 70_000, 140_000])
def test_lowest_temperature(classes):
    """p and q are 1 at one class each, so that loss and gradient are exact."""
    T = 2.0 ** -126
    z = torch.arange(classes, device="cuda").remainder(97).float().mul(0.01).repeat(3, 1)
    z[:, 11] = 2.0
    ids = torch.tensor([[11, 12, 13], [14, 15, 16], [17, 18, -1]], device="cuda")
    t = torch.tensor([[3.0, 1.0, 2.0], [1.0, 0.0, -1.0], [0.0, 1.0, 9.0]], device="cuda")
    loss, grad = hg.distill(z, ids, t, temperature=T, want_grad=True)
    picked = [11, 14, 18]
    for row, at in enumerate(picked):
        assert float(loss[row]) == float(2.0 - z[row, at]) / T  # (a difference in 32 bits)
        want = torch.zeros(classes, device="cuda")
        want[11] += 1 / T
        want[at] -= 1 / T
        assert torch.equal(grad[row], want)
    assert torch.equal(hg.distill(z, ids, t, temperature=T)[0], loss)
