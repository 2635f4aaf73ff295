"""Relative accuracy of routing weights and their gradient over many orders of magnitude."""
import pytest
import torch

pytestmark = pytest.mark.gpu
pkg = pytest.importorskip("paper_2609_04526_gb300")


@pytest.mark.parametrize("normalize", [True, False])
def test_weights_far_apart(normalize):
    """Two logits d apart, d up to 80: a fast 2^x is good to 2^-22 of itself and its argument adds nothing; a sum, a
    reciprocal or quotient and products round at 2^-24 each, five in a weight and eight in a gradient."""
    h = pkg.Handle()
    d = torch.linspace(0.01, 80.0, 4001, device="cuda")
    z = torch.stack([torch.zeros_like(d), -d], dim=1).contiguous()
    experts, weights = h.sq_route(z, 2, normalize=normalize)
    dz = h.sq_route_grad(z, experts, torch.tensor([[0.0, 1.0]], device="cuda").repeat(len(d), 1), normalize=normalize)
    h.sq_sync()
    q = torch.softmax(z.double(), dim=1)
    assert torch.equal(experts.cpu(), torch.tensor([[0, 1]], dtype=torch.int32).expand(len(d), 2))
    assert float(((weights.double() - q) / q).abs().max()) <= 2.0 ** -22 + 5 * 2.0 ** -24
    want = q[:, 1] * q[:, 0]
    assert float(((dz[:, 1].double() - want) / want).abs().max()) <= 2.0 ** -22 + 8 * 2.0 ** -24
