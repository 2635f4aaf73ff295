"""The example's training step, router to loss and back, against the same layer in 64 bits."""
import os
import sys

import pytest
import torch

from conftest import ROOT

pytestmark = pytest.mark.gpu
pkg = pytest.importorskip("paper_2609_04526_gb300")
sys.path.insert(0, os.path.join(ROOT, "examples"))

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _codes(w):
    """E2M1 values [E, N, K] of the packed codes."""
    lut = torch.tensor(GRID + tuple(-v for v in GRID), dtype=torch.float64, device=w.codes.device)
    return torch.stack([lut[(w.codes & 15).long()], lut[(w.codes >> 4).long()]], dim=-1).flatten(2)


def _reference(layer, X, labels, bytes_scale):
    """The step in 64 bits with autograd, rows one expert at a time; scales enter as leaves."""
    scale = {n: s.double().requires_grad_() for n, s in bytes_scale.items()}
    W = {n: _codes(w) * scale[n].repeat_interleave(w.K // scale[n].shape[2], dim=2) for n, w in layer.weights.items()}
    x = X.double().requires_grad_()
    logits = (X.float() @ layer.router.t()).double().requires_grad_()
    top, experts = torch.sort(logits, dim=1, descending=True, stable=True)
    p = torch.softmax(top[:, :layer.top_k], dim=1)
    y = torch.zeros_like(x)
    for j in range(layer.top_k):
        e = experts[:, j]
        rows = []
        for t in range(len(x)):
            gate, up = W["gate"][e[t]] @ x[t], W["up"][e[t]] @ x[t]
            rows.append(W["down"][e[t]] @ (gate * torch.sigmoid(gate) * up))
        y = y + p[:, j:j + 1] * torch.stack(rows)
    out = X.double() + y  # the residual path carries no gradient to x here: step() returns the experts' alone
    keep = labels >= 0
    z = out @ layer.head.double().t()
    loss = torch.logsumexp(z, dim=1) - z.gather(1, labels.clamp(min=0)[:, None])[:, 0]
    (loss * keep).sum().div(keep.sum()).backward()
    return torch.where(keep, loss, 0.0).detach(), x.grad, logits.grad, {n: s.grad for n, s in scale.items()}


@pytest.mark.parametrize("fmt", [0, 1])
def test_step_against_64_bits(fmt):
    import moe_step
    h = pkg.Handle()
    layer = moe_step.Layer(fmt, E=6, top_k=2, hidden=128, inter=96, vocab=515, seed=fmt)
    X, labels = moe_step.batch(layer, 45)
    got = moe_step.step(h, layer, X, labels)
    h.sq_sync()
    loss, dX, dlogits, dscale = _reference(layer, X, labels, layer.latent)

    def near(a, b, what, rel):
        err = float((a.double() - b).norm() / b.norm())
        assert err < rel, (what, err)

    # bf16 activations between the calls: each of the ~6 roundings on a path is at most 2^-8 of its value,
    # so below 2.4 % together where nothing cancels; the gradients' rows pass 10 of them
    near(got["loss"], loss, "loss", 0.01)
    near(got["dX"], dX, "dX", 0.04)
    near(got["dlogits"], dlogits, "dlogits", 0.04)
    for name in moe_step.LINEARS:
        near(got["scale_grads"][name], dscale[name], name, 0.04)


@pytest.mark.parametrize("fmt", [0, 1])
def test_training_lowers_the_loss(fmt):
    import moe_step
    layer = moe_step.Layer(fmt, E=8, top_k=2, hidden=256, inter=128, vocab=1000)
    X, labels = moe_step.batch(layer, 200)
    losses = moe_step.train(pkg.Handle(), layer, X, labels, steps=12, lr=0.1 if fmt else 0.05)
    assert losses[-1] < losses[0] - 0.05, losses


def test_padding_and_no_targets():
    """Padding tokens reach no expert; without a target the loss and every gradient are zero."""
    import moe_step
    h = pkg.Handle()
    layer = moe_step.Layer(0, E=4, top_k=2, hidden=64, inter=64, vocab=100)
    X, labels = moe_step.batch(layer, 33)
    valid = torch.ones(33, dtype=torch.uint8, device="cuda")
    valid[20:] = 0
    got = moe_step.step(h, layer, X, torch.full_like(labels, -100), valid=valid)
    assert got["rows"][-1] == 40
    assert torch.equal(got["out"][20:], X[20:])
    for t in [got["loss"], got["dX"], got["dlogits"], *got["scale_grads"].values()]:
        assert not t.any()
