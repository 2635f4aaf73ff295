"""Accuracy of the head loss and log-sum-exp beyond worst-case bounds of their sums."""
import pytest
import torch

pytestmark = pytest.mark.gpu
pkg = pytest.importorskip("paper_2609_04526_gb300")


@pytest.fixture(scope="module")
def h():
    return pkg.Handle()


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_large_logits_lose_nothing(h, sign):
    """Two logits of size 64 to 256, both exact in fp32, 1 to 4 apart: the loss depends on their difference alone.

    Of the ratio of both exponentials each has the 2^-22 of a fast 2^x, its argument (within -8 .. 0, once
    rounded: half a unit 2^-22, times log 2) and log2(e)'s own rounding of 2^-25 on a difference of at most 4; then
    a quotient and a log1p of 2 units: below 1.1e-6 together."""
    c = torch.arange(64, 128, 0.5)
    c = torch.cat([c, 2 * c])  # exact in bf16
    X = torch.zeros(len(c), 8)
    X[:, 0] = sign * c
    W = torch.zeros(2, 8)
    W[0, 0], W[1, 0] = 1.0, 1.0 - sign * 2.0 ** -6
    loss, lse = h.sq_head_loss(X.bfloat16().cuda(), W.bfloat16().cuda(), torch.zeros(len(c), dtype=torch.int64, device="cuda"))
    h.sq_sync()
    want = torch.log1p(torch.exp(-c.double() / 64))
    assert float(((loss.double().cpu() - want) / want).abs().max()) <= 1.1e-6
    full = sign * c.double() + want  # of up to 260, rounded to fp32 once more
    assert float((lse.double().cpu() - full).abs().max()) <= 2.0 ** -16 + 1.1e-6
