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


@pytest.mark.parametrize("T", [40, 512])
@pytest.mark.parametrize("lean", [0.0, 2.0])
def test_no_bias_of_wide_rows(h, T, lean):
    """Mean and root mean square error over the tokens, rows of width 4096.

    The tensor core truncates at each sixteenth product. Where 512 products are added up at a time, the logits that
    count (about 8) are eight such sums whose running value is about 1/2: 256 steps that take half a unit of 2^-24 off,
    4e-6 at most where all point the same way. In one sum of 4096 products the running value is about 4 and its
    unit eight times as large."""
    D, V = 4096, 8000
    g = torch.Generator(device="cuda").manual_seed(T)
    W = (torch.randn(V, D, generator=g, device="cuda") * 2.0 * D ** -0.5).bfloat16()
    labels = torch.randint(V, (T,), generator=g, device="cuda")
    X = (torch.randn(T, D, generator=g, device="cuda") + lean * W[labels].float()).bfloat16()
    loss, lse = h.sq_head_loss(X, W, labels)
    h.sq_sync()
    z = X.double() @ W.double().t()
    want = torch.logsumexp(z, dim=1)
    for got, exact in ((lse, want), (loss, want - z.gather(1, labels[:, None])[:, 0])):
        err = got.double() - exact
        assert abs(float(err.mean())) <= 4e-6 and float(err.square().mean().sqrt()) <= 4e-6, (float(err.mean()), float(err.std()))
