"""The head loss at each tile width that its rule picks for few tokens, on whatever number of SMs there is."""
import pytest
import torch

pytestmark = pytest.mark.gpu
pkg = pytest.importorskip("paper_2609_04526_gb300")


@pytest.fixture(scope="module")
def h():
    return pkg.Handle()


def _width(V, clusters):
    """Columns of a tile of the logits for up to 64 tokens: by the waves of the launch, a tile of 128 columns lasting
    0.54 and one of 64 lasting 0.4 of one of 256."""
    waves = lambda columns: -(-(-(-V // columns)) // clusters)  # noqa: E731
    wide, half, quarter = waves(256), 0.54 * waves(128), 0.4 * waves(64)
    if quarter < wide and quarter < half:
        return 64
    return 128 if half < wide else 256


def _vocabulary(columns, at_least):
    """An odd vocabulary of at least so many entries that takes tiles of this width."""
    clusters = torch.cuda.get_device_properties(0).multi_processor_count // 2
    return next(V for V in range(at_least | 1, 60000, 2) if _width(V, clusters) == columns)


def _case(T, D, V, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    W = (torch.randn(V, D, generator=g, device="cuda") * 2.0 * D ** -0.5).bfloat16()
    labels = torch.randint(V, (T,), generator=g, device="cuda")
    X = (torch.randn(T, D, generator=g, device="cuda") + 0.5 * W[labels].float()).bfloat16()
    return X, W, labels, torch.rand(T, generator=g, device="cuda") + 0.5


@pytest.mark.parametrize("columns, at_least", [(64, 3001), (128, 5001), (128, 20001), (256, 10001), (256, 24001)])
@pytest.mark.parametrize("T", [1, 16, 17, 33, 64])
def test_few_tokens(h, T, columns, at_least):
    """Loss, log-sum-exp and gradient against 64 bits; the same bits without the gradient and among more tokens.

    A logit is the sum of three sums of 512 products or fewer, 32 steps of 16 each, of which each step takes at most a
    unit of 2^-21 (values below 8) off: 5e-5; the sum of up to 60000 exponentials and its logarithm add 1e-5. The
    gradient is off by its own rounding and that of the exponentials, 2^-9 each."""
    D = 1096
    V = _vocabulary(columns, at_least)
    X, W, labels, dloss = _case(300, D, V, T + V)
    some = slice(100, 100 + T)
    x, y, g = X[some].contiguous(), labels[some].clone(), dloss[some].clone()
    loss, lse, dX = h.sq_head_loss_grad(x, W, y, g)
    loss2, lse2 = h.sq_head_loss(x, W, y)
    every, every_lse = h.sq_head_loss(X, W, labels)
    h.sq_sync()
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    assert torch.equal(loss, every[some]) and torch.equal(lse, every_lse[some])
    z = x.double() @ W.double().t()
    want = torch.logsumexp(z, dim=1)
    assert float((lse.double() - want).abs().max()) <= 6e-5
    assert float((loss.double() - want + z.gather(1, y[:, None])[:, 0]).abs().max()) <= 6e-5
    p = torch.softmax(z, dim=1)
    p[torch.arange(T, device="cuda"), y] -= 1
    dwant = (p * g.double()[:, None]) @ W.double()
    assert float(((dX.double() - dwant).norm(dim=1) / dwant.norm(dim=1)).max()) <= 1.25 * 2.0 ** -8


@pytest.mark.parametrize("T", [65, 128, 129, 200, 256])
def test_one_row_of_tiles(h, T):
    """More tokens in one row of tiles, of 128 or 64 columns where 256 leave clusters idle."""
    for columns, at_least in ((64, 3001), (128, 5001), (256, 12001)):
        V = _vocabulary(columns, at_least)
        X, W, labels, dloss = _case(T, 584, V, T + V)
        loss, lse, dX = h.sq_head_loss_grad(X, W, labels, dloss)
        h.sq_sync()
        z = X.double() @ W.double().t()
        want = torch.logsumexp(z, dim=1)
        assert float((lse.double() - want).abs().max()) <= 6e-5
        p = torch.softmax(z, dim=1)
        p[torch.arange(T, device="cuda"), labels] -= 1
        dwant = (p * dloss.double()[:, None]) @ W.double()
        assert float(((dX.double() - dwant).norm(dim=1) / dwant.norm(dim=1)).max()) <= 1.25 * 2.0 ** -8
