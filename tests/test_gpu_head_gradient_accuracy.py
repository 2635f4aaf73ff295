"""Accuracy of the head loss's gradient as a norm, where the rows of the vocabulary projection share a part
or one competitor of the label holds most of the probability: the terms of the gradient then cancel."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
pkg = pytest.importorskip("paper_2609_04526_gb300")


@pytest.fixture(scope="module")
def h():
    return pkg.Handle()


def _case(T, D, V, common, rival, lean, seed):
    """Rows of W of independent directions plus one part common to all, `common` times their size; hidden rows
    without a share in that part that lean towards their label's row and towards that of one rival."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    own, part = normal(V, D) * (2.0 / math.sqrt(D)), normal(D)
    part *= 2.0 / part.norm()
    labels, rivals = (torch.randint(V, (T,), generator=g, device="cuda") for _ in range(2))
    X = normal(T, D)
    X = X - (X @ part)[:, None] * part / (part @ part) + lean * own[labels] + rival * own[rivals]
    return X.bfloat16(), (own + common * part).bfloat16(), labels


def _gradient(X, W, labels, dloss):
    """In 64 bits, a few hundred rows at a time."""
    W = W.double()
    out = []
    for x, y, g in zip(X.split(256), labels.split(256), dloss.split(256)):
        p = torch.softmax(x.double() @ W.t(), dim=1)
        p[torch.arange(len(y), device=y.device), y] -= 1
        out.append((p * g.double()[:, None]) @ W)
    return torch.cat(out)


def _check(h, X, W, labels):
    """With p the other entries' shares among themselves, dX = -g (1 - p_label) (W_label - sum p_v W_v). Its own
    rounding is at most 2^-9 of each element. Exponentials rounded by d_v of themselves, |d_v| <= 2^-9, and
    divided by their sum move the difference by sum p_v d_v (W_v - mean), at most 2^-9 of the size of a row's own
    part, and the difference itself is not smaller than that of the label's. Those sizes are within 1 +- 0.25 of each
    other (512 and more columns, 5 deviations), so 2^-8 and a quarter of a row's gradient; fp32 sums add less."""
    dloss = torch.full((len(X),), 1.0 / len(X), device="cuda")
    dX = h.sq_head_loss_grad(X, W, labels, dloss)[2]
    h.sq_sync()
    want = _gradient(X, W, labels, dloss)
    err = (dX.double() - want).norm(dim=1) / want.norm(dim=1)
    assert float(err.max()) <= 1.25 * 2.0 ** -8, (float(err.max()), float(err.mean()))


@pytest.mark.parametrize("T", [40, 256])
@pytest.mark.parametrize("common", [0.0, 3.0, 10.0, 30.0])
@pytest.mark.parametrize("rival, lean", [(0.0, 0.0), (3.0, 0.0), (2.0, 4.0)])
def test_rounded_exponentials_cancel(h, T, common, rival, lean):
    """What the weights share leaves the gradient exactly, however the exponentials are rounded."""
    _check(h, *_case(T, 512, 8000, common, rival, lean, seed=int(common) + T))


def test_small_factor_of_an_unlikely_label(h):
    """Gradients far below 1 of labels whose competitors are 2^95 as likely: no factor leaves fp32's normal range."""
    T, D, V = 70, 64, 700
    X, W, labels = _case(T, D, V, 0.0, 0.0, 0.0, seed=3)
    X[:, 0], W[:, 0] = 8.0, 0.0
    W[333, 0] = 95 * math.log(2) / 8
    labels = torch.where(labels == 333, 334, labels)
    dloss = torch.full((T,), 2.0 ** -50, device="cuda")
    dX = h.sq_head_loss_grad(X, W, labels, dloss)[2]
    h.sq_sync()
    want = _gradient(X, W, labels, dloss)
    err = (dX.double() - want).norm(dim=1) / want.norm(dim=1)
    assert float(err.max()) <= 1.25 * 2.0 ** -8, float(err.max())


@pytest.mark.parametrize("T, D, V", [(2048, 1024, 50257), (64, 32768, 8300)])
def test_long_sums_cancel(h, T, D, V):
    """Tens of thousands of products that add up to a part which the label's row takes away again: a sum
    truncated at every sixteenth product would be off by 2^-25 of itself for each, here 60 times the rows' own
    part and thousands of steps."""
    _check(h, *_case(T, D, V, 60.0, 0.0, 0.0, seed=T))
