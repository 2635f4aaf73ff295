"""Cross entropy against the vocabulary projection and its gradient, against 64-bit forms."""
import math

import numpy as np
import pytest
import torch

import step_ref as ref

pytestmark = pytest.mark.gpu
pkg = pytest.importorskip("paper_2609_04526_gb300")


@pytest.fixture(scope="module")
def h():
    return pkg.Handle()


def _case(T, D, V, seed, ignored=0.25, lean=1.0, scale=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    W = (torch.randn(V, D, generator=g, device="cuda") * (scale / math.sqrt(D))).bfloat16()
    labels = torch.randint(V, (T,), generator=g, device="cuda")
    X = (torch.randn(T, D, generator=g, device="cuda") + lean * W[labels].float()).bfloat16()
    off = torch.rand(T, generator=g, device="cuda") < ignored
    labels = torch.where(off, torch.where(torch.rand(T, generator=g, device="cuda") < 0.5, -100, V), labels)
    dloss = torch.rand(T, generator=g, device="cuda") * 2 - 0.5
    return X, W, labels, dloss


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64) if t.is_floating_point() else t.cpu().numpy()


def _check(h, X, W, labels, dloss, rows=None):
    """Both entry points against the 64-bit form (of `rows`, where the whole is too large)."""
    loss, lse, dX = h.sq_head_loss_grad(X, W, labels, dloss)
    loss2, lse2 = h.sq_head_loss(X, W, labels)
    h.sq_sync()
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    at = slice(None) if rows is None else rows
    x = torch.where(((labels >= 0) & (labels < len(W)))[:, None], X, torch.zeros_like(X))
    want = ref.head_loss(_np(x[at]), _np(W), _np(labels[at]), _np(dloss[at]))
    for name, got in (("loss", loss), ("lse", lse), ("dX", dX)):
        err = np.abs(_np(got[at]) - want[name])
        assert np.all(err <= want[name + "_err"]), (name, float(np.nanmax(err)), int((~(err <= want[name + "_err"])).sum()))
    return loss, lse, dX


@pytest.mark.parametrize("T, D, V", [(1, 8, 1), (1, 8, 2), (3, 16, 5), (2, 64, 129), (7, 136, 255), (64, 512, 1000), (129, 264, 256),
                                     (257, 128, 257), (300, 1032, 640), (513, 72, 3001), (40, 2048, 4099), (130, 4096, 1111)])
def test_parity(h, T, D, V):
    _check(h, *_case(T, D, V, T + D + V))


@pytest.mark.parametrize("T", [1, 255, 256, 257, 700])
def test_no_token_or_every_token_labelled(h, T):
    X, W, labels, dloss = _case(T, 128, 300, T, ignored=0.0)
    _check(h, X, W, labels, dloss)
    X.fill_(float("nan"))
    loss, lse, dX = h.sq_head_loss_grad(X, W, torch.full_like(labels, -100), dloss)
    assert not loss.any() and not lse.any() and not dX.any()


def test_empty(h):
    X, W, labels, dloss = _case(1, 64, 100, 0)
    loss, lse, dX = h.sq_head_loss_grad(X[:0], W, labels[:0], dloss[:0])
    assert loss.numel() == lse.numel() == dX.numel() == 0


def test_unlabelled_rows_reach_nothing(h):
    """Rows, weights and labels of tokens that are no targets may hold anything."""
    X, W, labels, dloss = _case(400, 256, 1500, 17, ignored=0.4)
    off = (labels < 0) | (labels >= len(W))
    clean = _check(h, X, W, labels, dloss)
    X2, dloss2 = X.clone(), dloss.clone()
    X2[off] = float("nan")
    dloss2[off] = float("inf")
    labels2 = torch.where(off, torch.where(torch.arange(400, device="cuda") % 2 == 0, -2 ** 62, 2 ** 62), labels)
    for got, want in zip(h.sq_head_loss_grad(X2, W, labels2, dloss2), clean):
        assert torch.equal(got, want)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_not_finite_rows_stay_alone(h, bad):
    """A labelled row that holds NaN or an infinity has a loss that is not a number; no other has."""
    X, W, labels, dloss = _case(300, 256, 700, 23, ignored=0.0)
    clean = h.sq_head_loss_grad(X, W, labels, dloss)
    X2 = X.clone()
    X2[77, 5] = bad
    loss, lse, dX = h.sq_head_loss_grad(X2, W, labels, dloss)
    keep = torch.arange(300, device="cuda") != 77
    assert not torch.isfinite(loss[77]) and not torch.isfinite(lse[77])
    for got, want in zip((loss, lse, dX), clean):
        assert torch.equal(got[keep], want[keep])


@pytest.mark.parametrize("gap", [60.0, 90.0, 140.0, 250.0, 1000.0])
def test_labels_far_below_the_largest_logit(h, gap):
    """Logits up to `gap` above the label's, in some half tiles only: their reference moves, and the
    others' exponentials follow it."""
    T, D, V = 300, 128, 900
    X, W, labels, dloss = _case(T, D, V, 41, ignored=0.1)
    X[:, 0] = 8.0
    W[:, 0] = 0.0
    W[130:133, 0] = gap / 8
    W[500, 0] = gap / 16
    W[700, 0] = -gap / 8
    _check(h, X, W, labels, dloss)


def test_confident_labels(h):
    """Losses down to 1e-6 keep their leading digits: p_label - 1 is formed without cancellation."""
    X, W, labels, dloss = _case(256, 512, 2000, 5, ignored=0.0, lean=5.0)
    loss, lse, _ = _check(h, X, W, labels, dloss)
    want = ref.head_loss(_np(X), _np(W), _np(labels))["loss"]
    small = want < 1e-2
    assert small.sum() > 50
    z = _np(X) @ _np(W).T
    dz = 2 * ref.U32 * (512 + 4) * (np.abs(_np(X)) @ np.abs(_np(W)).T).max(1)  # bound of a logit's error
    assert np.all(np.abs(_np(loss) - want)[small] <= (4 * dz + 1e-4)[small] * want[small]), z.max()


def test_several_chunks(h):
    """More labelled tokens than the exponentials' scratch holds at once."""
    X, W, labels, dloss = _case(2500, 64, 131075, 3, ignored=0.02)
    rows = torch.tensor([0, 1, 255, 256, 1023, 2040, 2047, 2048, 2060, 2303, 2304, 2499], device="cuda")
    _check(h, X, W, labels, dloss, rows)


def test_several_pieces(h):
    """More tokens than are packed at once."""
    X, W, labels, dloss = _case(16384 * 2 + 77, 64, 500, 4, ignored=0.5)
    rows = torch.cat([torch.arange(a, a + 40, device="cuda") for a in (0, 16364, 16384 * 2 - 20, 16384 * 2 + 37)])
    _check(h, X, W, labels, dloss, rows)


@pytest.mark.parametrize("D, V", [(64, 300), (512, 5000)])
def test_gradient_against_differences(h, D, V):
    """sum(dloss loss) along one column of X, from central differences of the loss itself."""
    T, step = 64, 2.0 ** -4
    X, W, labels, dloss = _case(T, D, V, 6, ignored=0.2)
    X = (torch.round(X.float() * 16) / 16).clamp(-4, 4).bfloat16()  # X +- step stays exact in bf16
    loss, lse, dX = h.sq_head_loss_grad(X, W, labels, dloss)
    for d in range(0, D, D // 8):
        up, down = X.clone(), X.clone()
        up[:, d] += step
        down[:, d] -= step
        diff = (h.sq_head_loss(up, W, labels)[0] - h.sq_head_loss(down, W, labels)[0]).double() * dloss.double() / (2 * step)
        w = W[:, d].double().abs().max()
        # third derivative of the loss along a column: at most ~ (2 w)^3; fp32 noise of the losses; bf16 of dX
        bound = dloss.abs().double() * ((2 * w) ** 3 * step ** 2 / 6 + 2e-5 / step + 2.0 ** -7 * 2 * w)
        assert bool(((diff - dX[:, d].double()).abs() <= bound).all())


def test_same_result_every_time(h):
    X, W, labels, dloss = _case(700, 264, 9001, 8)
    first = h.sq_head_loss_grad(X, W, labels, dloss)
    other = pkg.Handle()
    for _ in range(3):
        for got, want in zip(other.sq_head_loss_grad(X, W, labels, dloss), first):
            assert torch.equal(got, want)


def test_other_stream_and_graph(h):
    X, W, labels, dloss = _case(300, 256, 2000, 9)
    want = h.sq_head_loss_grad(X, W, labels, dloss)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    X2, labels2 = torch.zeros_like(X), torch.full_like(labels, -100)
    with torch.cuda.stream(side):
        for got, w in zip(h.sq_head_loss_grad(X, W, labels, dloss), want):
            assert torch.equal(got, w)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = h.sq_head_loss_grad(X2, W, labels2, dloss)
    X2.copy_(X)
    labels2.copy_(labels)  # the number of labelled tokens is the replay's, not the capture's
    graph.replay()
    torch.cuda.synchronize()
    for got, w in zip(out, want):
        assert torch.equal(got, w)


def test_scratch_is_not_grown_in_a_capture():
    fresh = pkg.Handle()
    X, W, labels, dloss = _case(64, 64, 300, 2)
    out = [torch.empty(64, device="cuda"), torch.empty(64, device="cuda"), torch.empty_like(X)]
    fresh.sq_head_loss(X[:1], W[:8], labels[:1] * 0)  # the device is set up; this call's scratch is smaller
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(pkg.SQError, match="outside graph capture"):
            fresh.sq_head_loss_grad(X, W, labels, dloss, *out)
        X.add_(0)


def test_refusals(h):
    X, W, labels, dloss = _case(4, 64, 100, 1)
    with pytest.raises(ValueError, match="W must"):
        h.sq_head_loss(X, W.float(), labels)
    with pytest.raises(ValueError, match="W must"):
        h.sq_head_loss(X, W[:, :32], labels)
    with pytest.raises(ValueError, match="labels must"):
        h.sq_head_loss(X, W, labels.int())
    with pytest.raises(ValueError, match="dloss must"):
        h.sq_head_loss_grad(X, W, labels, dloss[:3])
    with pytest.raises(ValueError, match="labels is on"):
        h.sq_head_loss(X, W, labels.cpu())
    with pytest.raises(pkg.SQError, match="D="):
        h.sq_head_loss(X[:, :12].contiguous(), W[:, :12].contiguous(), labels)
    with pytest.raises(pkg.SQError, match="dX must not be X"):
        h.sq_head_loss_grad(X, W, labels, dloss, dX=X)


def test_loss_of_a_row_is_its_own(h):
    """Loss and log-sum-exp of a token have the same bits alone, among few and among many."""
    X, W, labels, _ = _case(1500, 264, 3001, 12, ignored=0.0)
    loss, lse = h.sq_head_loss(X, W, labels)
    for first, n in ((0, 1), (700, 7), (1000, 100), (3, 300)):
        for got, want in zip(h.sq_head_loss(X[first:first + n].contiguous(), W, labels[first:first + n].clone()), (loss, lse)):
            assert torch.equal(got, want[first:first + n])


def test_sums_of_a_large_vocabulary_in_chunks(h):
    """A vocabulary whose sums alone pass the scratch's bound: the rows go in several chunks."""
    T, D, V = 700, 8, 9_000_003
    X, W, labels, _ = _case(T, D, V, 13, ignored=0.1)
    loss, lse = h.sq_head_loss(X, W, labels)
    for t in (0, 255, 256, 399, 511, 512, 699):
        z = (X[t].double() @ W.double().t())
        want = torch.logsumexp(z, 0)
        if not 0 <= int(labels[t]) < V:
            assert lse[t] == 0 and loss[t] == 0
            continue
        # fp32 logits of 8 products, 64-term and 562,501-term sums of positive terms (256 + 35,157 roundings a path)
        tol = 1e-3
        assert abs(float(lse[t]) - float(want)) < tol
        assert abs(float(loss[t]) - float(want - z[labels[t]])) < tol


def test_inputs_written_just_before_the_call(h):
    """Calls of changing sizes back to back, every input written by a kernel right ahead of its call, give
    the bits of the same calls one by one."""
    cases = [_case(T, 520, 2003, 50 + i, ignored=0.3) for i, T in enumerate((300, 7, 64, 1, 700, 33, 256, 130))]
    want = []
    for case in cases:
        want.append([r.clone() for r in h.sq_head_loss_grad(*case)])
        torch.cuda.synchronize()
    X, W = torch.empty(700, 520, dtype=torch.bfloat16, device="cuda"), torch.empty_like(cases[0][1])
    labels, dloss = torch.empty(700, dtype=torch.int64, device="cuda"), torch.empty(700, device="cuda")
    got = []
    for _ in range(6):
        for x, w, y, d in cases:
            T = len(x)
            W.copy_(w), labels[:T].copy_(y), dloss[:T].copy_(d), X[:T].copy_(x)
            got.append([r.clone() for r in h.sq_head_loss_grad(X[:T], W, labels[:T], dloss[:T])])
    for i, results in enumerate(got):
        for r, first in zip(results, want[i % len(cases)]):
            assert torch.equal(r, first), i
