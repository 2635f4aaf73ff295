"""Routing and loss of slices that start on an element of a larger tensor."""
import pytest
import torch

pytestmark = pytest.mark.gpu
pkg = pytest.importorskip("paper_2609_04526_gb300")


@pytest.fixture(scope="module")
def h():
    return pkg.Handle()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def test_next_token_loss(h):
    """Rows up to the last but one, labels and weights from the second on; and one sequence of several of odd
    length."""
    B, S, D, V = 3, 37, 64, 300
    X = torch.randn(B, S, D, generator=_gen(1), device="cuda").bfloat16()
    W = torch.randn(V, D, generator=_gen(2), device="cuda").bfloat16()
    labels = torch.randint(V, (B, S), generator=_gen(3), device="cuda")
    dloss = torch.rand(B, S, generator=_gen(4), device="cuda")
    for b in range(B):
        x, y, g = X[b, :-1], labels[b, 1:], dloss[b, 1:]
        assert y.is_contiguous() and (y.data_ptr() % 16 or g.data_ptr() % 16)
        want = h.sq_head_loss_grad(x, W, y.clone(), g.clone())
        for got, w in zip(h.sq_head_loss_grad(x, W, y, g), want):
            assert torch.equal(got, w)
        assert torch.equal(h.sq_head_loss(x, W, y)[0], want[0])


@pytest.mark.parametrize("stream", [None, "side"])
@pytest.mark.parametrize("dtype", [torch.uint8, torch.bool])
def test_one_sequence_of_a_batch(h, stream, dtype):
    """A sequence's mask, experts and weights out of tensors over a batch of odd length."""
    B, S, E, k, D = 4, 37, 16, 3, 64
    if stream:
        stream = torch.cuda.Stream()
    z = torch.randn(B, S, E, generator=_gen(5), device="cuda")
    valid = (torch.rand(B, S, generator=_gen(6), device="cuda") < 0.7).to(dtype)
    X = torch.randn(B, S, D, generator=_gen(7), device="cuda").bfloat16()
    experts = torch.empty(B, S, k, dtype=torch.int32, device="cuda")
    row_of = torch.empty_like(experts)
    weights, dweights = torch.empty(B, S, k, device="cuda"), torch.empty(B, S, k, device="cuda")
    torch.cuda.synchronize()
    for b in range(B):
        def step(mask, experts, weights, row_of, dweights):
            kw = dict(stream=stream)
            h.sq_route(z[b], k, valid=mask, experts=experts, weights=weights, **kw)
            offsets, _, slot_of = h.sq_sort_tokens(experts, E, row_of=row_of, **kw)
            Xs = h.sq_dispatch(X[b], row_of, slot_of, **kw)
            Y = h.sq_combine(Xs, row_of, weights, **kw)
            dYs, _ = h.sq_combine_grad(Y, Xs, row_of, slot_of, weights, dweights=dweights, **kw)
            dX = h.sq_dispatch_grad(dYs, row_of, **kw)
            dz = h.sq_route_grad(z[b], experts, dweights, **kw)
            torch.cuda.synchronize()
            return [t.clone() for t in (experts, weights, row_of, dweights, offsets, slot_of, Xs, Y, dYs, dX, dz)]

        want = step(valid[b].clone(), experts[b].clone(), weights[b].clone(), row_of[b].clone(), dweights[b].clone())
        for got, w in zip(step(valid[b], experts[b], weights[b], row_of[b], dweights[b]), want):
            assert torch.equal(got, w)
