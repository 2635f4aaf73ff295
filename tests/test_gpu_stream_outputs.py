"""Outputs that a call allocates belong to the stream it is given."""
import pytest
import torch

pytestmark = pytest.mark.gpu
pkg = pytest.importorskip("paper_2609_04526_gb300")

T, E, K, D, V = 512, 16, 4, 1024, 2048
BF16 = torch.bfloat16


def _rows(n, seed):
    return torch.randn(n, D, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


def _calls(h):
    """(call with a stream, shape and type of the output that it allocates)."""
    z = torch.randn(T, E, device="cuda")
    experts, weights = h.sq_route(z, K)
    _, row_of, slot_of = h.sq_sort_tokens(experts, E)
    X, rows, W = _rows(T, 1), _rows(T * K, 2), _rows(V, 3)
    labels = torch.arange(T, device="cuda")
    dloss = torch.ones(T, device="cuda")
    return {
        "sq_route": (lambda s: h.sq_route(z, K, stream=s), (T, K), torch.int32),
        "sq_route_grad": (lambda s: h.sq_route_grad(z, experts, weights, stream=s), (T, E), torch.float32),
        "sq_sort_tokens": (lambda s: h.sq_sort_tokens(experts, E, stream=s), (T, K), torch.int32),
        "sq_dispatch": (lambda s: h.sq_dispatch(X, row_of, slot_of, stream=s), (T * K, D), BF16),
        "sq_dispatch_grad": (lambda s: h.sq_dispatch_grad(rows, row_of, stream=s), (T, D), BF16),
        "sq_combine": (lambda s: h.sq_combine(rows, row_of, weights, stream=s), (T, D), BF16),
        "sq_combine_grad": (lambda s: h.sq_combine_grad(X, rows, row_of, slot_of, weights, stream=s), (T * K, D), BF16),
        "sq_head_loss": (lambda s: h.sq_head_loss(X, W, labels, stream=s), (T,), torch.float32),
        "sq_head_loss_grad": (lambda s: h.sq_head_loss_grad(X, W, labels, dloss, stream=s), (T, D), BF16),
    }


@pytest.mark.parametrize("name", ["sq_route", "sq_route_grad", "sq_sort_tokens", "sq_dispatch", "sq_dispatch_grad", "sq_combine",
                                  "sq_combine_grad", "sq_head_loss", "sq_head_loss_grad"])
def test_memory_that_another_stream_still_reads(name):
    """A tensor freed on the current stream while work queued there has yet to read it: a call on another stream
    does not get its memory."""
    h = pkg.Handle()
    call, shape, dtype = _calls(h)[name]
    side = torch.cuda.Stream()
    call(side)  # scratch and kernels are set up
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    freed = [torch.full(shape, 77, dtype=dtype, device="cuda") for _ in range(4)]
    copies = [torch.empty_like(f) for f in freed]
    torch.cuda.synchronize()
    torch.cuda._sleep(int(2e8))  # 0.1 s, in which the copies wait
    for c, f in zip(copies, freed):
        c.copy_(f)
    del f, freed
    out = call(side)
    torch.cuda.synchronize()
    for c in copies:
        assert bool((c == 77).all())
    del out
