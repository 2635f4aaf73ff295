"""An empty batch passes the argument checks, whatever its (absent) tensors point to."""
import pytest

import test_route_abi as abi

pkg = abi.pkg
h = abi.h


@pytest.mark.parametrize("name, base", [
    ("sq_route", {**abi.ROUTE, "T": 0}), ("sq_route_grad", {**abi.ROUTE_GRAD, "T": 0}),
    ("sq_dispatch", {**abi.DISPATCH, "T": 0, "R": 0}), ("sq_dispatch_grad", {**abi.DISPATCH_GRAD, "T": 0, "R": 0}),
    ("sq_combine", {**abi.COMBINE, "T": 0, "R": 0}), ("sq_combine_grad", {**abi.COMBINE_GRAD, "T": 0, "R": 0}),
    ("sq_head_loss", {**abi.LOSS, "T": 0}), ("sq_head_loss_grad", {**abi.LOSS_GRAD, "T": 0}),
])
def test_no_tokens(h, name, base):
    """Without a GPU the next check, of the device, is the one that fails."""
    nothing = {key: None if value in (abi.A, abi.A + 4096) else value for key, value in base.items()}
    assert h.status_of(name, *nothing.values()) != -1


@pytest.mark.gpu
def test_no_tokens_on_a_gpu():
    import torch
    h = pkg.Handle()
    bf16 = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    labels = torch.zeros(0, dtype=torch.int64, device="cuda")
    loss, lse = h.sq_head_loss(bf16(0, 64), bf16(100, 64), labels)
    assert loss.shape == lse.shape == (0,)
    assert [t.shape[0] for t in h.sq_head_loss_grad(bf16(0, 64), bf16(100, 64), labels, lse)] == [0, 0, 0]
    experts, weights = h.sq_route(torch.zeros(0, 16, device="cuda"), 2)
    offsets, row_of, slot_of = h.sq_sort_tokens(experts, 16)
    assert not offsets.any()
    Xs = h.sq_dispatch(bf16(0, 64), row_of, slot_of)
    assert Xs.shape == (0, 64) and h.sq_combine(Xs, row_of, weights).shape == (0, 64)
    assert [t.shape[0] for t in h.sq_combine_grad(bf16(0, 64), Xs, row_of, slot_of, weights)] == [0, 0]
    assert h.sq_dispatch_grad(Xs, row_of).shape == (0, 64)
    assert h.sq_route_grad(torch.zeros(0, 16, device="cuda"), experts, weights).shape == (0, 16)
    h.sq_sync()
