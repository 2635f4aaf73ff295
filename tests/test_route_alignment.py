"""Alignment checks of the tensors that routing and head loss take by elements, made before any CUDA call."""
import pytest

import test_route_abi as abi

pkg = abi.pkg
h = abi.h
A = abi.A


@pytest.mark.parametrize("name, base, change, why", [
    ("sq_route", abi.ROUTE, {"experts": A + 2}, "experts must be non-NULL and 4-byte"),
    ("sq_route", abi.ROUTE, {"weights": A + 1}, "weights must be non-NULL and 4-byte"),
    ("sq_route_grad", abi.ROUTE_GRAD, {"dweights": A + 2}, "dweights must"),
    ("sq_sort_tokens", abi.SORT, {"row_of": A + 3}, "row_of must"),
    ("sq_combine", abi.COMBINE, {"row_of": A + 2}, "row_of must"),
    ("sq_head_loss", abi.LOSS, {"labels": A + 4}, "labels must be non-NULL and 8-byte"),
    ("sq_head_loss_grad", abi.LOSS_GRAD, {"dloss": A + 2}, "dloss must be non-NULL and 4-byte"),
])
def test_refusals(h, name, base, change, why):
    assert h.status_of(name, *{**base, **change}.values()) == -1
    assert why in h.last_error()
