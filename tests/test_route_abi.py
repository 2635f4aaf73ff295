"""Argument checks of the routing and head-loss entry points, made before any CUDA call."""
import pytest

pkg = pytest.importorskip("paper_2609_04526_gb300")

A = 0x10000  # aligned, never dereferenced: every call here fails its checks


@pytest.fixture(scope="module")
def h():
    from paper_2609_04526_gb300 import build
    build.build()
    return pkg.Handle()


ROUTE = dict(T=4, E=16, k=2, bf16=0, logits=A, valid=None, norm=1, experts=A, weights=A, stream=None)
ROUTE_GRAD = dict(T=4, E=16, k=2, bf16=0, logits=A, experts=A, dweights=A, norm=1, dlogits=A, stream=None)
SORT = dict(n=8, E=16, experts=A, offsets=A, row_of=A, slot_of=A, stream=None)
DISPATCH = dict(T=4, k=2, D=64, R=8, X=A, row_of=A, slot_of=A, Xs=A, stream=None)
DISPATCH_GRAD = dict(T=4, k=2, D=64, R=8, dXs=A, row_of=A, dX=A, stream=None)
COMBINE = dict(T=4, k=2, D=64, R=8, Ys=A, row_of=A, weights=A, Y=A, stream=None)
COMBINE_GRAD = dict(T=4, k=2, D=64, R=8, dY=A, Ys=A, row_of=A, slot_of=A, weights=A, dYs=A, dweights=A, stream=None)
LOSS = dict(T=4, D=64, V=100, X=A, W=A, labels=A, loss=A, lse=A, stream=None)
LOSS_GRAD = dict(T=4, D=64, V=100, X=A, W=A, labels=A, dloss=A, loss=A, lse=A, dX=A + 4096, stream=None)


@pytest.mark.parametrize("name, base, change, why", [
    ("sq_route", ROUTE, {"T": -1}, "T="), ("sq_route", ROUTE, {"T": 1 << 30, "k": 2}, "T="),
    ("sq_route", ROUTE, {"E": 0}, "E="), ("sq_route", ROUTE, {"E": 1025}, "E="),
    ("sq_route", ROUTE, {"k": 0}, "k="), ("sq_route", ROUTE, {"k": 17}, "k="), ("sq_route", ROUTE, {"E": 64, "k": 33}, "k="),
    ("sq_route", ROUTE, {"logits": None}, "logits"), ("sq_route", ROUTE, {"logits": A + 4}, "logits"),
    ("sq_route", ROUTE, {"valid": A + 1}, "valid"), ("sq_route", ROUTE, {"weights": None}, "weights"),
    ("sq_route_grad", ROUTE_GRAD, {"dweights": None}, "dweights"), ("sq_route_grad", ROUTE_GRAD, {"dlogits": A + 8}, "dlogits"),
    ("sq_route_grad", ROUTE_GRAD, {"experts": None}, "experts"), ("sq_route_grad", ROUTE_GRAD, {"k": -1}, "k="),
    ("sq_sort_tokens", SORT, {"n": -1}, "n="), ("sq_sort_tokens", SORT, {"n": 1 << 31}, "n="),
    ("sq_sort_tokens", SORT, {"E": 1025}, "E="), ("sq_sort_tokens", SORT, {"offsets": None}, "offsets"),
    ("sq_sort_tokens", SORT, {"n": 0, "offsets": A + 8}, "offsets"), ("sq_sort_tokens", SORT, {"row_of": None}, "row_of"),
    ("sq_dispatch", DISPATCH, {"D": 12}, "D="), ("sq_dispatch", DISPATCH, {"D": 0}, "D="), ("sq_dispatch", DISPATCH, {"k": 33}, "k="),
    ("sq_dispatch", DISPATCH, {"R": 9}, "R="), ("sq_dispatch", DISPATCH, {"R": -1}, "R="), ("sq_dispatch", DISPATCH, {"T": -4}, "T="),
    ("sq_dispatch", DISPATCH, {"T": 1 << 26, "D": 1 << 14}, "too many"), ("sq_dispatch", DISPATCH, {"Xs": None}, "Xs"),
    ("sq_dispatch", DISPATCH, {"slot_of": A + 4}, "slot_of"),
    ("sq_dispatch_grad", DISPATCH_GRAD, {"dX": None}, "dX"), ("sq_dispatch_grad", DISPATCH_GRAD, {"dXs": None}, "dXs"),
    ("sq_combine", COMBINE, {"weights": None}, "weights"), ("sq_combine", COMBINE, {"Y": A + 2}, "Y"),
    ("sq_combine_grad", COMBINE_GRAD, {"dY": None}, "dY"), ("sq_combine_grad", COMBINE_GRAD, {"dYs": A + 2}, "dYs"),
    ("sq_combine_grad", COMBINE_GRAD, {"dweights": None}, "dweights"), ("sq_combine_grad", COMBINE_GRAD, {"R": 100}, "R="),
    ("sq_head_loss", LOSS, {"T": -1}, "M="), ("sq_head_loss", LOSS, {"D": 4}, "D="), ("sq_head_loss", LOSS, {"D": 65544}, "D="),
    ("sq_head_loss", LOSS, {"V": 0}, "V="), ("sq_head_loss", LOSS, {"V": (1 << 24) + 1}, "V="),
    ("sq_head_loss", LOSS, {"loss": None, "lse": None}, "NULL"), ("sq_head_loss", LOSS, {"W": A + 2}, "W"),
    ("sq_head_loss", LOSS, {"labels": None}, "labels"), ("sq_head_loss", LOSS, {"lse": A + 4}, "lse"),
    ("sq_head_loss_grad", LOSS_GRAD, {"dloss": None}, "dloss"), ("sq_head_loss_grad", LOSS_GRAD, {"dX": None}, "dX"),
    ("sq_head_loss_grad", LOSS_GRAD, {"dX": A}, "dX must not be X"), ("sq_head_loss_grad", LOSS_GRAD, {"loss": A + 4}, "loss"),
])
def test_refusals(h, name, base, change, why):
    assert h.status_of(name, *{**base, **change}.values()) == -1
    assert why in h.last_error()


@pytest.mark.parametrize("name, base", [("sq_route", ROUTE), ("sq_route_grad", ROUTE_GRAD), ("sq_sort_tokens", SORT),
                                        ("sq_dispatch", DISPATCH), ("sq_dispatch_grad", DISPATCH_GRAD), ("sq_combine", COMBINE),
                                        ("sq_combine_grad", COMBINE_GRAD), ("sq_head_loss", LOSS), ("sq_head_loss_grad", LOSS_GRAD)])
def test_null_handle(h, name, base):
    assert getattr(pkg.load(), name)(None, *base.values()) == -1
