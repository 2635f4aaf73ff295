"""Argument checks of 4-bit rows and their products, made before any CUDA call."""
import ctypes

import pytest
import torch

pkg = pytest.importorskip("paper_2609_04526_gb300")

A = 0x10000  # aligned, never dereferenced: every call here fails its checks


@pytest.fixture(scope="module")
def h():
    from paper_2609_04526_gb300 import build
    build.build()
    return pkg.Handle()


ROWS = dict(fmt=0, K=64, R=4, codes=A, scales=A, ws2=1.0, row_ws2=A)
WEIGHT = dict(fmt=0, N=16, K=64, codes=A, scales=A, ws2=1.0)
GROUPED = dict(fmt=0, E=2, N=16, K=64, codes=A, scales=A)


def rows(change):
    return ctypes.byref(pkg._lib._SqRows(**{**ROWS, **change}))


BAD_ROWS = [({"fmt": 2}, "format"), ({"K": 0}, "K="), ({"K": 48}, "K="), ({"R": -1}, "R="), ({"R": 1 << 31}, "R="),
            ({"codes": None}, "codes"), ({"codes": A + 8}, "codes"), ({"scales": A + 2}, "scales"), ({"row_ws2": A + 2}, "row_ws2"),
            ({"ws2": 0.5}, "row_ws2"), ({"fmt": 1}, "row_ws2"), ({"ws2": 0.0, "row_ws2": None}, "ws2"),
            ({"ws2": float("nan"), "row_ws2": None}, "ws2"), ({"fmt": 1, "ws2": 2.0, "row_ws2": None}, "ws2")]


@pytest.mark.parametrize("change, why", BAD_ROWS)
def test_rows_are_checked_everywhere(h, change, why):
    q = rows(change)
    w, gw = pkg._lib._SqWeight(**WEIGHT), pkg._lib._SqGroupedWeight(**GROUPED, ws2=None)
    for name, args in (("sq_quantize", (q, change.get("R", 4), 1, A, None, None)), ("sq_dequantize", (q, A, None)),
                       ("sq_quant_fwd", (ctypes.byref(w), q, A, None)),
                       ("sq_grouped_quant_fwd", (ctypes.byref(gw), A, A, q, A, None))):
        assert h.status_of(name, *args) == -1, name
        assert why in h.last_error(), (name, h.last_error())


@pytest.mark.parametrize("change, T, k, X, slot_of, why", [
    ({}, 5, 1, A, None, "slot_of"), ({}, -1, 1, A, A, "M="), ({}, 4, 0, A, A, "k="), ({}, 4, 33, A, A, "k="),
    ({}, 1 << 30, 2, A, A, "T="), ({}, 4, 1, A, A + 2, "slot_of"), ({}, 4, 1, None, None, "X"), ({}, 4, 1, A + 8, None, "X"),
    ({"row_ws2": None, "ws2": 2.0 ** -127}, 4, 1, A, None, "ws2"), ({"row_ws2": None, "ws2": 2.0 ** 127}, 4, 1, A, None, "ws2")])
def test_quantize_refuses(h, change, T, k, X, slot_of, why):
    assert h.status_of("sq_quantize", rows(change), T, k, X, slot_of, None) == -1
    assert why in h.last_error()


@pytest.mark.parametrize("change, row_change, Y, why", [
    ({"N": 12}, {}, A, "N="), ({"K": 33}, {}, A, "K="), ({"scales": None}, {}, A, "scales"), ({"codes": A + 1}, {}, A, "codes"),
    ({"K": 128}, {}, A, "K=128"), ({"fmt": 1}, {}, A, "format"), ({}, {}, A + 8, "Y"), ({}, {}, None, "Y")])
def test_products_refuse(h, change, row_change, Y, why):
    w = pkg._lib._SqWeight(**{**WEIGHT, **change})
    assert h.status_of("sq_quant_fwd", ctypes.byref(w), rows(row_change), Y, None) == -1
    assert why in h.last_error()
    g = pkg._lib._SqGroupedWeight(**{**GROUPED, **change}, ws2=None)
    ws2 = None if change.get("fmt") == 1 else A
    assert h.status_of("sq_grouped_quant_fwd", ctypes.byref(g), ws2, A, rows(row_change), Y, None) == -1
    assert why in h.last_error()


@pytest.mark.parametrize("change, ws2, offsets, why", [
    ({"E": 0}, A, A, "E="), ({"E": 1025}, A, A, "E="), ({}, None, A, "ws2"), ({}, A + 2, A, "ws2"), ({"fmt": 1}, A, A, "ws2"),
    ({}, A, None, "offsets"), ({}, A, A + 4, "offsets")])
def test_experts_refuse(h, change, ws2, offsets, why):
    g = pkg._lib._SqGroupedWeight(**{**GROUPED, **change}, ws2=None)
    row = {"fmt": 1, "row_ws2": None} if change.get("fmt") == 1 else {}
    assert h.status_of("sq_grouped_quant_fwd", ctypes.byref(g), ws2, offsets, rows(row), A, None) == -1
    assert why in h.last_error()
    assert h.status_of("sq_grouped_quant_fwd", None, A, A, rows({}), A, None) == -1


def test_binding_checks_tensors(h):
    """Shapes, types and devices are refused before a pointer leaves Python (no GPU is needed for that)."""
    X = torch.zeros(4, 64, dtype=torch.bfloat16)
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    q = pkg.QuantRows(0, 4, 64, u8(4, 32), u8(4, 4), 1.0, torch.zeros(4))
    with pytest.raises(ValueError, match="row_ws2"):
        h.sq_quantize(0, X, ws2=0.5, out=q)
    with pytest.raises(ValueError, match="out holds"):
        h.sq_quantize(0, X[:3], out=q)
    with pytest.raises(ValueError, match="X must be"):
        h.sq_quantize(0, X.float(), out=q)
    with pytest.raises(ValueError, match="X must be"):
        h.sq_quantize(0, X.t().contiguous().t(), out=q)
    with pytest.raises(ValueError, match="codes must be"):
        h.sq_dequantize(pkg.QuantRows(0, 4, 64, u8(4, 64), u8(4, 4)), X=X)
    with pytest.raises(ValueError, match="CUDA device"):
        h.sq_dequantize(q, X=X)


def test_refused_rows_keep_their_scale(h):
    """A refused quantisation into existing rows leaves their scale as it was: their codes are still under it."""
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    q = pkg.QuantRows(0, 4, 64, u8(4, 32), u8(4, 4), 0.25)
    with pytest.raises(ValueError, match="X must be"):
        h.sq_quantize(0, torch.zeros(4, 64), ws2=0.5, out=q)
    assert q.ws2 == 0.25


def test_products_refuse_rows_elsewhere_before_their_output_is_made(h):
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    q = pkg.QuantRows(1, 4, 64, u8(4, 32), u8(4, 2))
    with pytest.raises(ValueError, match="CUDA device"):
        h.sq_dequantize(q)
    with pytest.raises(ValueError, match="CUDA device"):
        h.sq_quant_fwd(pkg.QuantWeight(1, 16, 64, u8(16, 32), u8(16, 2), 1.0), q)
    with pytest.raises(ValueError, match="CUDA device"):
        h.sq_grouped_quant_fwd(pkg.GroupedWeight(1, 2, 16, 64, u8(2, 16, 32), u8(2, 16, 2), None),
                               torch.zeros(3, dtype=torch.int64), q)
