"""4-bit rows of an empty batch pass the argument checks, whatever their (absent) tensors point to."""
import ctypes

import pytest

import test_quant_abi as abi

pkg = abi.pkg
h = abi.h

NOTHING = {"R": 0, "codes": None, "scales": None}


@pytest.mark.parametrize("row_ws2", [None, abi.A])
def test_no_rows(h, row_ws2):
    """Without a GPU the next check, of the device, is the one that fails."""
    q = abi.rows({**NOTHING, "row_ws2": row_ws2})
    w, gw = pkg._lib._SqWeight(**abi.WEIGHT), pkg._lib._SqGroupedWeight(**abi.GROUPED, ws2=None)
    for name, args in (("sq_quantize", (q, 0, 1, None, None, None)), ("sq_dequantize", (q, None, None)),
                       ("sq_quant_fwd", (ctypes.byref(w), q, None, None)),
                       ("sq_grouped_quant_fwd", (ctypes.byref(gw), abi.A, abi.A, q, None, None)),
                       # no slots of some tokens: an empty tensor has no address
                       ("sq_quantize", (q, 7, 2, abi.A, None, None))):
        assert h.status_of(name, *args) != -1, (name, h.last_error())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [pkg.NVFP4, pkg.MXFP4])
def test_no_rows_on_a_gpu(fmt):
    import torch
    h = pkg.Handle()
    X = torch.ones(7, 64, dtype=torch.bfloat16, device="cuda")
    q = h.sq_quantize(fmt, X, slot_of=torch.empty(0, dtype=torch.int32, device="cuda"), k=2)
    assert q.R == 0 and h.sq_dequantize(q).shape == (0, 64)
    h.sq_sync()
