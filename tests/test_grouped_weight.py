"""What the binding makes of a grouped weight's tensor scales and offsets (no GPU)."""
import ctypes

import pytest
import torch

pkg = pytest.importorskip("paper_2609_04526_gb300")

E, N, K = 3, 16, 64


@pytest.fixture(scope="module")
def h():
    from paper_2609_04526_gb300 import build
    build.build()
    return pkg.Handle()


def weight(fmt, ws2):
    return pkg.GroupedWeight(fmt, E, N, K, torch.zeros(E, N, K // 2, dtype=torch.uint8),
                             torch.zeros(E, N, K // pkg.BLOCK[fmt], dtype=torch.uint8), ws2)


def test_mxfp4_experts_without_tensor_scales():
    """None, as the 4-bit forward takes it, is every other grouped call's too."""
    w = weight(pkg.MXFP4, None)
    c, _ = w._c()
    assert not c.ws2
    assert w.expert(1).ws2 == 1.0


def test_nvfp4_experts_without_tensor_scales_are_refused(h):
    w = weight(pkg.NVFP4, None)
    c, _ = w._c()
    off = (ctypes.c_int64 * (E + 1))()
    assert h.status_of("sq_grouped_fwd", ctypes.byref(c), off, None, None, None) == -1
    assert "ws2" in h.last_error()


@pytest.mark.parametrize("ws2", [[0.5, 0.25, 2.0], torch.tensor([0.5, 0.25, 2.0])])
def test_nvfp4_tensor_scales(ws2):
    w = weight(pkg.NVFP4, ws2)
    c, keep = w._c()
    assert [c.ws2[e] for e in range(E)] == [0.5, 0.25, 2.0] and len(keep) == E
    assert w.expert(2).ws2 == 2.0


class Reads(torch.utils._python_dispatch.TorchDispatchMode):
    """Counts single elements read from tensors: each is a copy and a wait where the tensor is on a device."""
    count = 0

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        self.count += func is torch.ops.aten._local_scalar_dense.default
        return func(*args, **(kwargs or {}))


def test_tensors_are_read_at_once():
    """Tensor scales and offsets that are tensors come to the host as a whole, not value by value."""
    w = weight(pkg.NVFP4, torch.tensor([0.5, 0.25, 2.0]))
    with Reads() as reads:
        c, _ = w._c()
        _, vals = pkg._lib._offsets(torch.tensor([0, 4, 4, 9]), E)
    assert reads.count == 0
    assert [c.ws2[e] for e in range(E)] == [0.5, 0.25, 2.0] and vals == [0, 4, 4, 9]
