"""Routing and head-loss calls on tensors that are not on the GPU are refused on the host."""
import pytest
import torch

pkg = pytest.importorskip("paper_2609_04526_gb300")


@pytest.fixture(scope="module")
def h():
    from paper_2609_04526_gb300 import build
    build.build()
    return pkg.Handle()


T, E, K, D, V = 4, 16, 2, 64, 100
BF16 = torch.bfloat16
TENSORS = {
    "logits": torch.zeros(T, E), "experts": torch.zeros(T, K, dtype=torch.int32), "weights": torch.zeros(T, K),
    "row_of": torch.zeros(T, K, dtype=torch.int32), "slot_of": torch.zeros(T * K, dtype=torch.int32),
    "X": torch.zeros(T, D, dtype=BF16), "rows": torch.zeros(T * K, D, dtype=BF16), "W": torch.zeros(V, D, dtype=BF16),
    "labels": torch.zeros(T, dtype=torch.int64), "dloss": torch.zeros(T), "valid": torch.ones(T + 1, dtype=torch.bool)[1:],
}


@pytest.mark.parametrize("name, args", [
    ("sq_route", ("logits", K)), ("sq_route", ("logits", K, True, "valid")), ("sq_route_grad", ("logits", "experts", "weights")),
    ("sq_sort_tokens", ("experts", E)), ("sq_dispatch", ("X", "row_of", "slot_of")), ("sq_dispatch_grad", ("rows", "row_of")),
    ("sq_combine", ("rows", "row_of", "weights")), ("sq_combine_grad", ("X", "rows", "row_of", "slot_of", "weights")),
    ("sq_head_loss", ("X", "W", "labels")), ("sq_head_loss_grad", ("X", "W", "labels", "dloss")),
])
def test_host_tensors_are_refused(h, name, args):
    with pytest.raises(ValueError, match="is on cpu, not on the current CUDA device"):
        getattr(h, name)(*[TENSORS[a] if isinstance(a, str) else a for a in args])
