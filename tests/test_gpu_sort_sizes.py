"""The sort by expert at the sizes where its launches change: eight warps or 32, one CTA or several."""
import numpy as np
import pytest
import torch

import step_ref as ref

pytestmark = pytest.mark.gpu
pkg = pytest.importorskip("paper_2609_04526_gb300")


@pytest.mark.parametrize("n", [1023, 1024, 1025, 4095, 4096, 4097, 6143, 6144, 6145])
@pytest.mark.parametrize("E", [1, 16, 128, 129, 1024])
def test_sort(n, E):
    h = pkg.Handle()
    e = torch.randint(-1, E + 1, (n, 1), generator=torch.Generator(device="cuda").manual_seed(n + E), device="cuda", dtype=torch.int32)
    got = h.sq_sort_tokens(e, E)
    h.sq_sync()
    for x, want in zip(got, ref.sort(e.cpu().numpy(), E)):
        assert np.array_equal(x.cpu().numpy(), want)
