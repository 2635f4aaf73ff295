"""A training step of experts whose rows are kept in 4 bits, forward and backward with one weight object."""
import pytest
import torch

import quant_ref as ref
from test_gpu_quant_products import FORMATS, close, decoded, h, rows, weight  # noqa: F401

pkg = pytest.importorskip("paper_2609_04526_gb300")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts, N, K", [([3, 0, 70, 1], 136, 544), ([900, 0, 300, 1800], 2056, 1056)])
def test_experts_step_from_kept_rows(h, fmt, counts, N, K):  # noqa: F811
    """Forward in 4 bits, gradients from the kept codes, against their formulas in 64 bits. The tensor scales are what
    the forward takes: a device tensor (NVFP4), none (MXFP4)."""
    g = torch.Generator(device="cuda").manual_seed(sum(counts))
    E, R, B = len(counts), sum(counts), ref.BLOCK[fmt]
    codes, scales = weight(g, fmt, (E, N), K)
    ws2 = None if fmt == pkg.MXFP4 else torch.rand(E, generator=g, device="cuda") + 0.1
    w = pkg.GroupedWeight(fmt, E, N, K, codes, scales, ws2)
    offsets = torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], device="cuda")
    off = offsets.tolist()
    q = rows(g, h, fmt, R, K)
    dY = torch.randn(R, N, generator=g, device="cuda").bfloat16()
    Y = h.sq_grouped_quant_fwd(w, offsets, q)
    kept = h.sq_dequantize(q)
    grad = h.sq_grouped_scale_grad(w, off, kept, dY)
    dX = h.sq_grouped_bwd_dx(w, off, dY)
    h.sq_sync()
    x, dy = decoded(q).cuda(), dY.double()
    for e in range(E):
        part = slice(off[e], off[e + 1])
        if not counts[e]:
            assert (grad[e] == 0).all()
            continue
        s2 = 1.0 if ws2 is None else float(ws2[e])
        W = ref.values(fmt, codes[e].cpu(), scales[e].cpu()).cuda() * s2
        close(Y[part], x[part], W, f"expert {e}")
        c = ref.values(fmt, codes[e].cpu(), torch.full_like(scales[e], 0x38 if fmt == pkg.NVFP4 else 127).cpu()).cuda()
        want = ((dy[part].T @ x[part]) * c).view(N, K // B, B).sum(2)
        size = ((dy[part].abs().T @ x[part].abs()) * c.abs()).view(N, K // B, B).sum(2)
        # fp32 sums of steps of 16 rows, then of a block's products: each loses at most 2^-22 of what went into it
        assert ((grad[e].double() - want).abs() <= (counts[e] / 16 + 40) * 2.0 ** -22 * size).all(), e
        dx, dx_size = dy[part] @ W, dy[part].abs() @ W.abs()
        assert ((dX[part].double() - dx).abs() <= 2.0 ** -8 * dx.abs() + (N / 16 + 8) * 2.0 ** -22 * dx_size).all(), e
