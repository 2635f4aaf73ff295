"""The scale gradient of a step that keeps its rows in 4 bits, against the difference that a moved scale makes."""
import pytest
import torch

import quant_ref as ref
from test_gpu_quant_products import FORMATS, h, weight  # noqa: F401

pkg = pytest.importorskip("paper_2609_04526_gb300")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("R, N, K", [(70, 136, 544), (900, 264, 1056), (5000, 2056, 544)])
def test_scale_gradient_by_a_difference(h, fmt, R, N, K):  # noqa: F811
    """One feature's weight is one block, so that its outputs are that block's alone, and the gradient that comes in is
    those outputs: a moved scale then changes the loss by far more than the outputs' rounding."""
    g = torch.Generator(device="cuda").manual_seed(R + 1)
    B, n, b = ref.BLOCK[fmt], 5, 1
    codes, scales = weight(g, fmt, (N,), K)
    codes[n, : b * B // 2] = 0
    codes[n, (b + 1) * B // 2:] = 0
    ws2 = 1.0 if fmt == pkg.MXFP4 else 0.031
    X = torch.randn(R, K, generator=g, device="cuda").bfloat16()
    q = h.sq_quantize(fmt, X)
    w = pkg.QuantWeight(fmt, N, K, codes, scales, ws2)
    before = h.sq_quant_fwd(w, q)
    dY = torch.randn(R, N, generator=g, device="cuda").bfloat16()
    dY[:, n] = before[:, n]
    kept = h.sq_dequantize(q)
    grad = h.sq_scale_grad(w, kept, dY)
    moved = scales.clone()
    moved[n, b] += 16 if fmt == pkg.NVFP4 else 2  # four times as large
    step = float((ref.scale_values(fmt, moved.cpu()) - ref.scale_values(fmt, scales.cpu()))[n, b]) * ws2
    after = h.sq_quant_fwd(pkg.QuantWeight(fmt, N, K, codes, moved, ws2), q)
    h.sq_sync()
    dy = dY.double()
    change = ((after.double() - before.double()) * dy)[:, n].sum()
    # both outputs are rounded to bf16, by at most 2^-8 of them; the gradient's fp32 sums lose at most 2^-22 a step of
    # what goes into them
    slack = (2.0 ** -8 * (after.double().abs() + before.double().abs()) * dy.abs())[:, n].sum()
    block = slice(b * B, (b + 1) * B)
    c = ref.E2M1.cuda()[(ref.unpack(codes[n:n + 1])[0, block] % 8)]
    size = (dy[:, n].abs() @ kept.double()[:, block].abs() * c).sum()
    slack += abs(step) * (R / 16 + 40) * 2.0 ** -22 * size
    assert abs(change) > 50 * slack  # 3 of 5 units, each 2^-8: a gradient of zero, or of the wrong sign, is far outside
    assert abs(change - step * grad[n, b].double()) <= slack
    others = torch.arange(N, device="cuda") != n
    assert torch.equal(before[:, others], after[:, others])
