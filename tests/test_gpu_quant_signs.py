"""Rows whose own scale bytes are negative (their format allows it; sq_quantize writes none), in every kernel."""
import pytest
import torch

import quant_ref as ref
from test_gpu_quant_products import close, decoded, h, weight  # noqa: F401

pkg = pytest.importorskip("paper_2609_04526_gb300")
pytestmark = pytest.mark.gpu


def signed_rows(g, R, K, share):
    """NVFP4 rows of random codes, `share` of their scale bytes negative, every row under a scale of its own."""
    codes, scales = weight(g, pkg.NVFP4, (R,), K)
    signs = torch.rand(scales.shape, generator=g, device="cuda") < share
    row = torch.exp2(torch.randint(-3, 4, (R,), generator=g, device="cuda").float())
    return pkg.QuantRows(pkg.NVFP4, R, K, codes, scales + 128 * signs.to(torch.uint8), 1.0, row)


# few-token kernel with scale bytes by TMA and by warps; pair kernel with stages of one and two slices; tall tiles
@pytest.mark.parametrize("share", [0.5, 0.001])
@pytest.mark.parametrize("R, N, K", [(3, 136, 1024), (100, 264, 800), (1900, 2056, 2048), (5000, 2056, 288), (3000, 4104, 2720),
                                     (2048, 4096, 2912)])
@pytest.mark.parametrize("both", [False, True])
def test_rows_with_negative_scales(h, R, N, K, share, both):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(R + K)
    codes, scales = weight(g, pkg.NVFP4, (N,), K, signs=both)
    q = signed_rows(g, R, K, share)
    Y = h.sq_quant_fwd(pkg.QuantWeight(pkg.NVFP4, N, K, codes, scales, 0.0173), q)
    back = h.sq_dequantize(q)
    h.sq_sync()
    x = decoded(q)
    assert torch.equal(back.double().cpu(), x)  # powers of two: nothing is rounded
    close(Y, x, ref.values(pkg.NVFP4, codes.cpu(), scales.cpu()) * float(torch.tensor(0.0173)))


@pytest.mark.parametrize("counts, N, K", [([3, 0, 70, 40], 200, 544), ([5, 129, 64, 250], 136, 1024),
                                          ([900, 0, 1, 224, 225, 448, 3200], 1032, 544)])
def test_experts_rows_with_negative_scales(h, counts, N, K):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(K)
    E, R = len(counts), sum(counts)
    codes, scales = weight(g, pkg.NVFP4, (E, N), K)
    q = signed_rows(g, R, K, 0.3)
    ws2 = torch.rand(E, generator=g, device="cuda") + 0.1
    offsets = torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], device="cuda")
    Y = h.sq_grouped_quant_fwd(pkg.GroupedWeight(pkg.NVFP4, E, N, K, codes, scales, ws2), offsets, q)
    h.sq_sync()
    x, off = decoded(q), offsets.tolist()
    for e in range(E):
        if counts[e]:
            close(Y[off[e]:off[e + 1]], x[off[e]:off[e + 1]], ref.values(pkg.NVFP4, codes[e].cpu(), scales[e].cpu()) * float(ws2[e]))


@pytest.mark.parametrize("fmt", [pkg.NVFP4, pkg.MXFP4])
@pytest.mark.parametrize("per, N, K", [(1, 136, 544), (9, 264, 1056)])
def test_as_many_experts_as_there_may_be(h, fmt, per, N, K):  # noqa: F811
    """1024 experts: one row of every third (few-token kernel), and up to nine each (CTA pairs)."""
    from test_gpu_quant_products import check_grouped
    counts = [int(e % 3 == 0) if per == 1 else e % (per + 1) for e in range(1024)]
    check_grouped(h, fmt, counts, N, K, seed=per)
