"""4-bit products at the sizes of tests/quant_shapes.py: rings of an odd number of slots that are gone through again,
tall tiles whose accumulators are used again, experts on the pair kernel captured and replayed, long sums."""
import pytest
import torch

import quant_ref as ref
import quant_shapes as shapes
from test_gpu_quant_products import check_dense, check_grouped, close, decoded, h, weight  # noqa: F401

pkg = pytest.importorskip("paper_2609_04526_gb300")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", shapes.THREE_SLOTS + shapes.FIVE_SLOTS, ids=lambda c: f"{c[0]}-{len(c[1])}-{c[2]}-{c[3]}")
def test_experts_in_odd_rings(h, case):  # noqa: F811
    fmt, counts, N, K = case
    check_grouped(h, fmt, counts, N, K, seed=K + len(counts))
    if fmt == pkg.NVFP4:
        check_grouped(h, fmt, counts, N, K, seed=K + 1, signs=True)


@pytest.mark.parametrize("case", shapes.THREE_SLOTS_DENSE)
def test_dense_products_in_odd_rings(h, case):  # noqa: F811
    check_dense(h, *case, seed=sum(case))
    if case[0] == pkg.NVFP4:
        check_dense(h, *case, seed=sum(case) + 1, signs=True)


@pytest.mark.parametrize("case", shapes.TALL + shapes.TALL_AND_SHORT)
def test_tall_tiles_use_their_accumulators_again(h, case):  # noqa: F811
    """The third tile of a CTA pair, whose accumulator shares columns with the two before it, and later ones."""
    check_dense(h, *case, seed=sum(case))


@pytest.mark.parametrize("case", [c for c in shapes.TALL + shapes.TALL_AND_SHORT if c[0] == pkg.NVFP4])
def test_tall_tiles_with_negative_scales(h, case):  # noqa: F811
    check_dense(h, *case, seed=sum(case) + 1, signs=True)


@pytest.mark.parametrize("case", shapes.PAIR_EXPERTS)
def test_pair_experts_captured_and_replayed_with_other_offsets(h, case):  # noqa: F811
    """A captured product by expert follows the rows and offsets that a replay finds: unequal ones, all rows one
    expert's, none of some, rows of no expert behind the last."""
    fmt, counts, N, K = case
    g = torch.Generator(device="cuda").manual_seed(23)
    E, R = len(counts), sum(counts)
    codes, scales = weight(g, fmt, (E, N), K)
    w = pkg.GroupedWeight(fmt, E, N, K, codes, scales, None if fmt == pkg.MXFP4 else torch.rand(E, generator=g, device="cuda") + 0.5)
    X = torch.randn(R, K, generator=g, device="cuda").bfloat16()
    offsets = torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], device="cuda")
    Y = torch.zeros(R, N, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()

    def step():
        h.sq_grouped_quant_fwd(w, offsets, h.sq_quantize(fmt, X), Y=Y)

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for ends in (counts, [0, R, 0, 0], [1, 223, 225, R - 449], [R - 1000, 0, 0, 300], [0, 0, 0, 0]):
        X.copy_(torch.randn(R, K, generator=g, device="cuda"))
        offsets.copy_(torch.tensor([0, *torch.tensor(ends).cumsum(0).tolist()]))
        Y.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = Y.clone()
        Y.fill_(7.0)
        step()
        h.sq_sync()
        assert torch.equal(got, Y) and (got[sum(ends):] == 7.0).all()
        x = decoded(h.sq_quantize(fmt, X))
        first = 0
        for e, n in enumerate(ends):
            if n:
                v = ref.values(fmt, codes[e].cpu(), scales[e].cpu()) * (1.0 if w.ws2 is None else float(w.ws2[e]))
                close(got[first:first + n], x[first:first + n], v, f"{ends} expert {e}")
            first += n


@pytest.mark.parametrize("fmt, R, N, K", shapes.LONG)
def test_long_sums(h, fmt, R, N, K):  # noqa: F811
    """Sums of 2^18 products, all of one sign: a few rows and features over and over, the same bits wherever they lie."""
    g = torch.Generator(device="cuda").manual_seed(24)
    few, some = 20, 26
    codes, scales = weight(g, fmt, (some,), K)
    x_codes, x_scales = weight(g, fmt, (few,), K)
    codes, x_codes = codes & 0x77, x_codes & 0x77
    q = pkg.QuantRows(fmt, R, K, x_codes.repeat(R // few, 1), x_scales.repeat(R // few, 1))
    Y = h.sq_quant_fwd(pkg.QuantWeight(fmt, N, K, codes.repeat(N // some, 1), scales.repeat(N // some, 1), 1.0), q)
    h.sq_sync()
    assert torch.equal(Y, Y[:few, :some].repeat(R // few, N // some))
    close(Y[:few, :some], ref.values(fmt, x_codes.cpu(), x_scales.cpu()), ref.values(fmt, codes.cpu(), scales.cpu()))
