"""Products with both operands in 4 bits, dense and by expert, against 64-bit sums of the decoded values."""
import pytest
import torch

import quant_ref as ref

pkg = pytest.importorskip("paper_2609_04526_gb300")
pytestmark = pytest.mark.gpu
FORMATS = [pkg.NVFP4, pkg.MXFP4]


@pytest.fixture(scope="module")
def h():
    return pkg.Handle()


def weight(g, fmt, shape, K, signs=False):
    """Random codes, and scale bytes around one (every byte sign where asked)."""
    codes = torch.randint(0, 256, (*shape, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    lo, hi = (0x28, 0x48) if fmt == pkg.NVFP4 else (122, 128)
    scales = torch.randint(lo, hi, (*shape, K // ref.BLOCK[fmt]), generator=g, device="cuda", dtype=torch.uint8)
    if signs:
        scales = scales + 128 * torch.randint(0, 2, scales.shape, generator=g, device="cuda", dtype=torch.uint8)
    return codes, scales


def rows(g, h, fmt, R, K, ws2=None):
    X = torch.randn(R, K, generator=g, device="cuda") * torch.exp(torch.randn(R, 1, generator=g, device="cuda"))
    return h.sq_quantize(fmt, X.bfloat16(), ws2=ws2)


def decoded(q):
    v = ref.values(q.fmt, q.codes.cpu(), q.scales.cpu())
    return v * (q.row_ws2.cpu().double()[:, None] if q.row_ws2 is not None else q.ws2)


def close(got, x, w, what=""):
    """Half a step of bf16, and for each step of 64 products (and the addition of parts) a rounding of the fp32
    sum by at most 2^-22 of all magnitudes that went into it."""
    x, w = x.cuda(), w.cuda()
    want, size = x @ w.T, x.abs() @ w.abs().T
    steps = x.shape[1] / 64 + 9
    bound = 2.0 ** -8 * want.abs() + steps * 2.0 ** -22 * size
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {((got.double() - want).abs() / bound).max()}"


def check_dense(h, fmt, R, N, K, seed, ws2=None, signs=False, w_ws2=0.0173):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes, scales = weight(g, fmt, (N,), K, signs)
    q = rows(g, h, fmt, R, K, ws2)
    w_ws2 = 1.0 if fmt == pkg.MXFP4 else w_ws2
    Y = h.sq_quant_fwd(pkg.QuantWeight(fmt, N, K, codes, scales, w_ws2), q)
    h.sq_sync()
    close(Y, decoded(q), ref.values(fmt, codes.cpu(), scales.cpu()) * float(torch.tensor(w_ws2)), f"{R} {N} {K}")
    return q, Y


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("R, N, K", [(1, 8, 32), (1, 128, 256), (5, 136, 512), (8, 256, 64), (9, 384, 96), (33, 1048, 2720),
                                     (64, 520, 1056), (128, 512, 4096), (100, 264, 2912), (1, 4096, 4096), (17, 2880, 2880)])
def test_few_tokens(h, fmt, R, N, K):
    check_dense(h, fmt, R, N, K, seed=R + N + K)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("R, N, K", [(129, 264, 288), (256, 256, 1024), (300, 520, 2720), (1000, 1048, 544), (2048, 2048, 2048),
                                     (4097, 72, 4128)])
def test_many_tokens(h, fmt, R, N, K):
    check_dense(h, fmt, R, N, K, seed=R + N + K)


@pytest.mark.parametrize("R, N, K", [(3, 136, 800), (64, 256, 1024), (500, 520, 1312), (1024, 512, 512)])
def test_negative_scales(h, R, N, K):
    check_dense(h, pkg.NVFP4, R, N, K, seed=R + N + K, signs=True)
    check_dense(h, pkg.NVFP4, R, N, K, seed=R + N + K + 1, signs=True, ws2=0.003)


def check_grouped(h, fmt, counts, N, K, seed, tail=3, signs=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    E, R = len(counts), sum(counts) + tail
    codes, scales = weight(g, fmt, (E, N), K, signs)
    offsets = torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], device="cuda")
    q = rows(g, h, fmt, R, K)
    ws2 = None if fmt == pkg.MXFP4 else torch.rand(E, generator=g, device="cuda") + 0.1
    Y = torch.full((R, N), 7.0, dtype=torch.bfloat16, device="cuda")
    w = pkg.GroupedWeight(fmt, E, N, K, codes, scales, ws2)
    h.sq_grouped_quant_fwd(w, offsets, q, Y=Y)
    h.sq_sync()
    x, off = decoded(q), offsets.tolist()
    for e in range(E):
        if counts[e]:
            v = ref.values(fmt, codes[e].cpu(), scales[e].cpu()) * (1.0 if ws2 is None else float(ws2[e]))
            close(Y[off[e]:off[e + 1]], x[off[e]:off[e + 1]], v, f"expert {e}")
    assert (Y[off[E]:] == 7.0).all()  # rows of no expert are left as they were
    return w, offsets, q, Y


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts, N, K", [
    ([1], 8, 32), ([0, 1, 0], 136, 64), ([5, 0, 7, 1, 128, 129, 0], 200, 352), ([0, 0, 0], 64, 256),
    ([1] * 9 + [0] * 55, 768, 2048), ([300, 1, 513, 40], 264, 1056), ([1000, 0, 700, 333], 520, 512),
    ([7] * 130, 72, 288), ([600, 599, 601, 0, 1024], 392, 2720)])
def test_experts_of_ragged_sizes(h, fmt, counts, N, K):
    check_grouped(h, fmt, counts, N, K, seed=len(counts) + N)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("E, per, N, K", [(96, 120, 264, 4096), (96, 60, 392, 2560), (160, 3, 264, 4096), (96, 120, 264, 2080)])
def test_experts_in_rings_of_an_odd_number_of_slots(h, fmt, E, per, N, K):
    """Two CTAs share an SM and its shared memory: rings of 3 and 5 slots, gone through many times."""
    counts = [per + (e * 5) % 9 - 4 if per > 8 else e % (per + 1) for e in range(E)]
    check_grouped(h, fmt, counts, N, K, seed=E + K)


def test_experts_with_negative_scales(h):
    check_grouped(h, pkg.NVFP4, [3, 0, 70, 400], 200, 544, seed=1, signs=True)
    check_grouped(h, pkg.NVFP4, [900, 0, 1300], 328, 1024, seed=2, signs=True)


@pytest.mark.parametrize("rows_", [40, 900])
def test_offsets_outside_the_rows_are_kept_within(h, rows_):
    """Offsets that decrease, or lie outside the rows: what lies within is computed, nothing else touched."""
    g = torch.Generator(device="cuda").manual_seed(9)
    N, K, E = 136, 320, 4
    codes, scales = weight(g, pkg.MXFP4, (E, N), K)
    q = rows(g, h, pkg.MXFP4, rows_, K)
    w = pkg.GroupedWeight(pkg.MXFP4, E, N, K, codes, scales, None)
    Y = h.sq_grouped_quant_fwd(w, torch.tensor([-5, 10, 4, 30, 1 << 40], device="cuda"), q)
    h.sq_sync()
    x = decoded(q)
    for e, (lo, hi) in enumerate(((0, 10), (10, 10), (4, 30), (30, rows_))):
        if e in (0, 3):
            span = slice(lo, 4) if e == 0 else slice(lo, hi)  # rows 4 .. 9 are two experts'
            close(Y[span], x[span], ref.values(pkg.MXFP4, codes[e].cpu(), scales[e].cpu()))


@pytest.mark.parametrize("counts", [[3, 0, 20, 1], [500, 0, 300, 900]])
def test_captured_and_replayed_with_other_offsets(h, counts):
    """A captured pass from the router's choice to the experts' rows follows new tokens and offsets."""
    g = torch.Generator(device="cuda").manual_seed(11)
    E, N, K, k, T = len(counts), 264, 544, 2, sum(counts) // 2
    codes, scales = weight(g, pkg.NVFP4, (E, N), K)
    w = pkg.GroupedWeight(pkg.NVFP4, E, N, K, codes, scales, torch.rand(E, generator=g, device="cuda") + 0.5)
    X = torch.zeros(T, K, dtype=torch.bfloat16, device="cuda")
    logits = torch.zeros(T, E, device="cuda")

    def step():
        experts, weights = h.sq_route(logits, k)
        offsets, row_of, slot_of = h.sq_sort_tokens(experts, E)
        q = h.sq_quantize(pkg.NVFP4, X, slot_of=slot_of, k=k)
        return h.sq_combine(h.sq_grouped_quant_fwd(w, offsets, q), row_of, weights)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = step()
    for _ in range(3):
        X.copy_(torch.randn(T, K, generator=g, device="cuda"))
        logits.copy_(torch.randn(T, E, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, step())
    h.sq_sync()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("R", [0, 1, 40, 700])
def test_not_finite_rows_stay_alone(h, fmt, R):
    """A row with a NaN spoils its own outputs only; no rows are no work."""
    g = torch.Generator(device="cuda").manual_seed(R)
    N, K = 136, 352
    codes, scales = weight(g, fmt, (N,), K)
    X = torch.randn(R, K, generator=g, device="cuda").bfloat16()
    w = pkg.QuantWeight(fmt, N, K, codes, scales, 1.0)
    clean = h.sq_quant_fwd(w, h.sq_quantize(fmt, X))
    if R:
        X[R // 2, 5] = float("nan")
    Y = h.sq_quant_fwd(w, h.sq_quantize(fmt, X))
    h.sq_sync()
    keep = torch.arange(R, device="cuda") != R // 2
    assert torch.equal(Y[keep], clean[keep]) and torch.isnan(Y[~keep].float()).all()


@pytest.mark.parametrize("R, N, K", [(30, 136, 544), (6000, 2056, 544)])
def test_offsets_that_descend_write_no_other_rows(h, R, N, K):
    """Experts that claim the same rows, more of them than the launch has tiles for: rows outside every claim keep
    what they held, and the call after it is right."""
    g = torch.Generator(device="cuda").manual_seed(17)
    E, lo, hi = 24, 5, R - 7
    codes, scales = weight(g, pkg.NVFP4, (E, N), K)
    q = rows(g, h, pkg.NVFP4, R, K)
    w = pkg.GroupedWeight(pkg.NVFP4, E, N, K, codes, scales, torch.ones(E, device="cuda"))
    buf = torch.full((R + 512, N), 7.0, dtype=torch.bfloat16, device="cuda")
    offsets = torch.tensor([hi if e % 2 else lo for e in range(E + 1)], dtype=torch.int64, device="cuda")
    h.sq_grouped_quant_fwd(w, offsets, q, Y=buf[256:R + 256])
    h.sq_sync()
    assert (buf[:256 + lo] == 7).all() and (buf[256 + hi:] == 7).all()
    assert torch.isfinite(buf.float()).all()
    check_grouped(h, pkg.NVFP4, [R // 3, 0, R - R // 3], N, K, seed=18)
