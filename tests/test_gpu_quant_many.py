"""4-bit products of many rows (the kernel of CTA pairs and the launch that lays out its scales), and what is
shared between calls: scratch, streams, graphs, threads."""
import threading

import pytest
import torch

import quant_ref as ref
from test_gpu_quant_products import FORMATS, check_dense, check_grouped, close, decoded, h, rows, weight  # noqa: F401

pkg = pytest.importorskip("paper_2609_04526_gb300")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("R, N, K", [(5000, 2056, 288), (2500, 4104, 96), (2000, 8200, 352), (4100, 4096, 32), (3000, 4104, 2912),
                                     (4097, 2880, 4128), (2049, 8192, 256)])
def test_many_rows(h, fmt, R, N, K):  # noqa: F811
    check_dense(h, fmt, R, N, K, seed=R + N + K)


@pytest.mark.parametrize("R, N, K", [(5000, 2056, 288), (3000, 4104, 2720), (2048, 8192, 1024)])
def test_many_rows_with_negative_scales(h, R, N, K):  # noqa: F811
    check_dense(h, pkg.NVFP4, R, N, K, seed=R + N + K, signs=True)
    check_dense(h, pkg.NVFP4, R, N, K, seed=R + N + K + 1, ws2=0.004)  # and none: what the call before left is not read


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("counts, N, K", [
    ([900, 0, 1, 224, 225, 448, 3200], 1032, 544), ([3000, 0, 0, 2000], 2056, 2720), ([0] * 5 + [6000], 1200, 1024),
    ([50 + 13 * (e % 9) for e in range(96)], 264, 2080), ([17] * 512, 520, 352)])
def test_many_rows_of_ragged_experts(h, fmt, counts, N, K):  # noqa: F811
    check_grouped(h, fmt, counts, N, K, seed=len(counts) + N)


def test_many_rows_of_no_expert(h):  # noqa: F811
    check_grouped(h, pkg.NVFP4, [0] * 6, 2056, 544, seed=2, tail=6000)


def test_ragged_experts_with_negative_scales(h):  # noqa: F811
    check_grouped(h, pkg.NVFP4, [900, 0, 1, 224, 225, 448, 3200], 1032, 544, seed=3, signs=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_not_finite_stay_alone_among_many(h, fmt):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(8)
    R, N, K = 4000, 2056, 352
    codes, scales = weight(g, fmt, (N,), K)
    X = torch.randn(R, K, generator=g, device="cuda").bfloat16()
    w = pkg.QuantWeight(fmt, N, K, codes, scales, 1.0)
    clean = h.sq_quant_fwd(w, h.sq_quantize(fmt, X))
    X[::97, 5] = float("inf")
    Y = h.sq_quant_fwd(w, h.sq_quantize(fmt, X))
    h.sq_sync()
    bad = torch.zeros(R, dtype=torch.bool, device="cuda")
    bad[::97] = True
    assert torch.equal(Y[~bad], clean[~bad]) and torch.isnan(Y[bad].float()).all()


def test_outputs_past_two_to_the_31(h):  # noqa: F811
    """More than 2^31 outputs: the last rows against their formula, rows in between against a call of their own."""
    R, N, K = 70001, 32768, 32
    g = torch.Generator(device="cuda").manual_seed(9)
    codes, scales = weight(g, pkg.MXFP4, (N,), K)
    q = rows(g, h, pkg.MXFP4, R, K)
    w = pkg.QuantWeight(pkg.MXFP4, N, K, codes, scales, 1.0)
    Y = h.sq_quant_fwd(w, q)
    part = slice(R - 300, R)
    tail = pkg.QuantRows(pkg.MXFP4, 300, K, q.codes[part].contiguous(), q.scales[part].contiguous())
    close(Y[part], decoded(tail), ref.values(pkg.MXFP4, codes.cpu(), scales.cpu()))
    part = slice(65530, 65560)  # around 2^31 / N
    few = pkg.QuantRows(pkg.MXFP4, 30, K, q.codes[part].contiguous(), q.scales[part].contiguous())
    close(Y[part], decoded(few), ref.values(pkg.MXFP4, codes.cpu(), scales.cpu()))


def test_runs_alike(h):  # noqa: F811
    """The same bits at every run."""
    for R, N, K in ((100, 264, 2912), (5000, 2056, 544)):
        q, Y = check_dense(h, pkg.NVFP4, R, N, K, seed=1)
        _, again = check_dense(h, pkg.NVFP4, R, N, K, seed=1)
        assert torch.equal(Y, again)


def test_graphs_captured_before_the_scratch_grew():
    """A captured product replays right after a larger call of the same handle, and again."""
    h2 = pkg.Handle()
    g = torch.Generator(device="cuda").manual_seed(12)
    R, N, K = 5000, 2056, 288
    codes, scales = weight(g, pkg.NVFP4, (N,), K)
    w = pkg.QuantWeight(pkg.NVFP4, N, K, codes, scales, 0.5)
    q = rows(g, h2, pkg.NVFP4, R, K)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        fresh = torch.cuda.CUDAGraph()
        with pytest.raises(pkg.SQError) as err, torch.cuda.graph(fresh, stream=side):  # scratch cannot be allocated there
            h2.sq_quant_fwd(w, q)
        assert err.value.status == -2
        want = h2.sq_quant_fwd(w, q)
    side.synchronize()
    out = torch.empty_like(want)
    with torch.cuda.graph(graph, stream=side):
        h2.sq_quant_fwd(w, q, Y=out)
    check_dense(h2, pkg.NVFP4, 6000, 4096, 1056, seed=13)
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    h2.sq_sync()


def test_calls_on_another_stream(h):  # noqa: F811
    """Inputs written and outputs used in the order of the stream that is named."""
    g = torch.Generator(device="cuda").manual_seed(14)
    R, N, K = 700, 520, 1056
    codes, scales = weight(g, pkg.NVFP4, (N,), K)
    w = pkg.QuantWeight(pkg.NVFP4, N, K, codes, scales, 1.0)
    X = torch.randn(R, K, generator=g, device="cuda").bfloat16()
    want = h.sq_quant_fwd(w, h.sq_quantize(pkg.NVFP4, X))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    late = torch.zeros_like(X)
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        late.copy_(X)
    q = h.sq_quantize(pkg.NVFP4, late, stream=side)
    Y = h.sq_quant_fwd(w, q, stream=side)
    back = h.sq_dequantize(q, stream=side)
    h.sq_sync(side)
    assert torch.equal(Y, want) and torch.equal(back, h.sq_dequantize(h.sq_quantize(pkg.NVFP4, X)))


def test_two_threads_with_a_handle_each():
    failures = []

    def work(seed):
        try:
            mine, stream = pkg.Handle(), torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for i in range(3):
                    check_dense(mine, pkg.NVFP4, 60 + i, 264, 544, seed=seed)
                    check_dense(mine, pkg.MXFP4, 5000 + i, 2056, 288, seed=seed)
        except Exception as e:  # noqa: BLE001
            failures.append(e)

    threads = [threading.Thread(target=work, args=(s,)) for s in (1, 2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("R, N, K", [(70, 136, 544), (900, 264, 1056)])
def test_a_step_that_keeps_its_rows_in_four_bits(h, fmt, R, N, K):  # noqa: F811
    """Forward in 4 bits, backward from the kept codes: the scale gradient is the derivative of that forward, by its
    formula in 64 bits and by the difference that a changed scale makes."""
    g = torch.Generator(device="cuda").manual_seed(R)
    B = ref.BLOCK[fmt]
    codes, scales = weight(g, fmt, (N,), K)
    ws2 = 1.0 if fmt == pkg.MXFP4 else 0.031
    w = pkg.QuantWeight(fmt, N, K, codes, scales, ws2)
    X = torch.randn(R, K, generator=g, device="cuda").bfloat16()
    dY = torch.randn(R, N, generator=g, device="cuda").bfloat16()
    q = h.sq_quantize(fmt, X)
    kept = h.sq_dequantize(q)
    grad = h.sq_scale_grad(w, kept, dY)
    dX = h.sq_bwd_dx(w, dY)
    h.sq_sync()
    x, dy = decoded(q).cuda(), dY.double()
    assert torch.equal(kept.double(), x)  # the rows that the forward saw, exactly
    c = ref.values(fmt, codes.cpu(), torch.full_like(scales, 0x38 if fmt == pkg.NVFP4 else 127).cpu()).cuda()  # the codes alone
    want = ((dy.T @ x) * c).view(N, K // B, B).sum(2)
    size = ((dy.abs().T @ x.abs()) * c.abs()).view(N, K // B, B).sum(2)
    # fp32 sums of R K-blocks of 16 exact products, B x 1 additions: each loses at most 2^-22 of what went into it
    assert ((grad.double() - want).abs() <= (R / 16 + 40) * 2.0 ** -22 * size).all()
    W = ref.values(fmt, codes.cpu(), scales.cpu()).cuda() * float(torch.tensor(ws2))
    dx, dx_size = dy @ W, dy.abs() @ W.abs()
    assert ((dX.double() - dx).abs() <= 2.0 ** -8 * dx.abs() + (N / 16 + 8) * 2.0 ** -22 * dx_size).all()
    # one scale to the next byte: the outputs' change, through the 4-bit forward, against the gradient
    n, b = 5, 1
    moved = scales.clone()
    moved[n, b] += 1
    step = float((ref.scale_values(fmt, moved.cpu()) - ref.scale_values(fmt, scales.cpu()))[n, b]) * ws2
    before, after = h.sq_quant_fwd(w, q), h.sq_quant_fwd(pkg.QuantWeight(fmt, N, K, codes, moved, ws2), q)
    h.sq_sync()
    change = ((after.double() - before.double())[:, n] * dy[:, n]).sum()
    # both outputs are rounded to bf16, by at most 2^-8 of them
    slack = (2.0 ** -8 * (after.double().abs() + before.double().abs())[:, n] * dy[:, n].abs()).sum()
    assert abs(change - step * grad[n, b].double()) <= slack
    others = torch.arange(N, device="cuda") != n
    assert torch.equal(before[:, others], after[:, others])


def by_slot(h, fmt, X, slots, k, ws2=None):
    """The rows of `slots` out of X, zeros where there is none, quantised as rows of their own."""
    on = (slots >= 0) & (slots < X.shape[0] * k)
    rows_ = torch.zeros(slots.shape[0], X.shape[1], dtype=X.dtype, device=X.device)
    rows_[on] = X[(slots[on] // k).long()]
    return h.sq_quantize(fmt, rows_, ws2)


def alike(a, b):
    return (torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales) and a.ws2 == b.ws2
            and (a.row_ws2 is None) == (b.row_ws2 is None) and (a.row_ws2 is None or torch.equal(a.row_ws2, b.row_ws2)))


@pytest.mark.parametrize("fmt, ws2", [(pkg.NVFP4, None), (pkg.NVFP4, 0.0031), (pkg.MXFP4, None)])
@pytest.mark.parametrize("T, K, k", [(2000, 2048, 8), (2000, 2880, 8), (1500, 2912, 8), (4000, 1056, 8), (5001, 20512, 3), (300, 32, 1)])
def test_many_rows_of_few_tokens(h, fmt, ws2, T, K, k):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(T + K)
    X = torch.randn(T, K, generator=g, device="cuda").bfloat16()
    X[3, 17], X[4, 20] = float("nan"), float("-inf")
    slots = torch.randperm(T * k, generator=g, device="cuda").int()[:T * k - 5].clone()
    slots[:4] = torch.tensor([-1, T * k, -(1 << 31), (1 << 31) - 1], dtype=torch.int32, device="cuda")
    slots[50:60] = 3 * k  # a row of one token again and again, one that is not finite
    slots[60:70] = T * k - 1
    q = h.sq_quantize(fmt, X, ws2, slot_of=slots, k=k)
    h.sq_sync()
    assert alike(q, by_slot(h, fmt, X, slots, k, ws2))


@pytest.mark.parametrize("fmt", FORMATS)
def test_many_rows_of_no_token(h, fmt):  # noqa: F811
    slots = torch.zeros(1000000, dtype=torch.int32, device="cuda")
    X = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    q = h.sq_quantize(fmt, X, slot_of=slots, k=4)
    h.sq_sync()
    assert alike(q, by_slot(h, fmt, X, torch.full_like(slots, -1), 4))


def test_rows_by_slot_captured_with_scratch_and_without():
    """A first call inside a capture, a captured one that has scratch, and one whose scratch grew since: the same rows,
    of what the tokens and slots are when it runs."""
    h2 = pkg.Handle()
    g = torch.Generator(device="cuda").manual_seed(21)
    T, K, k = 2000, 2880, 8
    X = torch.randn(T, K, generator=g, device="cuda").bfloat16()
    slots = torch.randperm(T * k, generator=g, device="cuda").int()
    h2.sq_quantize(pkg.NVFP4, X[:1])  # the device is set up
    graphs, outs = [], []
    side = torch.cuda.Stream()
    for i in range(2):
        with torch.cuda.stream(side):
            out = pkg.QuantRows(pkg.NVFP4, T * k, K, torch.zeros(T * k, K // 2, dtype=torch.uint8, device="cuda"),
                                torch.zeros(T * k, K // 16, dtype=torch.uint8, device="cuda"), 1.0, torch.zeros(T * k, device="cuda"))
            if i:
                h2.sq_quantize(pkg.NVFP4, X, slot_of=slots, k=k)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            h2.sq_quantize(pkg.NVFP4, X, slot_of=slots, k=k, out=out)
        graphs.append(graph)
        outs.append(out)
    big = torch.randn(2 * T, K, generator=g, device="cuda").bfloat16()
    more = torch.randperm(2 * T * k, generator=g, device="cuda").int()
    assert alike(h2.sq_quantize(pkg.NVFP4, big, slot_of=more, k=k), by_slot(h2, pkg.NVFP4, big, more, k))
    for _ in range(2):
        X.copy_(torch.randn(T, K, generator=g, device="cuda").bfloat16())
        slots.copy_(torch.randperm(T * k, generator=g, device="cuda").int())
        want = by_slot(h2, pkg.NVFP4, X, slots, k)
        for graph, out in zip(graphs, outs):
            graph.replay()
            torch.cuda.synchronize()
            assert alike(out, want)
    h2.sq_sync()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("R, N, K", [(2048, 4096, 2912), (2047, 4096, 2080), (1024, 8192, 2880), (1000, 8200, 4128), (1999, 4104, 2272),
                                     (480, 19456, 2080)])
def test_rows_in_tiles_of_more_than_224(h, fmt, R, N, K):  # noqa: F811
    """Sizes at which tiles of 240 or 256 rows save a wave: their accumulators share columns."""
    check_dense(h, fmt, R, N, K, seed=R + N + K)


@pytest.mark.parametrize("R, N, K", [(2048, 4096, 2912), (1000, 8200, 2080), (2100, 2056, 8224)])
def test_tall_tiles_and_deep_stages_with_negative_scales(h, R, N, K):  # noqa: F811
    check_dense(h, pkg.NVFP4, R, N, K, seed=R + N + K, signs=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("R, N, K", [(3000, 4104, 544), (3000, 4104, 800), (2500, 4104, 4384), (2500, 4104, 4640)])
def test_an_odd_number_of_slices(h, fmt, R, N, K):  # noqa: F811
    """K whose last stage has one slice, none in stages of one, or a second one past its end."""
    check_dense(h, fmt, R, N, K, seed=R + N + K)
