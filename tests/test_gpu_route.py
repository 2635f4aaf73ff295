"""Routing around the experts against 64-bit forms: top-k and its gradient, the sort by expert,
rows to the experts and back with their gradients."""
import numpy as np
import pytest
import torch

import step_ref as ref

pytestmark = pytest.mark.gpu
pkg = pytest.importorskip("paper_2609_04526_gb300")


@pytest.fixture(scope="module")
def h():
    return pkg.Handle()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64) if t.is_floating_point() else t.cpu().numpy()


def _logits(T, E, bf16, seed, kind="gauss"):
    z = torch.randn(T, E, generator=_gen(seed), device="cuda") * 2.0
    if kind == "ties":
        z = torch.round(z)
    elif kind == "masked":  # experts at the type's lowest value, at -inf and NaN; some rows all masked
        u = torch.rand(T, E, generator=_gen(seed + 1), device="cuda")
        z = torch.where(u < 0.3, torch.full_like(z, -float("inf")), z)
        z = torch.where((u >= 0.3) & (u < 0.5), torch.full_like(z, torch.finfo(torch.bfloat16 if bf16 else torch.float32).min), z)
        z = torch.where((u >= 0.5) & (u < 0.55), torch.full_like(z, float("nan")), z)
        z[::5] = -float("inf")
        if T > 1:
            z[1::7] = float("nan")
    return z.bfloat16() if bf16 else z


def _check_weights(w, want, z, E):
    z = np.where(np.isfinite(z) & (np.abs(z) < 1e30), z, 0.0)
    tol = (E + 16 + 4 * np.abs(z).max()) * ref.U32
    assert np.all(np.abs(w - want) <= tol * np.abs(want) + 1e-37), np.abs(w - want).max()


@pytest.mark.parametrize("E, k", [(1, 1), (5, 3), (8, 8), (32, 2), (33, 4), (60, 6), (64, 32), (128, 8), (200, 4), (256, 1),
                                  (384, 8), (512, 10), (777, 5), (1024, 32)])
@pytest.mark.parametrize("kind, bf16", [("gauss", False), ("ties", True), ("masked", False), ("masked", True)])
def test_route(h, E, k, kind, bf16):
    T = 37
    z = _logits(T, E, bf16, 3 * E + k, kind)
    valid = torch.rand(T, generator=_gen(9), device="cuda") < 0.8
    for norm in (True, False):
        for v in (None, valid):
            experts, weights = h.sq_route(z, k, normalize=norm, valid=v)
            want_e, want_w = ref.route(_np(z), k, norm, None if v is None else _np(v))
            assert np.array_equal(_np(experts), want_e)
            _check_weights(_np(weights), want_w, _np(z), E)
        dw = torch.randn(T, k, generator=_gen(5), device="cuda")
        dw = torch.where(experts >= 0, dw, float("nan"))  # a slot without an expert is in no sum
        dz = h.sq_route_grad(z, experts, dw, normalize=norm)
        assert dz.dtype == z.dtype
        want, size = ref.route_grad(_np(z), _np(experts), _np(dw), norm)
        finite = np.where(np.isfinite(_np(z)) & (np.abs(_np(z)) < 1e30), _np(z), 0.0)
        tol = 4 * (E + 16 + 4 * np.abs(finite).max()) * ref.U32
        err = np.abs(_np(dz) - want)
        assert np.all(err <= tol * size + (1.01 * ref.U16 * np.abs(want) if bf16 else 0) + 1e-37), err.max()


@pytest.mark.parametrize("E, k", [(9, 9), (100, 16), (128, 12), (131, 9), (256, 16)])
@pytest.mark.parametrize("kind, bf16", [("gauss", False), ("ties", True), ("masked", True)])
def test_route_of_more_choices(h, E, k, kind, bf16):
    test_route(h, E, k, kind, bf16)


def test_route_infinite_logit(h):
    z = torch.zeros(2, 8, device="cuda")
    z[0, 3] = float("inf")
    z[1, 2], z[1, 6] = float("inf"), float("inf")
    experts, weights = h.sq_route(z, 2)
    assert experts.tolist() == [[3, 0], [2, 6]]
    assert weights.tolist() == [[1.0, 0.0], [0.5, 0.5]]


@pytest.mark.parametrize("T", [0, 1, 8, 9, 4099])
def test_route_token_counts(h, T):
    z = _logits(T, 128, False, 70 + T)
    experts, weights = h.sq_route(z, 8)
    assert experts.shape == (T, 8)
    if T:
        want_e, want_w = ref.route(_np(z[-9:]), 8, True)
        assert np.array_equal(_np(experts[-9:]), want_e)
        _check_weights(_np(weights[-9:]), want_w, _np(z), 128)


@pytest.mark.parametrize("norm", [True, False])
def test_route_gradient_against_differences(h, norm):
    """d sum(dw w) along one logit, from central differences of the weights the forward returns."""
    T, E, k = 16, 24, 4
    z = _logits(T, E, False, 31)
    dw = torch.randn(T, k, generator=_gen(32), device="cuda").double()
    experts, _ = h.sq_route(z, k, normalize=norm)
    dz = h.sq_route_grad(z, experts, dw.float(), normalize=norm).double()
    step = 2.0 ** -6  # differences' error: step^2 / 6 of a third derivative of at most ~8 |dw|, and fp32 noise / step
    for e in range(0, E, 3):
        up, down = z.clone(), z.clone()
        up[:, e] += step
        down[:, e] -= step
        eu, wu = h.sq_route(up, k, normalize=norm)
        ed, wd = h.sq_route(down, k, normalize=norm)
        same = (eu.sort(1).values == ed.sort(1).values).all(1)  # tokens whose choice the step leaves alone

        def of(ex, w):  # weights in the slots of `experts`
            full = torch.zeros(T, E, dtype=torch.float64, device="cuda").scatter_(1, ex.long(), w.double())
            return full.gather(1, experts.long())

        diff = ((of(eu, wu) - of(ed, wd)) * dw).sum(1) / (2 * step)
        bound = (8 * step ** 2 / 6 + 64 * 2.0 ** -24 / step) * dw.abs().sum(1)
        assert bool(((diff - dz[:, e]).abs() <= bound)[same].all())


@pytest.mark.parametrize("n", [0, 1, 31, 32, 33, 257, 2048, 2049, 8192, 8193, 30011, 262144])
@pytest.mark.parametrize("E", [1, 7, 128, 1000])
def test_sort(h, n, E):
    e = torch.randint(-1 if n % 2 else 0, E + (n % 3 == 0), (n, 1), generator=_gen(n + E), device="cuda", dtype=torch.int32)
    offsets, row_of, slot_of = h.sq_sort_tokens(e, E)
    want = ref.sort(_np(e), E)
    for got, w in zip((offsets, row_of, slot_of), want):
        assert np.array_equal(_np(got), w)


@pytest.mark.parametrize("value", [-1, 0, 5, 127, 128, 2 ** 31 - 1, -2 ** 31])
def test_sort_one_value(h, value):
    e = torch.full((9001, 2), value, device="cuda", dtype=torch.int32)
    for got, w in zip(h.sq_sort_tokens(e, 128), ref.sort(_np(e), 128)):
        assert np.array_equal(_np(got), w)


def _plan(h, T, E, k, seed, off=0.2):
    e = torch.argsort(torch.rand(T, E, generator=_gen(seed), device="cuda"), dim=1)[:, :k].int()
    e = torch.where(torch.rand(T, k, generator=_gen(seed + 1), device="cuda") < off, -1, e).contiguous()
    offsets, row_of, slot_of = h.sq_sort_tokens(e, E)
    w = torch.rand(T, k, generator=_gen(seed + 2), device="cuda")
    return int(offsets[-1]), row_of, slot_of, torch.where(e < 0, float("nan"), w)  # weights without an expert: not read


MOVES = [(1, 8, 1, 8), (1, 2880, 4, 8), (7, 264, 3, 5), (187, 256, 8, 60), (40, 1032, 9, 16), (33, 512, 32, 32), (65, 2048, 8, 128),
         (300, 4096, 2, 8), (1000, 1288, 6, 64)]


@pytest.mark.parametrize("T, D, k, E", MOVES)
@pytest.mark.parametrize("whole", [True, False])
def test_rows_out_and_back(h, T, D, k, E, whole):
    M, row_of, slot_of, w = _plan(h, T, E, k, T + D)
    R = T * k if whole else M
    X = torch.randn(T, D, generator=_gen(1), device="cuda").bfloat16()
    X[(row_of < 0).all(1)] = float("nan")  # a token without experts is not read
    Xs = h.sq_dispatch(X, row_of, slot_of, Xs=torch.full((R, D), float("nan"), dtype=torch.bfloat16, device="cuda"))
    assert np.array_equal(_np(Xs), ref.dispatch(_np(X), _np(slot_of), k, R))

    Ys = torch.randn(R, D, generator=_gen(2), device="cuda").bfloat16()
    Ys[M:] = float("inf")  # rows past the routed ones are not read
    for weights in (w, None):
        Y = h.sq_combine(Ys, row_of, w) if weights is not None else h.sq_dispatch_grad(Ys, row_of)
        want, size = ref.combine(_np(Ys), _np(row_of), None if weights is None else _np(w))
        err = np.abs(_np(Y) - want)
        assert np.all(err <= (k + 2) * ref.U32 * size + 1.01 * ref.U16 * np.abs(want)), err.max()

    dY = torch.randn(T, D, generator=_gen(3), device="cuda").bfloat16()
    dY[(row_of < 0).all(1)] = float("nan")
    dYs, dw = h.sq_combine_grad(dY, Ys, row_of, slot_of, w, dYs=torch.full_like(Ys, float("nan")))
    want, want_dw, size = ref.combine_grad(_np(dY), _np(Ys), _np(row_of), _np(slot_of), _np(w))
    assert np.all(np.abs(_np(dYs) - want) <= (1.01 * ref.U16) * np.abs(want) + 1e-37)
    assert np.all(np.abs(_np(dw) - want_dw) <= (D + 16) * ref.U32 * size)


@pytest.mark.parametrize("k", [1, 2, 4, 8, 9])
def test_no_expert_rows_at_all(h, k):
    """Tokens that no expert serves, with an expert tensor of no rows: zeros, and nothing is read."""
    T, D = 37, 264
    _, row_of, slot_of = h.sq_sort_tokens(torch.full((T, k), -1, dtype=torch.int32, device="cuda"), 8)
    none = torch.empty(0, D, dtype=torch.bfloat16, device="cuda")
    w = torch.rand(T, k, generator=_gen(k), device="cuda")
    X = torch.full((T, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    assert h.sq_dispatch(X, row_of, slot_of, Xs=none.clone()).numel() == 0
    assert not h.sq_combine(none, row_of, w, Y=X.clone()).any()
    assert not h.sq_dispatch_grad(none, row_of, dX=X.clone()).any()
    dYs, dw = h.sq_combine_grad(X, none, row_of, slot_of, w)
    assert dYs.numel() == 0 and not dw.any()


def test_combine_gradient_against_differences(h):
    """sum(dY Y) is linear in the weights and in Ys, so differences give the gradients exactly, up to
    the bf16 rounding of Y (2^-8 of each element)."""
    T, D, k = 12, 64, 4
    M, row_of, slot_of, w = _plan(h, T, 8, k, 5)
    Ys, dY = (torch.randn(n, D, generator=_gen(n), device="cuda").bfloat16() for n in (T * k, T))
    dYs, dw = h.sq_combine_grad(dY, Ys, row_of, slot_of, w)
    value = lambda y, ww: (h.sq_combine(y, row_of, ww).double() * dY.double()).sum(1)  # noqa: E731
    noise = (2.0 ** -8) * (h.sq_combine(Ys.abs(), row_of, w + 64).double() * dY.double().abs()).sum(1)
    for j in range(k):
        up, down = w.clone(), w.clone()
        up[:, j] += 64
        down[:, j] -= 64
        diff = (value(Ys, up) - value(Ys, down)) / 128
        on = row_of[:, j] >= 0
        assert bool(((diff - dw[:, j].double()).abs() <= 2 * noise / 128 + 1e-5)[on].all())
        assert bool((dw[:, j] == 0)[~on].all())
    d = 7
    up, down = Ys.clone(), Ys.clone()
    up[:, d] += 64
    down[:, d] -= 64
    diff = (h.sq_combine(up, row_of, w).double() - h.sq_combine(down, row_of, w).double())[:, d] * dY[:, d].double()
    rows = torch.where((row_of >= 0), dYs[row_of.clamp(min=0).long(), d].double(), 0.0).sum(1) * (up - down)[0, d].double()
    # the steps' own bf16 rounding (0.25 per row and side, twice), that of Y (2^-8 of up to 68 per weight
    # and side) and that of dYs (2^-8 of 128 per weight): together below 3 per unit of weight
    size = (torch.where(row_of >= 0, w, 0.0).sum(1).double() + 1) * dY[:, d].double().abs()
    assert bool(((diff - rows).abs() <= 3 * size).all())


def test_rows_past_32_bits(h):
    """Rows whose element offsets pass 2^31 (and byte offsets 2^32)."""
    T, k, D = 4200, 8, 65536
    e = torch.arange(T * k, device="cuda", dtype=torch.int32).reshape(T, k) % 4
    offsets, row_of, slot_of = h.sq_sort_tokens(e.contiguous(), 4)
    X = (torch.arange(T, device="cuda") % 251).bfloat16()[:, None].expand(T, D).contiguous()
    Xs = h.sq_dispatch(X, row_of, slot_of)
    some = torch.cat([torch.arange(0, 64, device="cuda"), torch.arange(T * k - 64, T * k, device="cuda")])
    assert torch.equal(Xs[some, -8:], X[(slot_of[some] // k).long(), -8:])
    w = torch.full((T, k), 0.125, device="cuda")
    assert torch.equal(h.sq_combine(Xs, row_of, w), X)
    dYs, dw = h.sq_combine_grad(X, Xs, row_of, slot_of, w)
    want = (torch.arange(T, device="cuda") % 251).double() ** 2 * D
    assert bool(((dw.double() - want[:, None]).abs() <= D * 2.0 ** -24 * want[:, None]).all())
    assert torch.equal(dYs[some, -8:].float(), X[(slot_of[some] // k).long(), -8:].float() * 0.125)


def test_other_stream_and_graph(h):
    """Calls follow the stream they are given, and a captured step replays on new inputs."""
    T, E, k, D = 500, 64, 4, 520
    z = torch.randn(T, E, generator=_gen(1), device="cuda")
    X = torch.randn(T, D, generator=_gen(2), device="cuda").bfloat16()

    def step(z, X, stream=None):
        experts, weights = h.sq_route(z, k, stream=stream)
        _, row_of, slot_of = h.sq_sort_tokens(experts, E, stream=stream)
        Xs = h.sq_dispatch(X, row_of, slot_of, stream=stream)
        return h.sq_combine(Xs, row_of, weights, stream=stream)

    want = step(z, X)
    assert bool(((want.float() - X.float()).abs() <= 2.0 ** -8 * X.float().abs() + 1e-6).all())  # weights sum to 1
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert torch.equal(step(z, X), want)
        z2, X2 = torch.zeros_like(z), torch.zeros_like(X)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step(z2, X2)
    z2.copy_(z)
    X2.copy_(X)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_refusals(h):
    z = torch.zeros(4, 16, device="cuda")
    with pytest.raises(pkg.SQError, match="k="):
        h.sq_route(z, 17)
    with pytest.raises(pkg.SQError, match="E="):
        h.sq_route(torch.zeros(1, 1025, device="cuda"), 2)
    with pytest.raises(ValueError, match="logits"):
        h.sq_route(z.double(), 2)
    with pytest.raises(ValueError, match="logits"):
        h.sq_route(torch.zeros(16, 4, device="cuda").t(), 2)
    with pytest.raises(ValueError, match="valid"):
        h.sq_route(z, 2, valid=torch.ones(5, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="weights is on"):
        h.sq_route(z, 2, weights=torch.zeros(4, 2))
    with pytest.raises(ValueError, match="experts"):
        h.sq_sort_tokens(torch.zeros(4, 2, dtype=torch.int64, device="cuda"), 16)
    experts, weights = h.sq_route(z, 2)
    _, row_of, slot_of = h.sq_sort_tokens(experts, 16)
    X = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="X must"):
        h.sq_dispatch(X.float(), row_of, slot_of)
    with pytest.raises(ValueError, match="X must"):
        h.sq_dispatch(torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")[:, ::2], row_of, slot_of)
    with pytest.raises(pkg.SQError, match="D="):
        h.sq_dispatch(torch.zeros(4, 12, dtype=torch.bfloat16, device="cuda"), row_of, slot_of)
    with pytest.raises(pkg.SQError, match="R="):
        h.sq_combine(torch.zeros(9, 64, dtype=torch.bfloat16, device="cuda"), row_of, weights)
    with pytest.raises(pkg.SQError, match="16-byte"):
        h.sq_dispatch(torch.zeros(4 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(4, 64), row_of, slot_of)


def test_inputs_written_just_before_the_call(h):
    """Steps of changing sizes back to back, logits and rows written by kernels right ahead of them, give
    the bits of the same steps one by one."""
    E, k, D = 60, 4, 264
    sizes = (2000, 1, 37, 500, 1999, 8)
    zs = [torch.randn(T, E, generator=_gen(T), device="cuda") for T in sizes]
    xs = [torch.randn(T, D, generator=_gen(T + 1), device="cuda").bfloat16() for T in sizes]

    def step(z, x):
        experts, weights = h.sq_route(z, k)
        offsets, row_of, slot_of = h.sq_sort_tokens(experts, E)
        Xs = h.sq_dispatch(x, row_of, slot_of)
        Y = h.sq_combine(Xs, row_of, weights)
        dYs, dw = h.sq_combine_grad(x, Xs, row_of, slot_of, weights)
        return experts, weights, offsets, row_of, slot_of, Y, dYs, dw, h.sq_dispatch_grad(dYs, row_of), h.sq_route_grad(z, experts, dw)

    want = []
    for z, x in zip(zs, xs):
        want.append([r.clone() for r in step(z, x)])
        torch.cuda.synchronize()
    z, x = torch.empty(2000, E, device="cuda"), torch.empty(2000, D, dtype=torch.bfloat16, device="cuda")
    got = []
    for _ in range(8):
        for T, zi, xi in zip(sizes, zs, xs):
            x[:T].copy_(xi), z[:T].copy_(zi)
            got.append([r.clone() for r in step(z[:T], x[:T])])
    for i, results in enumerate(got):
        for j, (r, first) in enumerate(zip(results, want[i % len(sizes)])):
            assert torch.equal(r, first), (i, j)
