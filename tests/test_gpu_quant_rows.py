"""Activations to microscaled 4 bits and back, against the definition in 64 bits.

Every rounding of the definition is decided in exact arithmetic here (comparisons in 64 bits of
numbers that 64 bits hold exactly), so codes, scale bytes and row scales have to be equal."""
import pytest
import torch

import quant_ref as ref

pkg = pytest.importorskip("paper_2609_04526_gb300")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    return pkg.Handle()


def check(h, fmt, X, ws2=None, slot_of=None, k=1):
    q = h.sq_quantize(fmt, X, ws2=ws2, slot_of=slot_of, k=k)
    back = h.sq_dequantize(q)
    h.sq_sync()
    src = X if slot_of is None else ref.gathered(X, slot_of, k)
    codes, scales, row = ref.quantize(fmt, src.cpu(), ws2)
    assert torch.equal(q.scales.cpu(), scales)
    if q.row_ws2 is not None:
        assert torch.equal(q.row_ws2.cpu().double(), row)
    finite = ref.block_finite(fmt, src.cpu())
    same = ref.unpack(q.codes.cpu()) == codes
    assert (same | ~finite).all(), f"{int((~same & finite).sum())} codes differ"
    values = ref.values(fmt, q.codes.cpu(), q.scales.cpu())
    want = (values.float() * (row.float() if q.row_ws2 is not None else torch.tensor(1.0 if ws2 is None else ws2))[..., None]
            if q.row_ws2 is not None else values.float() * (1.0 if ws2 is None else ws2)).bfloat16()
    assert torch.equal(back.cpu().view(torch.int16)[finite], want.view(torch.int16)[finite])
    assert torch.isnan(back.cpu().float()[~finite]).all()
    return q


SHAPES = [(1, 32), (1, 4096), (3, 64), (5, 544), (187, 2720), (33, 1056), (2, 14336), (7, 16416), (1, 70016)]


@pytest.mark.parametrize("T, K", SHAPES)
@pytest.mark.parametrize("fmt, ws2", [(pkg.NVFP4, None), (pkg.NVFP4, 0.00317), (pkg.MXFP4, None)])
def test_rows_of_all_widths(h, fmt, ws2, T, K):
    g = torch.Generator(device="cuda").manual_seed(T * 7 + K)
    X = torch.randn(T, K, generator=g, device="cuda") * torch.exp(torch.randn(T, K, generator=g, device="cuda"))
    check(h, fmt, X.bfloat16(), ws2)


@pytest.mark.parametrize("fmt, ws2", [(pkg.NVFP4, None), (pkg.NVFP4, 1.0), (pkg.NVFP4, 0.25), (pkg.MXFP4, None)])
def test_values_on_the_borders(h, fmt, ws2):
    """Rows whose values lie on borders between codes: m * s with every midpoint m and E4M3 significand s."""
    check(h, fmt, ref.border_rows().cuda(), ws2)


@pytest.mark.parametrize("fmt, ws2", [(pkg.NVFP4, None), (pkg.NVFP4, 1.7), (pkg.MXFP4, None)])
def test_every_bf16_value(h, fmt, ws2):
    bits = torch.arange(65536, dtype=torch.int32)
    X = bits.to(torch.int16).view(torch.bfloat16).view(-1, 128)  # neighbours share a binade, some rows are not finite
    check(h, fmt, X.cuda(), ws2)


@pytest.mark.parametrize("ws2", [2.0 ** -126, 1e-30, 3.3e-9, 1e-3, 7.0, 1e30, 2.0 ** 126])
def test_fixed_scales_far_from_the_values(h, ws2):
    g = torch.Generator(device="cuda").manual_seed(3)
    X = torch.randn(40, 256, generator=g, device="cuda") * 10.0 ** torch.randint(-30, 30, (40, 1), generator=g, device="cuda")
    check(h, pkg.NVFP4, X.bfloat16(), ws2)


@pytest.mark.parametrize("fmt", [pkg.NVFP4, pkg.MXFP4])
def test_rows_not_finite_and_empty(h, fmt):
    g = torch.Generator(device="cuda").manual_seed(4)
    X = torch.randn(16, 320, generator=g, device="cuda").bfloat16()
    X[0] = 0
    X[1] = float("nan")
    X[2, 5], X[3, 64], X[4, 319] = float("inf"), float("-inf"), float("nan")
    X[5, 16:32] = 3.38e38
    X[6] = 1e-38
    X[7] = -0.0
    check(h, fmt, X)


@pytest.mark.parametrize("fmt", [pkg.NVFP4, pkg.MXFP4])
@pytest.mark.parametrize("k", [1, 4])
def test_rows_by_slot(h, fmt, k):
    g = torch.Generator(device="cuda").manual_seed(5)
    T, K = 50, 416
    X = torch.randn(T, K, generator=g, device="cuda").bfloat16()
    slots = torch.randperm(T * k, generator=g, device="cuda").int()
    slots[7], slots[20], slots[31] = -1, T * k, -(1 << 31)
    q = check(h, fmt, X, slot_of=slots, k=k)
    # the rows that sq_dispatch copies, quantised
    row_of = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
    on = (slots >= 0) & (slots < T * k)
    row_of[slots[on].long()] = torch.arange(T * k, device="cuda", dtype=torch.int32)[on]
    slot_of = torch.where(on, slots, -1)
    other = h.sq_quantize(fmt, h.sq_dispatch(X, row_of.view(T, k), slot_of))
    assert torch.equal(other.codes, q.codes) and torch.equal(other.scales, q.scales)


@pytest.mark.parametrize("fmt", [pkg.NVFP4, pkg.MXFP4])
@pytest.mark.parametrize("T", [3, 2000])
def test_tensors_that_start_on_16_bytes(h, fmt, T):
    """Rows read and written from a 16-byte boundary that is none of 32, and scale bytes of a slice."""
    K = 544
    g = torch.Generator(device="cuda").manual_seed(6)
    room = torch.randn(T * K + 8, generator=g, device="cuda").bfloat16()
    X = room[8:].view(T, K)
    assert X.data_ptr() % 32 == 16
    q = check(h, fmt, X)
    back = torch.empty(T * K + 8, dtype=torch.bfloat16, device="cuda")[8:].view(T, K)
    assert torch.equal(h.sq_dequantize(q, X=back), h.sq_dequantize(q))
    part = pkg.QuantRows(fmt, T - 1, K, q.codes[1:], q.scales[1:], 1.0, None if q.row_ws2 is None else q.row_ws2[1:])
    assert part.scales.data_ptr() % 16 != 0
    assert torch.equal(h.sq_dequantize(part), h.sq_dequantize(q)[1:])
    codes = torch.randint(0, 256, (136, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.full((136, K // ref.BLOCK[fmt]), 0x38 if fmt == pkg.NVFP4 else 120, dtype=torch.uint8, device="cuda")
    w = pkg.QuantWeight(fmt, 136, K, codes, scales, 1.0)
    assert torch.equal(h.sq_quant_fwd(w, part), h.sq_quant_fwd(w, pkg.QuantRows(fmt, T - 1, K, part.codes, part.scales.clone(), 1.0, part.row_ws2)))


def test_no_tokens_but_rows_by_slot(h):
    q = h.sq_quantize(pkg.NVFP4, torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"),
                      slot_of=torch.zeros(5, dtype=torch.int32, device="cuda"), k=2)
    assert (h.sq_dequantize(q) == 0).all() and (q.scales == 1).all()


def test_tensors_elsewhere_are_refused(h):
    X = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    q = h.sq_quantize(pkg.NVFP4, X)
    host = pkg.QuantWeight(pkg.NVFP4, 16, 64, torch.zeros(16, 32, dtype=torch.uint8), torch.zeros(16, 4, dtype=torch.uint8), 1.0)
    with pytest.raises(ValueError, match="w.codes"):
        h.sq_quant_fwd(host, q)
    with pytest.raises(ValueError, match="slot_of"):
        h.sq_quantize(pkg.NVFP4, X, slot_of=torch.zeros(4, dtype=torch.int32))
    gw = pkg.GroupedWeight(pkg.NVFP4, 2, 16, 64, torch.zeros(2, 16, 32, dtype=torch.uint8, device="cuda"),
                           torch.zeros(2, 16, 4, dtype=torch.uint8, device="cuda"), [1.0, 1.0])
    with pytest.raises(ValueError, match="w.ws2"):
        h.sq_grouped_quant_fwd(gw, torch.zeros(3, dtype=torch.int64, device="cuda"), q)
    gw.ws2 = torch.ones(2, device="cuda")
    with pytest.raises(ValueError, match="offsets"):
        h.sq_grouped_quant_fwd(gw, torch.zeros(3, dtype=torch.int64), q)
    with pytest.raises(pkg.SQError, match="format"):
        h.sq_quant_fwd(pkg.QuantWeight(pkg.MXFP4, 16, 64, gw.codes[0], torch.zeros(16, 2, dtype=torch.uint8, device="cuda"), 1.0), q)


@pytest.mark.parametrize("fmt, ws2", [(pkg.NVFP4, None), (pkg.NVFP4, 0.00317), (pkg.MXFP4, None)])
@pytest.mark.parametrize("T, K", [(2100, 5024), (1500, 14336), (330000, 32), (5, 4194400)])
def test_many_values(h, fmt, ws2, T, K):
    """So many that rows without scales of their own are cut evenly, with a last piece that is shorter; from 16 bytes
    that are no boundary of 32 too. Infinite and empty blocks stay where they are."""
    g = torch.Generator(device="cuda").manual_seed(T)
    room = torch.randn(T * K + 8, generator=g, device="cuda").bfloat16()
    for X in (room[8:].view(T, K), room[:T * K].view(T, K)):
        X[T // 2, K - 1], X[T // 3, :32], X[T - 1, K - 32:] = float("inf"), 0, -0.0
        q = h.sq_quantize(fmt, X, ws2)
        few = [q]
        for lo in (0, T // 3, T - 2):  # a few rows alone, cut by rows
            part = h.sq_quantize(fmt, X[lo:lo + 2], ws2)
            few.append(part)
            assert torch.equal(q.codes[lo:lo + 2], part.codes) and torch.equal(q.scales[lo:lo + 2], part.scales)
        back = h.sq_dequantize(q, X=torch.empty(T * K + 8, dtype=torch.bfloat16, device="cuda")[8:].view(T, K))
        for lo, part in zip((0, T // 3, T - 2), few[1:]):
            rows = h.sq_dequantize(part)
            assert torch.equal(back[lo:lo + 2].nan_to_num(7), rows.nan_to_num(7)) and torch.equal(back[lo:lo + 2].isnan(), rows.isnan())
        if T * K < 12e6:
            check(h, fmt, X, ws2)
    h.sq_sync()
