"""The 4-bit formats by their definition, in 64 bits on the host."""
import torch

BLOCK = (16, 32)
E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
E4M3 = torch.tensor([(1 + b % 8 / 8) * 2.0 ** (b // 8 - 7) if b >= 8 else b * 2.0 ** -9 for b in range(127)],
                    dtype=torch.float64)
POWERS = torch.tensor([2.0 ** i for i in range(-127, 128)], dtype=torch.float64)


def nearest(table, x, unit=1.0):
    """Index of the entry of table * unit nearest to x >= 0, the even one of two as near: x is compared with
    (the sum of neighbours) * unit / 2, a product that 64 bits hold exactly."""
    index = torch.zeros_like(x, dtype=torch.int64)
    for i in range(len(table) - 1):
        border = (table[i] + table[i + 1]) / 2 * unit
        index += (x > border) | ((x == border) & (i % 2 == 1))
    return index


def gathered(X, slot_of, k):
    """Row r is X[slot_of[r] // k], zeros where there is no such slot."""
    s = slot_of.long()
    on = (s >= 0) & (s < len(X) * k)
    return torch.where(on[:, None], X[torch.where(on, s, 0) // k], torch.zeros_like(X[:1]))


def block_finite(fmt, X):
    """Which values lie in blocks without infinities and NaN, [R, K]."""
    B = BLOCK[fmt]
    ok = torch.isfinite(X.float()).view(len(X), -1, B).all(2, keepdim=True)
    return ok.expand(-1, -1, B).reshape(X.shape)


def quantize(fmt, X, ws2=None):
    """Codes [R, K] (0 .. 15), scale bytes [R, K/B] u8 and row scales [R] of bf16 rows on the host."""
    R, K = X.shape
    B = BLOCK[fmt]
    finite = block_finite(fmt, X)
    x = torch.where(finite, X.double(), 0.0)
    row = torch.ones(R, dtype=torch.float64)
    if fmt == 0 and ws2 is None:
        up = torch.tensor([2.0 ** i for i in range(-116, 120)], dtype=torch.float64)
        most = x.abs().amax(1) if K else row * 0
        row = up[torch.searchsorted(up * 2688, most)]
        x = x / row[:, None]
    elif fmt == 0:
        inverse = float(torch.tensor(1.0) / torch.tensor(ws2, dtype=torch.float32))
        x = (x * inverse).clamp(-3e38, 3e38).float().double()  # a product of 8 and 24 bits, rounded to 24 once
    x = x.view(R, -1, B)
    top = x.abs().amax(2, keepdim=True)
    if fmt == 0:
        byte = nearest(E4M3, top, 6.0).clamp(min=1)
        s = E4M3[byte]
        byte[~finite.view(R, -1, B)[..., :1]] = 0x7F
    else:
        byte = (torch.searchsorted(4 * POWERS, top, right=True) - 1).clamp(min=0)
        s = POWERS[byte]
        byte[~finite.view(R, -1, B)[..., :1]] = 0xFF
    code = nearest(E2M1, x.abs(), s) + 8 * torch.signbit(X.float()).view(R, -1, B)
    return code.view(R, K), byte.view(R, -1).to(torch.uint8), row


def unpack(codes):
    """Packed codes [..., K/2] to [..., K], the even one in the low nibble."""
    c = codes.long()
    return torch.stack([c & 15, c >> 4], -1).flatten(-2)


def scale_values(fmt, scales):
    b = scales.long()
    if fmt == 1:
        return torch.where(b == 255, torch.nan, POWERS[b.clamp(max=254)])
    v = torch.where(b % 128 == 127, torch.nan, E4M3[(b % 128).clamp(max=126)])
    return torch.where(b >= 128, -v, v)


def values(fmt, codes, scales):
    """Codes times block scales, [..., K] in 64 bits."""
    c = unpack(codes)
    v = E2M1[c % 8] * (1 - 2 * (c // 8))
    B = BLOCK[fmt]
    return (v.unflatten(-1, (-1, B)) * scale_values(fmt, scales)[..., None]).flatten(-2)


def border_rows():
    """bf16 rows of 64 that hold, block by block, 6 * s and m * s, -m * s and their neighbours for every
    midpoint m of E2M1 and significand s of E4M3 over several binades."""
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    rows = []
    for e in (-9, -4, 0, 5):
        for m8 in range(8, 16):
            s = m8 / 8 * 2.0 ** e
            for i in range(0, 7):
                near = torch.tensor([mids[i] * s], dtype=torch.bfloat16)
                bits = near.view(torch.int16)
                vals = [6 * s] + [float((bits + d).view(torch.bfloat16)) for d in (-2, -1, 0, 1, 2)]
                vals += [-v for v in vals[1:]] + [m * s for m in mids[:5]]
                rows.append(vals[:16] * 4)
    return torch.tensor(rows, dtype=torch.float64).bfloat16()
