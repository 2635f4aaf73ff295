"""The measured cases of the 4-bit operators: rows to and from microscaled FP4, and the products of
such rows with FP4 weights, dense and grouped by expert.

Kinds of case:

  rows     bf16 rows quantised to E2M1 codes with a scale byte for each block (NVFP4: blocks of 16,
           E4M3 scales under an fp32 scale that is given or found for each row; MXFP4: blocks of 32,
           E8M0 scales) and read back as bf16: how a training step keeps activations in 4 bits
  linear   a linear layer with both operands in FP4: bf16 rows quantised, then multiplied with the
           weight's codes and scales
  experts  the same through the experts of an MoE layer: tokens quantised into their experts' rows
           (sorted by expert, ragged counts, the offsets on the device), then each expert's product.
           Rows behind the last routed one keep what they held

Shapes are the package's synthetic workloads' (a decoder layer of width 4096 and 14336, 128 experts
of 768 x 2048 routed top-8 and of 2880 x 2880 routed top-4, batches of 16 x 2048 tokens) and generic
ones of the same range.
"""
import math

import torch

own = False

NVFP4, MXFP4 = 0, 1
BLOCK = (16, 32)


def listed():
    return [
        # the rows of one decoded token: launches and host calls count
        {"name": "rows_token", "kind": "rows", "fmt": NVFP4, "T": 1, "K": 4096, "fixed": False},
        # one short example, width not a multiple of 64
        {"name": "rows_example", "kind": "rows", "fmt": MXFP4, "T": 187, "K": 2720, "fixed": False},
        # one 2048-token sequence behind an MLP's first half, with a scale fixed by calibration
        {"name": "rows_seq", "kind": "rows", "fmt": NVFP4, "T": 2048, "K": 14336, "fixed": True},
        # the layer input of the full 16 x 2048 batch, kept in 4 bits for the backward pass
        {"name": "rows_batch", "kind": "rows", "fmt": NVFP4, "T": 32768, "K": 4096, "fixed": False},
        # one token through a square linear: the weight is read once
        {"name": "linear_token", "kind": "linear", "fmt": NVFP4, "T": 1, "N": 4096, "K": 4096, "fixed": False},
        # a batch of decoded tokens through an MLP's first half
        {"name": "linear_decode", "kind": "linear", "fmt": MXFP4, "T": 48, "N": 14336, "K": 4096, "fixed": False},
        # one short example, odd sizes
        {"name": "linear_example", "kind": "linear", "fmt": NVFP4, "T": 187, "N": 1048, "K": 2720, "fixed": True},
        # one sequence through an MLP's second half
        {"name": "linear_seq", "kind": "linear", "fmt": NVFP4, "T": 2048, "N": 4096, "K": 14336, "fixed": False},
        # eight sequences through its first half: a prompt batch of a served model
        {"name": "linear_batch", "kind": "linear", "fmt": NVFP4, "T": 16384, "N": 14336, "K": 4096, "fixed": False},
        # one token through the 8 experts it chose
        {"name": "experts_token", "kind": "experts", "fmt": NVFP4, "T": 1, "E": 128, "k": 8, "N": 768, "K": 2048, "pad": 0.0, "fixed": False},
        # one sequence, some of it padding: about 128 rows for each expert
        {"name": "experts_seq", "kind": "experts", "fmt": NVFP4, "T": 2048, "E": 128, "k": 8, "N": 768, "K": 2048, "pad": 0.05, "fixed": False},
        # four sequences without their padding through wide experts
        {"name": "experts_batch", "kind": "experts", "fmt": MXFP4, "T": 8111, "E": 128, "k": 4, "N": 2880, "K": 2880, "pad": 0.0, "fixed": False},
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(("rows", "linear", "linear", "experts", "experts"))
    fmt = rng.choice((NVFP4, MXFP4))
    c = {"kind": kind, "fmt": fmt, "fixed": fmt == NVFP4 and rng.random() < 0.3}
    if kind == "rows":
        K = 32 * int(_log(rng, 8, 448.5))
        return {**c, "T": int(_log(rng, 1, 32768 * 4096 // K + 0.5)), "K": K}
    if kind == "linear":
        N, K = 8 * int(_log(rng, 32, 1792.5)), 32 * int(_log(rng, 8, 448.5))
        return {**c, "T": int(_log(rng, 1, min(16384, 16384 * 14336 * 4096 // (N * K)) + 0.5)), "N": N, "K": K}
    E, k = rng.choice((8, 16, 60, 64, 128)), rng.choice((1, 2, 4, 6, 8))
    N, K = 8 * int(_log(rng, 32, 512.5)), 32 * int(_log(rng, 8, 128.5))
    most = min(16384, 8111 * 4 * 2880 * 2880 // (k * N * K))
    return {**c, "T": int(_log(rng, 1, most + 0.5)), "E": E, "k": k, "N": N, "K": K, "pad": rng.choice((0.0, 0.05, 0.3))}


# ------------------------------------------------------------------ inputs

def _acts(g, T, K):
    """Activations: a few channels far larger than the others, rows of unequal size."""
    channel = torch.exp(0.7 * torch.randn(K, generator=g, device="cuda"))
    row = torch.exp(0.4 * torch.randn(T, 1, generator=g, device="cuda"))
    return (torch.randn(T, K, generator=g, device="cuda") * channel * row).bfloat16()


def _weight(g, fmt, E, N, K):
    """Codes [E, N, K/2], scale bytes [E, N, K/B] and tensor scales [E] of a checkpoint's weights."""
    codes = torch.randint(0, 256, (E, N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    G = K // BLOCK[fmt]
    if fmt == NVFP4:  # E4M3 from 0.5 to just below 8
        scales = torch.randint(0x30, 0x50, (E, N, G), generator=g, device="cuda", dtype=torch.uint8)
        ws2 = (0.5 + torch.rand(E, generator=g, device="cuda")) * (0.1 / math.sqrt(K))
    else:  # E8M0: powers of two around the size of the weights
        mid = 126 - int(0.5 * math.log2(K))
        scales = torch.randint(mid - 2, mid + 1, (E, N, G), generator=g, device="cuda", dtype=torch.uint8)
        ws2 = torch.ones(E, device="cuda")
    return codes, scales, ws2


def _rows_by_expert(g, T, E, k, pad):
    """Sorted routing of T tokens to k experts each, experts of unequal popularity: the E + 1 offsets
    and each row's slot t * k + j (-1 past the last routed one)."""
    z = torch.randn(T, E, generator=g, device="cuda") + 0.3 * torch.randn(E, generator=g, device="cuda")
    experts = torch.topk(z, k, dim=1).indices
    on = torch.rand(T, generator=g, device="cuda") >= pad
    on[:1] = True
    key = torch.where(on[:, None], experts, E).reshape(-1)
    order = torch.argsort(key, stable=True)
    ends = torch.searchsorted(key[order].contiguous(), torch.arange(E + 1, device="cuda"))
    offsets = ends.to(torch.int64)
    rows = torch.arange(T * k, device="cuda")
    return offsets, torch.where(rows < offsets[E], order, -1).int()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    fmt, T, K = case["fmt"], case["T"], case["K"]
    G = K // BLOCK[fmt]
    s["X"] = _acts(g, T, K)
    # a calibrated scale: the largest value that was seen, here a little below some of the batch
    s["xs2"] = 0.9 * float(s["X"].abs().max()) / (6 * 448) if case["fixed"] else None
    R = T * case.get("k", 1)
    dev = "cuda"
    s["codes"] = torch.empty(R, K // 2, dtype=torch.uint8, device=dev)
    s["scales"] = torch.empty(R, G, dtype=torch.uint8, device=dev)
    s["row_ws2"] = torch.empty(R, device=dev) if fmt == NVFP4 and not case["fixed"] else None
    if case["kind"] == "rows":
        s["back"] = torch.empty(T, K, dtype=torch.bfloat16, device=dev)
        return s
    if case["kind"] == "experts":
        s["offsets"], s["slot_of"] = _rows_by_expert(g, T, case["E"], case["k"], case["pad"])
        s["bounds"] = s["offsets"].tolist()  # the plain form's loop over the experts
    s["wcodes"], s["wscales"], s["wws2"] = _weight(g, fmt, case.get("E", 1), case["N"], K)
    s["ws2"] = s["wws2"].tolist()
    s["Y"] = torch.zeros(R, case["N"], dtype=torch.bfloat16, device=dev)
    return s


# ------------------------------------------------------------------ one pass

_handle = None


def _h():
    """The one handle a program keeps."""
    global _handle
    if _handle is None:
        import paper_2609_04526_gb300 as pkg
        _handle = pkg.Handle()
    return _handle


def run(s):
    if own:
        return _run_own(s)
    if s["kind"] == "rows":
        values, row_ws2 = _quantize(s["fmt"], s["X"], s["xs2"])
        out = {"values": (values * row_ws2[:, None]).bfloat16()}
        if s["row_ws2"] is not None:
            out["row_ws2"] = row_ws2
        return out
    if s["kind"] == "linear":
        values, row_ws2 = _quantize(s["fmt"], s["X"], s["xs2"])
        w = _decode(s["fmt"], s["wcodes"][0], s["wscales"][0])
        return {"Y": (values @ w.t() * s["ws2"][0] * row_ws2[:, None]).bfloat16()}
    slot = s["slot_of"].long()
    token = torch.div(slot.clamp(min=0), s["k"], rounding_mode="floor")
    X = torch.where((slot >= 0)[:, None], s["X"][token], 0.0)
    values, row_ws2 = _quantize(s["fmt"], X, s["xs2"])
    Y = torch.zeros(X.shape[0], s["N"], dtype=torch.bfloat16, device=X.device)
    for e, (lo, hi) in enumerate(zip(s["bounds"], s["bounds"][1:])):
        if hi > lo:
            w = _decode(s["fmt"], s["wcodes"][e], s["wscales"][e])
            Y[lo:hi] = (values[lo:hi] @ w.t() * s["wws2"][e] * row_ws2[lo:hi, None]).bfloat16()
    return {"Y": Y}


def _run_own(s):
    import paper_2609_04526_gb300 as pkg
    h = _h()
    fmt, K = s["fmt"], s["K"]
    q = pkg.QuantRows(fmt, s["codes"].shape[0], K, s["codes"], s["scales"], s["xs2"] or 1.0, s["row_ws2"])
    if s["kind"] == "rows":
        h.sq_quantize(fmt, s["X"], ws2=s["xs2"], out=q)
        h.sq_dequantize(q, X=s["back"])
        return {"values": s["back"]} if q.row_ws2 is None else {"values": s["back"], "row_ws2": q.row_ws2}
    if s["kind"] == "linear":
        h.sq_quantize(fmt, s["X"], ws2=s["xs2"], out=q)
        w = pkg.QuantWeight(fmt, s["N"], K, s["wcodes"][0], s["wscales"][0], s["ws2"][0])
        h.sq_quant_fwd(w, q, Y=s["Y"])
        return {"Y": s["Y"]}
    h.sq_quantize(fmt, s["X"], ws2=s["xs2"], slot_of=s["slot_of"], k=s["k"], out=q)
    w = pkg.GroupedWeight(fmt, s["E"], s["N"], K, s["wcodes"], s["wscales"], s["wws2"])
    h.sq_grouped_quant_fwd(w, s["offsets"], q, Y=s["Y"])
    return {"Y": s["Y"]}


# ------------------------------------------------------------------ plain forms

def _power(e):
    """2^e in fp32 of whole exponents -127 .. 127, exactly."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).int().view(torch.float32)


def _round(x, steps, lowest):
    """x >= 0 to the nearest number of `steps` mantissa steps (8 for E4M3, 2 for E2M1) and at least
    the exponent `lowest`, ties to even."""
    _, e = torch.frexp(x)
    ulp = _power((e - 1).clamp(min=lowest)) / steps
    return torch.round(x / ulp) * ulp


def _quantize(fmt, X, ws2):
    """The values of the rows' codes under their block scales, fp32 [R, K], and each row's scale
    above those, fp32 [R]. The steps are exact in 32 bits or, as quotients, never round onto a border
    between two codes or scales that they do not lie on."""
    x = X.float()
    R, K = x.shape
    one = torch.ones(R, device=x.device)
    if fmt == MXFP4:
        row = one
    elif ws2 is not None:
        row = one * ws2
        x = x * (1.0 / row)[:, None]
    else:  # the smallest power of two, of at least 2^-116, that brings the row's largest to 6 * 448
        m, e = torch.frexp(x.abs().amax(1))
        e = e - 12 + (m > 0.65625).int()
        row = _power(e.clamp(min=-116))
        x = x / row[:, None]
    x = x.view(R, K // BLOCK[fmt], BLOCK[fmt])
    top = x.abs().amax(2, keepdim=True)
    if fmt == MXFP4:
        _, e = torch.frexp(top)
        scale = _power((e - 3).clamp(min=-127))
    else:
        scale = _round(top / 6, 8, -6).clamp(min=2.0 ** -9, max=448.0)
    code = _round((x.abs() / scale).clamp(max=6.0), 2, 0).clamp(max=6.0)
    return (torch.copysign(code, x) * scale).view(R, K), row


def _decode(fmt, codes, scales):
    """The values of packed codes [N, K/2] under their scale bytes [N, K/B], fp32 [N, K]."""
    N = codes.shape[0]
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                         device=codes.device)
    c = table[torch.stack([codes & 15, codes >> 4], 2).view(N, -1).int()]
    b = scales.int()
    if fmt == MXFP4:
        s = _power(b - 127)
    else:
        e, m = (b >> 3) & 15, (b & 7).float()
        s = torch.where(e > 0, (1 + m / 8) * _power(e - 7), m * 2.0 ** -9)
        s = torch.where(b >= 128, -s, s)
    return (c.view(N, -1, BLOCK[fmt]) * s[:, :, None]).view(N, -1)


# ------------------------------------------------------------------ work and exact results

def _bytes(fmt, values):
    """Codes and scale bytes of so many values."""
    return values / 2 + values / BLOCK[fmt]


def work(case):
    fmt, T, K = case["fmt"], case["T"], case["K"]
    if case["kind"] == "rows":
        # rows read, codes and scales written; those read, rows written
        return {"bytes": 4.0 * T * K + 2 * _bytes(fmt, T * K), "flops": 6.0 * T * K}
    N = case["N"]
    if case["kind"] == "linear":
        return {"bytes": 2.0 * T * K + _bytes(fmt, N * K) + 2.0 * T * N, "flops": 2.0 * T * N * K}
    E, k = case["E"], case["k"]
    on = max(1.0, T * (1.0 - case["pad"]))
    experts = E * (1.0 - (1.0 - k / E) ** on)  # that a row reaches, of equally popular ones
    return {"bytes": 2.0 * on * K + 4.0 * T * k + 8.0 * (E + 1) + experts * _bytes(fmt, N * K) + 2.0 * on * k * N,
            "flops": 2.0 * on * k * N * K}


def exact(case, seed):
    s = prepare(case, seed)
    fmt, B = case["fmt"], BLOCK[case["fmt"]]
    R = case["T"] * case.get("k", 1)
    if 2.0 * R * case.get("N", 1) * case["K"] > 1e13:
        return None  # 64-bit products of this size take too long
    dev = "cuda"
    e2m1 = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=dev)
    e4m3 = torch.tensor([(1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 7) if b >= 8 else b * 2.0 ** -9 for b in range(127)],
                        dtype=torch.float64, device=dev)

    powers = torch.tensor([2.0 ** i for i in range(-127, 128)], dtype=torch.float64, device=dev)

    def nearest(table, x):
        """Index of the table's entry nearest to x >= 0, the even one of two as near."""
        mid = (table[1:] + table[:-1]) / 2
        above = torch.searchsorted(mid, x, right=False)  # borders below x
        tie = (above < len(mid)) & (mid[above.clamp(max=len(mid) - 1)] == x)
        return torch.where(tie & (above % 2 == 1), above + 1, above)

    def quantized(rows):
        """Values of some bf16 rows under their block scales, and their row scales, in 64 bits."""
        x = rows.double()
        n = len(rows)
        if fmt == MXFP4:
            row = torch.ones(n, 1, dtype=torch.float64, device=dev)
        elif case["fixed"]:
            row = torch.full((n, 1), s["xs2"], dtype=torch.float32, device=dev).double()
            inverse = (1.0 / row).float().double()
            x = (x * inverse).float().double()  # rounded to 32 bits once, by definition
        else:
            most = x.abs().max(1, keepdim=True).values
            up = torch.tensor([2.0 ** i for i in range(-116, 129)], dtype=torch.float64, device=dev)
            row = up[torch.searchsorted(2688 * up, most)]
            x = x / row
        x = x.view(n, -1, B)
        top = x.abs().max(2, keepdim=True).values
        if fmt == MXFP4:
            scale = powers[(torch.searchsorted(4 * powers, top, right=True) - 1).clamp(min=0)]  # top in [4, 8) scales
        else:
            scale = e4m3[nearest(6 * e4m3, top).clamp(min=1)]
        return (torch.sign(x) * e2m1[nearest(e2m1, x.abs() / scale)] * scale).view(n, -1), row

    def weight(e):
        c = s["wcodes"][e].long()
        c = torch.stack((c % 16, c // 16), dim=-1).flatten(1)
        b = s["wscales"][e].long()
        scale = powers[b] if fmt == MXFP4 else e4m3[b]
        value = e2m1[c % 8] * (1 - 2 * (c // 8))
        return value.view(len(b), -1, B).mul(scale[..., None]).flatten(1) * s["wws2"][e].double()

    if case["kind"] == "rows":
        parts = [quantized(s["X"][i:i + 2048]) for i in range(0, R, 2048)]
        out = {"values": torch.cat([v * r for v, r in parts])}
        if s["row_ws2"] is not None:
            out["row_ws2"] = torch.cat([r[:, 0] for _, r in parts])
        return out
    Y = torch.zeros(R, case["N"], dtype=torch.float64, device=dev)
    if case["kind"] == "linear":
        W = weight(0)
        for i in range(0, R, 2048):
            v, r = quantized(s["X"][i:i + 2048])
            Y[i:i + 2048] = torch.mm(v, W.T) * r
        return {"Y": Y}
    for e in range(case["E"]):
        lo, hi = s["bounds"][e], s["bounds"][e + 1]
        if hi > lo:
            v, r = quantized(s["X"][s["slot_of"][lo:hi].long() // case["k"]])
            Y[lo:hi] = torch.mm(v, weight(e).T) * r
    return {"Y": Y}
