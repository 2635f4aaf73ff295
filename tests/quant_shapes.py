"""Sizes of 4-bit products that tests rely on for what they make of the kernels, with the plan they are there for
(tests/test_quant_plans.py holds them to it). Dense: (fmt, R, N, K). By expert: (fmt, counts, N, K)."""

NVFP4, MXFP4 = 0, 1
FORMATS = (NVFP4, MXFP4)


def _ragged(rows, experts):
    """About `rows` rows, unequal, one expert of eight without any."""
    return [0 if e % 8 == 5 else rows // experts + (e * 5) % 9 - 4 for e in range(experts)]


# few-token kernel, rings of 3 slots that a CTA goes through more than once; scale bytes by TMA and by warps
THREE_SLOTS = [(fmt, _ragged(1000, 8), 2600, K) for fmt in FORMATS for K in (2048, 2080, 4128)]
THREE_SLOTS_DENSE = [(fmt, 1900, 2056, 2048) for fmt in FORMATS] + [(fmt, 400, 9000, 1056) for fmt in FORMATS]
# ... of 5, scale bytes by TMA and by warps
FIVE_SLOTS = [(fmt, [1 + e % 2 for e in range(60)], 520, K) for fmt in FORMATS for K in (4096, 4128)]
# pair kernel by expert: several tiles of a CTA pair
PAIR_EXPERTS = [(fmt, [2000, 0, 2500, 1500], 2056, 544) for fmt in FORMATS]
# pair kernel, tiles of 240 or 256 rows, three and more of them for some CTA pairs; one or (MXFP4) two slices a stage
TALL = [(fmt, R, N, K) for fmt in FORMATS for R, N, K in ((704, 15616, 2080), (720, 15616, 4128), (461, 38216, 2080))]
# ... with a last tile of 32 rows or fewer, two tiles of a CTA pair
TALL_AND_SHORT = [(NVFP4, 3361, 2552, 2880), (MXFP4, 4638, 1824, 8224)]
# one part of the contraction, thousands of steps long
LONG = [(NVFP4, 1500, 2600, 1 << 18), (MXFP4, 1500, 2600, 1 << 18)]
