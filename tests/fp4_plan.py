"""Which kernel, tiles and ring a product with both operands in 4 bits gets: fp4_plan of csrc/sq_internal.h compiled
into a small program, for tests that need a certain plan."""
import atexit
import functools
import os
import shutil
import subprocess
import tempfile
from collections import namedtuple

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_04526_gb300", "csrc")
CUDA_INC = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
SMS = 152
# clusters of 1 .. 8 CTAs of the few-token kernel that a GB300 of 152 SMs says it runs at once
CLUSTERS = (152, 76, 46, 36, 28, 23, 15, 15)

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include "sq_internal.h"
int main() {
  sqi::Fp4Clusters fit = {};
  fit.alone[0] = 1;
  for (int c = 1; c <= 8; ++c) {
    if (std::scanf("%d", &fit.alone[c]) != 1) return 1;
    fit.shared[c] = fit.alone[c];
  }
  long long fmt, R, E, N, K;
  while (std::scanf("%lld %lld %lld %lld %lld", &fmt, &R, &E, &N, &K) == 5) {
    static const int64_t offsets[1] = {0};
    sqi::Fp4Args p = {};
    p.R = R;
    p.E = E ? (int)E : 1;
    p.N = (int)N;
    p.K = (int)K;
    p.G = (int)(K / (fmt == 0 ? 16 : 32));
    p.offsets = E ? offsets : nullptr;  // only looked at
    sqi::fp4_plan((int)fmt, SMS, fit, p);
    std::printf("%d %d %lld %d %d %d %d\n", p.pair, p.tile_tokens, (long long)p.units, p.splits, p.stages, p.pair ? p.slices : 1,
                p.pair ? p.depth : (int)((K + 255) / 256));
  }
  return 0;
}
"""

# pair: the kernel of CTA pairs; units: tiles; depth: stages of a tile's contraction (of all parts); raw: scale bytes
# come by TMA (few-token kernel)
Plan = namedtuple("Plan", "pair tile_tokens units splits stages slices depth raw")


@functools.lru_cache(maxsize=1)
def _program():
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None or not os.path.exists(os.path.join(CUDA_INC, "cuda.h")):
        return None
    d = tempfile.mkdtemp(prefix="fp4_plan")
    atexit.register(shutil.rmtree, d, True)
    src, exe = os.path.join(d, "fp4_plan.cpp"), os.path.join(d, "fp4_plan")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", f"-DSMS={SMS}", f"-I{CSRC}", f"-I{CUDA_INC}", src, "-o", exe], check=True)
    return exe


def plan(fmt, R, N, K, E=0):
    """Plan of a product of R rows with one weight [N, K] or with E experts; None without a host compiler."""
    if _program() is None:
        return None
    text = " ".join(map(str, CLUSTERS)) + f"\n{fmt} {R} {E} {N} {K}\n"
    out = subprocess.run([_program()], input=text, capture_output=True, text=True, check=True).stdout.split()
    v = [int(x) for x in out]
    return Plan(bool(v[0]), *v[1:], raw=K // (16, 32)[fmt] % 16 == 0)
