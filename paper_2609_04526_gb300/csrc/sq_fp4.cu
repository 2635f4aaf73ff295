// Products of FP4 rows with FP4 weights (sm_103a), dense and grouped by expert:
//
//   Y[m, n] = ws2 row[m] sum_b sx[m, b] sw[n, b] sum_{k in b} cx[m, k] cw[n, k]
//
// on tcgen05.mma with block scales: codes go from memory to the tensor cores as they are, packed two
// to a byte, and the tensor cores apply the scale bytes of both operands to each block's products
// before they add them up in fp32. What is left to the SM is to bring the scale bytes, row-major
// planes in memory, into the order that the tensor cores read: atoms of 128 rows x 4 bytes, the words
// of rows l, l + 32, l + 64 and l + 96 side by side in line l. For many tokens a launch ahead lays both
// planes out as atoms, which TMA then brings like the codes; for few, TMA brings 16 bytes of each row
// and a warp turns them into atoms, in place, or, where rows are not whole 16-byte pieces (K / 16 or K /
// 32 not a multiple of 16) and have no TMA descriptor, loads them itself. (A stage of many tokens takes 550
// to 650 cycles with atoms; turned by a warp 750, whatever its MMAs; loaded by warps 1,600: such loads take 37
// wavefronts each, the lanes' rows being different lines, and the proxy fence behind the atoms waits for the
// loads that run ahead. So where warps load it is the reader that executes the fence, behind the barrier.)
//
// The tensor cores take E4M3 scales without a sign. A negative scale byte (training may drive one below
// zero) goes in as its magnitude, and the codes of its block, in shared memory by then, change their
// signs.
//
// A stage is a slice of the contraction 256 deep, 128 bytes of codes and 16 (NVFP4) or 8 (MXFP4) scale bytes of
// each row, or, in most dense products of the pair kernel, two slices (fp4_plan).
#include <type_traits>

#include "sq_gemm_kernels.cuh"
#include "sq_launch.cuh"

namespace sqi {
namespace {

constexpr int kDeep = 256;                 // contraction of a slice
constexpr int kAtom = 512;                 // bytes of a scale atom
template <int FMT>
struct Fp4 {
  static constexpr int kBlock = FMT == 0 ? 16 : 32;
  static constexpr int kBytes = kDeep / kBlock;  // scale bytes of a row and stage
  static constexpr int kWords = kBytes / 4;      // atoms of 128 rows and a stage: one per 64 (NVFP4) or 128 of its depth
};
constexpr int kSpan = 16;                  // scale bytes of a row that a TMA box brings (MXFP4: those of two stages)
constexpr int kScales = 128 * kSpan;       // ... of 128 rows, and the room of their atoms

// Instruction descriptor of block-scaled FP4 products: E2M1 operands (bits 7-9 and 10-12 = 1), N >> 3 in
// bits 17-22, scales E8M0 (bit 23) or E4M3, M >> 4 in bits 24-28, and which of a word's scale bytes an
// MMA of depth 64 begins with, of B in bits 4-5 and of A in 29-30 (MXFP4: two of four).
template <int FMT>
__host__ __device__ constexpr uint32_t idesc_fp4(int M, int N, int byte) {
  return (static_cast<uint32_t>(byte) << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(N >> 3) << 17) |
         (FMT == 1 ? 1u << 23 : 0u) | (static_cast<uint32_t>(M >> 4) << 24) | (static_cast<uint32_t>(byte) << 29);
}

// An atom in shared memory for tcgen05.cp: 8-row groups of 16-byte lines, 128 bytes apart, no swizzle.
__device__ __forceinline__ uint64_t atom_desc(uint32_t saddr) {
  return static_cast<uint64_t>((saddr >> 4) & 0x3FFFu) | (static_cast<uint64_t>(1) << 16) |
         (static_cast<uint64_t>(128 >> 4) << 32) | (static_cast<uint64_t>(1) << 46);
}

// One atom to 4 columns of tensor memory, the same in all four lane quadrants, and a product of depth 64,
// by an elected lane of a converged warp.
__device__ __forceinline__ void atom_to_tmem_elect(uint32_t taddr, uint64_t desc) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "@e tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(taddr),
      "l"(desc)
      : "memory");
}
template <int FMT>
__device__ __forceinline__ void umma_fp4_elect(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa,
                                               uint32_t sb, uint32_t accumulate) {
  if (FMT == 0)
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "elect.sync _|e, 0xFFFFFFFF;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "elect.sync _|e, 0xFFFFFFFF;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
}

// A bounded wait of a whole warp without a call and with votes for its branches. In a loop around a call,
// or one that lanes might leave apart, the compiler keeps the MMAs' descriptors in ordinary registers and
// moves them to the uniform ones at every use: an instruction then takes 30 cycles to issue, not 8. The
// MMA warps for that reason go on after a wait that ran out: they issue what is left (on whatever the
// shared memory holds), every later wait returns at once, and the error word is set.
// CLUSTER: for a barrier that threads of the peer CTA arrive on or signal. They release at cluster scope, and
// only an acquire at that scope, in whichever CTA, orders what follows behind what they did.
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_test(uint64_t *bar, uint32_t parity) {
  return CLUSTER ? mbar_test_wait_cluster(bar, parity) : mbar_test_wait(bar, parity);
}
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, volatile int *abort_flag, int *err) {
  if (__all_sync(0xFFFFFFFFu, warp_test<CLUSTER>(bar, parity))) return true;
  const unsigned long long t0 = globaltimer();
  while (true) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (__all_sync(0xFFFFFFFFu, warp_test<CLUSTER>(bar, parity))) return true;
    const bool late = globaltimer() - t0 > kWaitLimitNs;
    if (__any_sync(0xFFFFFFFFu, late || *abort_flag)) {
      if (__any_sync(0xFFFFFFFFu, late)) {
        *abort_flag = 1;
        atomicOr(err, kErrWaitTimeout);
      }
      return false;
    }
  }
}

// Barrier arrivals and TMA loads by an elected lane of a converged warp, for the same reason.
__device__ __forceinline__ void expect_tx_elect(uint64_t *bar, uint32_t bytes) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "@e mbarrier.arrive.expect_tx.release.cta.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(smem_u32(bar)),
      "r"(bytes)
      : "memory");
}
__device__ __forceinline__ void tma_load_2d_elect(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int32_t x, int32_t y) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], "
      "[%2];\n\t}" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d_elect(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int32_t x, int32_t y,
                                                  int32_t z) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "@e cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], "
      "[%2];\n\t}" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}

__device__ __forceinline__ void tma_prefetch_3d_elect(const CUtensorMap *map, int32_t x, int32_t y, int32_t z) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "@e cp.async.bulk.prefetch.tensor.3d.L2.global [%0, {%1, %2, %3}];\n\t}" ::"l"(reinterpret_cast<uint64_t>(map)),
      "r"(x), "r"(y), "r"(z)
      : "memory");
}

// The same of a CTA pair, where `go`, counted on a barrier of either CTA (`bar_cluster`).
__device__ __forceinline__ void tma_load_2d_pair_elect(uint32_t go, uint32_t dst, const CUtensorMap *map,
                                                       uint32_t bar_cluster, int32_t x, int32_t y) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "setp.ne.and.b32 e, %5, 0, e;\n\t"
      "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], "
      "[%2];\n\t}" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar_cluster), "r"(x), "r"(y), "r"(go)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair_elect(uint32_t go, uint32_t dst, const CUtensorMap *map,
                                                       uint32_t bar_cluster, int32_t x, int32_t y, int32_t z) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "setp.ne.and.b32 e, %6, 0, e;\n\t"
      "@e cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4, %5}], "
      "[%2];\n\t}" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar_cluster), "r"(x), "r"(y), "r"(z), "r"(go)
      : "memory");
}
__device__ __forceinline__ void expect_tx_elect(uint32_t go, uint32_t bar, uint32_t bytes) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "setp.ne.and.b32 e, %2, 0, e;\n\t"
      "@e mbarrier.arrive.expect_tx.release.cta.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar),
      "r"(bytes), "r"(go)
      : "memory");
}
// A value that is the same in all lanes, in a uniform register.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __reduce_max_sync(0xFFFFFFFFu, x); }

// The scale bytes of 128 rows, stage by stage, for one warp that loads them itself: lane l takes rows l,
// l + 32, l + 64 and l + 96. A row's bytes start anywhere, so a stage's are cut out of the two aligned
// pieces of kBytes that hold them; all four rows of a lane lie alike to those, being 32 rows apart (32 K
// / 16 is a multiple of 64, 32 K / 32 of 32). Pieces are read kAhead of the warp's stages early.
template <int FMT>
struct ScaleRows {
  static constexpr int kBytes = Fp4<FMT>::kBytes, kWords = Fp4<FMT>::kWords;
  static constexpr int kAhead = 2;
  const uint8_t *at;        // aligned piece of the lane's first row and stage 0
  const uint8_t *end;       // of the plane
  int64_t apart;            // bytes of 32 rows
  int G, shift, rows;       // scale bytes of a row; bytes from `at` to the row's; the lane's rows that exist
  uint32_t v[kAhead][4][2 * kWords];

  __device__ __forceinline__ void open(const uint8_t *plane, int64_t plane_rows, int64_t row0, int rows_left, int G_, int lane) {
    G = G_;
    const uint8_t *first = plane + (row0 + lane) * G;
    shift = static_cast<int>(reinterpret_cast<uintptr_t>(first) % kBytes);
    at = first - shift;
    end = plane + plane_rows * G;
    apart = 32 * static_cast<int64_t>(G);
    rows = rows_left > lane ? (rows_left - lane + 31) / 32 : 0;  // of the lane's
  }
  // Stage `it` into slot d; past the last one (cnt) nothing is read. All loads first, without a branch
  // between them: one by one they took a microsecond each.
  __device__ __forceinline__ void load(int d, int it, int cnt) {
    bool cut = false;  // the plane ends inside a piece
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t *w = &v[d][r][j * kWords];
        const uint8_t *p = at + r * apart + static_cast<int64_t>(it + j) * kBytes;
        const bool in = r < rows && it < cnt && (j == 0 || (it + 1) * kBytes - shift < G);
        const bool whole = in && p + kBytes <= end;
        cut |= in && !whole;
        if constexpr (kWords == 4) {
          uint4 x = make_uint4(0, 0, 0, 0);
          if (whole) x = *reinterpret_cast<const uint4 *>(p);
          w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
        } else {
          uint2 x = make_uint2(0, 0);
          if (whole) x = *reinterpret_cast<const uint2 *>(p);
          w[0] = x.x, w[1] = x.y;
        }
      }
    }
    if (cut) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint8_t *p = at + r * apart + static_cast<int64_t>(it + j) * kBytes;
          if (r < rows && p < end && p + kBytes > end && (j == 0 || (it + 1) * kBytes - shift < G))
#pragma unroll
            for (int b = 0; b < kBytes; ++b)
              if (p + b < end) v[d][r][j * kWords + b / 4] |= static_cast<uint32_t>(p[b]) << (8 * (b % 4));
        }
    }
  }
  // The scale bytes of row r (0 .. 3) in slot d, stage `it`; those behind the row's end are zero.
  __device__ __forceinline__ void take(int d, int r, int it, uint32_t (&w)[kWords]) const {
    uint32_t y[2 * kWords];
#pragma unroll
    for (int i = 0; i < 2 * kWords; ++i) y[i] = v[d][r][i];
    if constexpr (kWords == 4) {
      if (shift & 8) {
#pragma unroll
        for (int i = 0; i < 6; ++i) y[i] = y[i + 2];
      }
    }
    if (shift & 4) {
#pragma unroll
      for (int i = 0; i < kWords + 1; ++i) y[i] = y[i + 1 < 2 * kWords ? i + 1 : i];
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = __funnelshift_r(y[i], y[i + 1], 8 * (shift & 3));
    const int valid = G - it * kBytes;
    if (valid < kBytes) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        const int b = valid - 4 * i;
        w[i] = b <= 0 ? 0u : (b < 4 ? w[i] & ((1u << (8 * b)) - 1) : w[i]);
      }
    }
  }
};

// Changes the signs of the codes under the negative scale bytes of a row's stage: word p covers 64 of
// the stage's depth, 32 bytes of the row's 128 in the swizzled tile, byte j of it 8 of those.
__device__ __noinline__ void flip_codes(uint32_t tile, int row, int p, uint32_t word) {
  for (int j = 0; j < 4; ++j)
    if (word & (0x80u << (8 * j))) {
      const uint32_t a = tile + row * 128 + (((2 * p + (j >> 1)) ^ (row & 7)) << 4) + (j & 1) * 8;
      uint32_t lo, hi;
      asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(lo), "=r"(hi) : "r"(a));
      asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(a), "r"(lo ^ 0x88888888u), "r"(hi ^ 0x88888888u) : "memory");
    }
}

// Where the codes of 128 rows of scales lie: row r of the scales is row r + lift of the `rows` rows of
// codes that a stage has `off` bytes from its start.
struct CodeRows {
  int off, lift, rows;
};

// A stage's scale bytes of 128 rows, lane l's rows l + 32 r, to their atoms. Codes of blocks with a
// negative scale are mended, once they have landed (LANDED: they have; else `landed` says so). Returns
// false if that wait ran out.
template <int FMT, bool LANDED>
__device__ __forceinline__ bool store_scales(uint32_t (&w)[4][Fp4<FMT>::kWords], uint32_t atoms, uint32_t stage,
                                             const CodeRows &c, uint64_t *landed, uint32_t parity,
                                             volatile int *abort_flag, int *err) {
  constexpr int W = Fp4<FMT>::kWords;
  const int lane = threadIdx.x & 31;
  bool ok = true;
  if (FMT == 0) {
    uint32_t sign = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < W; ++i) sign |= w[r][i];
    if (__any_sync(0xFFFFFFFFu, sign & 0x80808080u)) {
      if (!LANDED) ok = __all_sync(0xFFFFFFFFu, mbar_wait(landed, parity, abort_flag, err));
      if (ok) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int i = 0; i < W; ++i) {
            const int row = lane + 32 * r + c.lift;
            if ((w[r][i] & 0x80808080u) && row >= 0 && row < c.rows) flip_codes(stage + c.off, row, i, w[r][i]);
            w[r][i] &= 0x7F7F7F7Fu;
          }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < W; ++i) st_shared_v4(atoms + i * kAtom + lane * 16, w[0][i], w[1][i], w[2][i], w[3][i]);
  return ok;
}

// The bytes that TMA brought, 16 of each of up to 128 rows from `at` on (`rows` of them were asked for),
// to atoms in their place. MXFP4: those of stage `it` are one half.
template <int FMT>
__device__ __forceinline__ void turn_scales(uint32_t at, int rows, int it, uint32_t stage, const CodeRows &c) {
  constexpr int W = Fp4<FMT>::kWords;
  const int lane = threadIdx.x & 31;
  uint32_t w[4][W];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    uint4 x = make_uint4(0, 0, 0, 0);
    if (lane + 32 * r < rows) x = lds128(at + (lane + 32 * r) * kSpan);
    if constexpr (FMT == 0) {
      w[r][0] = x.x, w[r][1] = x.y, w[r][2] = x.z, w[r][3] = x.w;
    } else {
      w[r][0] = it & 1 ? x.z : x.x, w[r][1] = it & 1 ? x.w : x.y;
    }
  }
  __syncwarp();  // all of them are read
  store_scales<FMT, true>(w, at, stage, c, nullptr, 0, nullptr, nullptr);
}

// The stages of one of two warps that share an operand's scales: those whose slot of the ring is even, or
// odd. A wait by parity cannot tell a use of a slot from the one two before, and need not where every
// use of a slot is the same warp's. (Every other stage, in a ring of an odd number of slots, ran into that.)
struct ScaleStages {
  int it, s;    // stage and slot
  uint32_t ph;  // parity of the slot's use
  __device__ __forceinline__ explicit ScaleStages(int set) : it(set), s(set), ph(0) {}
  __device__ __forceinline__ void next(int S) {
    if (s + 2 < S) {
      it += 2;
      s += 2;
    } else {  // on to slot 0 or 1
      it += S - s + (s & 1);
      s &= 1;
      ph ^= 1u;
    }
  }
};

// ---------------------------------------------------------------- tiles of ragged experts
//
// The rows of expert e are offsets[e] .. offsets[e + 1] - 1, read on the device and kept within the R
// rows that there are, whatever they hold.
__device__ __forceinline__ void expert_rows(const Fp4Args &p, int e, int &lo, int &hi) {
  const int64_t a = p.offsets[e], b = p.offsets[e + 1];
  lo = static_cast<int>(max(int64_t(0), min(a, p.R)));
  hi = static_cast<int>(min(p.R, max(b, static_cast<int64_t>(lo))));
}

// Rows of the token tiles that `rows` rows are cut into, `most` at most: equal ones, whole steps of the MMA's N.
__device__ __forceinline__ int tile_count(int rows, int most) { return (rows + most - 1) / most; }
__device__ __forceinline__ int tile_height(int rows, int most, int unit) {
  const int tiles = tile_count(rows, most);
  return tiles > 0 ? ((rows + tiles - 1) / tiles + unit - 1) / unit * unit : unit;
}

// Token tile tt of the experts' tiles, expert by expert: its expert, first row and
// rows (0 past the last tile). Called by a whole CTA, which reads all offsets at once, between barriers of its
// own; each lane of warp 0 counts the tiles of its share of the experts.
struct TileSearch {
  int lo[kRouteMaxExperts], rows[kRouteMaxExperts];
  int found[3];
};
__device__ __forceinline__ void find_tile(const Fp4Args &p, TileSearch &f, int tt, int most, int unit, int &e, int &row0, int &rows) {
  for (int x = threadIdx.x; x < p.E; x += blockDim.x) {
    int lo, hi;
    expert_rows(p, x, lo, hi);
    f.lo[x] = lo;
    f.rows[x] = hi - lo;
  }
  if (threadIdx.x < 3) f.found[threadIdx.x] = 0;
  __syncthreads();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x, per = (p.E + 31) / 32, first = lane * per, last = min(p.E, first + per);
    int mine = 0;
    for (int x = first; x < last; ++x) mine += tile_count(f.rows[x], most);
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, upto, d);
      if (lane >= d) upto = min(upto + v, (1 << 30) - 1);  // offsets that descend may give every expert all rows
    }
    if (tt >= upto - mine && tt < upto) {  // one lane, or none
      int left = tt - (upto - mine);
      for (int x = first; x < last; ++x) {
        const int tiles = tile_count(f.rows[x], most), height = tile_height(f.rows[x], most, unit);
        if (left < tiles) {
          f.found[0] = x;
          f.found[1] = f.lo[x] + left * height;
          f.found[2] = max(0, min(height, f.rows[x] - left * height));
          break;
        }
        left -= tiles;
      }
    }
  }
  __syncthreads();
  e = f.found[0];
  row0 = f.found[1];
  rows = f.found[2];
}

// ---------------------------------------------------------------- few tokens
//
// The weights are the MMA's A operand (128 output features), up to 128 tokens its N, so tensor work
// and traffic follow the token count. A cluster of up to 8 CTAs cuts the contraction of a tile where
// few tiles would leave SMs idle; its CTAs add their parts up through distributed shared memory, in
// the order of the parts.

struct Fp4FewCfg {
  static constexpr int kF = 128;
  static constexpr int kThreads = 192;  // warps 0-1: scales of the weights, 2-3: of the tokens (each every other stage); TMA; MMA
  static constexpr int kTmaWarp = 4, kMmaWarp = 5;
  static constexpr int kMaxStages = 8;
  static constexpr int kTmemCols = 256;  // 128 of the accumulator; scales: two stages of 16 + 16
  static constexpr int kScaleCols = 32;
};

template <int FMT, bool RAW>
__global__ void __launch_bounds__(Fp4FewCfg::kThreads, 2)
    sq_fp4_few_kernel(const __grid_constant__ Fp4Maps maps, const Fp4Args p) {
  using C = Fp4FewCfg;
  constexpr int W = Fp4<FMT>::kWords;
  extern __shared__ uint8_t fp4_smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(fp4_smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ uint64_t bars[3 * C::kMaxStages + 1];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;
  __shared__ float row_scale[kFp4FewTokens];
  volatile int *abort_flag = &abort_word;
  uint64_t *full = bars;                     // [S] codes of both operands landed          (1 arrival + tx)
  uint64_t *sfull = full + C::kMaxStages;    // [S] their scales are in place              (2 warps)
  uint64_t *empty = sfull + C::kMaxStages;   // [S] the MMAs reading the stage are done    (commit)
  uint64_t *done = empty + C::kMaxStages;    // every MMA of the tile is done              (commit)

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int S = p.stages, splits = p.splits;
  const int part = splits > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int unit = static_cast<int>(blockIdx.x) / splits;
  const int tt = unit / p.ftiles, ft = unit - tt * p.ftiles;
  const int f0 = ft * C::kF;

  if (warp == C::kTmaWarp && lane == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&sfull[s], 2);
      mbar_init(&empty[s], 1);
    }
    mbar_init(done, 1);
    abort_word = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == C::kMmaWarp) tmem_alloc(&tmem_slot, C::kTmemCols);
  // The weight's way to the L2 needs nothing that the launch ahead writes: it begins beside that launch.
  // (An older line that it brings is overwritten there like any other.)
  const int cnt_all = (p.K + kDeep - 1) / kDeep, it0 = cnt_all * part / splits;
  if (!p.offsets && warp == C::kTmaWarp)
    for (int it = it0; it < cnt_all * (part + 1) / splits && it < it0 + 4; ++it)
      tma_prefetch_3d_elect(&maps.w, it * (kDeep / 2), f0, 0);
  dependency_wait();
  dependency_start();
  int expert = 0, row0 = tt * p.tile_tokens, rows = static_cast<int>(min(p.R - row0, static_cast<int64_t>(p.tile_tokens)));
  if (p.offsets) {
    find_tile(p, *reinterpret_cast<TileSearch *>(smem), tt, p.tile_tokens, 8, expert, row0, rows);
    fence_proxy_async_smem();  // the search's memory is the ring's
  }
  // read here and not where they are used: one after the other there took 3 us of a tile
  if (threadIdx.x < rows) row_scale[threadIdx.x] = p.row_ws2 ? p.row_ws2[row0 + threadIdx.x] : p.x_ws2;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const int cnt = __any_sync(0xFFFFFFFFu, rows > 0) ? cnt_all * (part + 1) / splits - it0 : 0;
  const int n8 = (rows + 7) & ~7;
  const uint32_t ring = smem_u32(smem);
  const int x_off = C::kF * 128, sf_off = x_off + p.tile_tokens * 128, stage = sf_off + 2 * kScales;
  int box = 0;  // the smallest that holds the tile's rows; of a dense product all tiles have one
  while ((8 << box) < (p.offsets ? rows : p.tile_tokens)) ++box;

  if (warp == C::kTmaWarp) {
    // ------------------------------------------------------ codes
    int it = 0, s = 0;
    uint32_t ph = 0;
    for (; it < cnt; ++it) {
      if (it >= S && !warp_wait(&empty[s], ph ^ 1u, abort_flag, p.err)) break;
      expect_tx_elect(&full[s], (C::kF + (8u << box)) * (128 + (RAW ? kSpan : 0)));
      const int x = (it0 + it) * (kDeep / 2);
      tma_load_3d_elect(ring + s * stage, &maps.w, &full[s], x, f0, expert);
      tma_load_2d_elect(ring + s * stage + x_off, &maps.x[box], &full[s], x, row0);
      if (RAW) {
        const int b = (it0 + it) * Fp4<FMT>::kBytes / kSpan * kSpan;
        tma_load_3d_elect(ring + s * stage + sf_off, &maps.w_scales, &full[s], b, f0, expert);
        tma_load_2d_elect(ring + s * stage + sf_off + kScales, &maps.x_scales[box], &full[s], b, row0);
      }
      if (++s == S) {
        s = 0;
        ph ^= 1u;
      }
    }
    if (*abort_flag)
      for (int i = (it > S ? it - S : 0); i < it; ++i) mbar_drain(&full[i % S], static_cast<uint32_t>(i / S) & 1u);
  } else if (warp == C::kMmaWarp) {
    // ------------------------------------------------------ MMA issuer (one elected lane of the converged warp)
    const uint64_t ad0 = smem_desc_sw128(ring, 16, 1024), bd0 = smem_desc_sw128(ring + x_off, 16, 1024);
    const uint64_t sd0 = atom_desc(ring + sf_off);
    int s = 0;
    uint32_t ph = 0;
    for (int it = 0; it < cnt; ++it) {
      warp_wait(&sfull[s], ph, abort_flag, p.err);
      if (!RAW) warp_wait(&full[s], ph, abort_flag, p.err);
      if (!RAW) fence_proxy_async_smem();
      tc_fence_after();
      const uint32_t so = static_cast<uint32_t>(s * stage) >> 4;
      const uint32_t sa = tmem + 128 + (it & 1) * C::kScaleCols, sb = sa + 4 * W;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        atom_to_tmem_elect(sa + 4 * i, sd0 + so + i * (kAtom >> 4));
        atom_to_tmem_elect(sb + 4 * i, sd0 + so + ((kScales + i * kAtom) >> 4));
      }
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {  // past the end of K: codes and scales are zeros
        const int word = FMT == 0 ? kk : kk / 2;
        const uint32_t idesc = idesc_fp4<FMT>(C::kF, 0, FMT == 0 ? 0 : 2 * (kk & 1)) | (static_cast<uint32_t>(n8 >> 3) << 17);
        umma_fp4_elect<FMT>(tmem, ad0 + so + 2 * kk, bd0 + so + 2 * kk, idesc, sa + 4 * word, sb + 4 * word,
                            (it > 0 || kk > 0) ? 1u : 0u);
      }
      umma_commit_elect(&empty[s]);
      if (++s == S) {
        s = 0;
        ph ^= 1u;
      }
    }
    umma_commit_elect(done);
    mbar_drain(done, 0);
  } else {
    // ------------------------------------------------------ scales, half of the stages of one operand
    const bool tokens = warp >= 2;
    const int at = sf_off + (tokens ? kScales : 0);
    const CodeRows codes = {tokens ? x_off : 0, 0, tokens ? 8 << box : C::kF};
    ScaleStages c(warp & 1);
    bool ok = true;
    auto next = [&] {
      __syncwarp();
      if (lane == 0) mbar_arrive(&sfull[c.s]);
      c.next(S);
    };
    if constexpr (RAW) {
      while (c.it < cnt) {
        if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(&full[c.s], c.ph, abort_flag, p.err)))) break;
        const uint32_t base = ring + c.s * stage;
        turn_scales<FMT>(base + at, codes.rows, it0 + c.it, base, codes);
        fence_proxy_async_smem();
        next();
      }
    } else {
      using Rows = ScaleRows<FMT>;
      Rows sc;
      if (tokens)
        sc.open(p.x_scales, p.R, row0, rows, p.G, lane);
      else
        sc.open(p.w_scales, static_cast<int64_t>(p.E) * p.N, static_cast<int64_t>(expert) * p.N + f0, p.N - f0, p.G, lane);
      const int last = it0 + cnt;
      ScaleStages ahead = c;
#pragma unroll
      for (int d = 0; d < Rows::kAhead; ++d, ahead.next(S)) sc.load(d, it0 + ahead.it, last);
      while (c.it < cnt && ok) {
#pragma unroll
        for (int d = 0; d < Rows::kAhead; ++d) {
          if (c.it >= cnt) break;
          if (c.it >= S && !(ok = __all_sync(0xFFFFFFFFu, mbar_wait(&empty[c.s], c.ph ^ 1u, abort_flag, p.err)))) break;
          const uint32_t base = ring + c.s * stage;
          uint32_t w[4][W];
#pragma unroll
          for (int r = 0; r < 4; ++r) sc.take(d, r, it0 + c.it, w[r]);
          ok = store_scales<FMT, false>(w, base + at, base, codes, &full[c.s], c.ph, abort_flag, p.err);
          if (!ok) break;
          sc.load(d, it0 + ahead.it, last);
          ahead.next(S);
          next();
        }
      }
    }
    // ------------------------------------------------------ accumulator to shared memory, [token][feature] in fp32
    __syncwarp();
    if (cnt > 0) mbar_wait(done, 0, abort_flag, p.err);
    __syncwarp();
    tc_fence_after();
    const uint32_t t_row = tmem + (static_cast<uint32_t>(warp * 32) << 16);
    float *sums = reinterpret_cast<float *>(smem) + warp * 32 + lane;
#pragma unroll 1
    for (int c = 0; c < rows; c += 32) {
      uint32_t v[32];
      if (cnt > 0) {
        tmem_ld32(t_row + c, v);
        tmem_ld_wait();
      }
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (c + i < rows) sums[(c + i) * C::kF] = cnt > 0 ? __uint_as_float(v[i]) : 0.f;
    }
  }
  // ------------------------------------------------------ parts added up, scaled, rounded, stored
  __syncwarp();
  tc_fence_before();
  if (splits > 1)
    cluster_sync_all();
  else
    __syncthreads();
  if (warp == C::kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, C::kTmemCols);
  }
  const float ws2 = p.w_ws2 ? p.w_ws2[expert] : p.ws2;
  const int j = threadIdx.x & 15, f = f0 + 8 * j;
  if (f < p.N) {
    for (int t = part * (C::kThreads / 16) + (threadIdx.x >> 4); t < rows; t += splits * (C::kThreads / 16)) {
      float y[8] = {};
      const uint32_t mine = ring + (t * C::kF + 8 * j) * 4;
      for (int q0 = 0; q0 < splits; q0 += 4) {  // the loads of four parts, then their sums in order
        float4 v[8];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v[2 * q] = v[2 * q + 1] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (q0 + q < splits) {
            const uint32_t at = splits > 1 ? mapa_shared(mine, q0 + q) : mine;
#pragma unroll
            for (int i = 0; i < 2; ++i)
              asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                           : "=f"(v[2 * q + i].x), "=f"(v[2 * q + i].y), "=f"(v[2 * q + i].z), "=f"(v[2 * q + i].w)
                           : "r"(at + 16 * i));
          }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            y[4 * i] += v[2 * q + i].x, y[4 * i + 1] += v[2 * q + i].y;
            y[4 * i + 2] += v[2 * q + i].z, y[4 * i + 3] += v[2 * q + i].w;
          }
      }
      const float row = row_scale[t];
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(y[2 * i] * ws2 * row, y[2 * i + 1] * ws2 * row);
        o[i] = *reinterpret_cast<const uint32_t *>(&h);
      }
      *reinterpret_cast<uint4 *>(p.out + (static_cast<int64_t>(row0) + t) * p.N + f) = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
  if (splits > 1) cluster_sync_all();  // the others have read this CTA's sums
}

// ---------------------------------------------------------------- many tokens
//
// A cluster of two CTAs per tile of 256 features and up to 256 tokens, 224 of an expert (tcgen05.mma.cta_group::2): each CTA
// holds the codes of 128 of the features and half of the tokens, the atoms of its features and those of
// all the tokens. The tokens are the MMA's N, of any multiple of 16: an expert's rows, cut into equal
// tiles, cost what they are (32444 rows of 128 experts of 2880 x 2880: 157 us, and 171 with the tokens as the 256 rows of
// a tile). Persistent, with two accumulators, so a tile's epilogue runs under the next one's MMAs.
//
// A launch ahead (sq_fp4_atoms_kernel) writes the atoms: of each token tile two blocks of 128 rows (the second
// of fewer), of each feature tile two, for every stage, and whether it met a negative scale.
// Only then the pair kernel has a warp that mends the codes of each stage before the MMAs may read it: every stage of
// the launch, for one negative byte anywhere. That warp is slower than the MMAs (16384 x 14336 x 4096 309 us, 1765 with
// one such byte, 4684 with half of them).

struct Fp4PairCfg {
  static constexpr int kEpiWarps = 8;  // 32 features w % 4, every other 32 tokens from w / 4 on
  static constexpr int kTmaWarp = kEpiWarps, kMmaWarp = kTmaWarp + 1, kMendWarp = kMmaWarp + 1;
  static constexpr int kThreads = 32 * (kMendWarp + 1);
  static constexpr int kA = 128 * 128;
  static constexpr int kMaxStages = 8;
  static constexpr int kBox = 16 * 64;  // 16 tokens x 32 features of an epilogue warp
};
// Tensor memory: two accumulators and, behind them, 48 columns of a slice's scales. Those of wide tiles overlap, the
// second begins at column 208: the epilogue reads the columns that both use before the others, and the MMAs of the
// next tile wait for that much of it, some 2,500 cycles a tile (estimated from products of 16 and 32 slices;
// fp4_pair_tokens charges 1.23 times the tile's own time).
constexpr int kPairOver = 208, kPairScales = 464;
static_assert(2 * kFp4PairApart <= kPairScales && kPairOver + kFp4PairTokens <= kPairScales && kPairScales + 48 <= 512 &&
                  kFp4PairTokens - kPairOver <= 64 && kPairOver % 16 == 0,
              "two accumulators and a slice's scales in tensor memory; two groups of 32 columns hold the shared ones");

__device__ __forceinline__ void atom_to_tmem_pair_elect(uint32_t taddr, uint64_t desc) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "@e tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(taddr),
      "l"(desc)
      : "memory");
}
template <int FMT>
__device__ __forceinline__ void umma_fp4_pair_elect(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa,
                                                    uint32_t sb, uint32_t accumulate) {
  if (FMT == 0)
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "elect.sync _|e, 0xFFFFFFFF;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "elect.sync _|e, 0xFFFFFFFF;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void commit_pair_mc_elect(uint64_t *bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(
          smem_u32(bar)),
      "h"(static_cast<unsigned short>(3))
      : "memory");
}
__device__ __forceinline__ void commit_pair_elect(uint64_t *bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}

// A grouped launch's experts in shared memory: first token tile [E + 1], first row, rows and rows of a token
// tile [E].
struct Fp4Experts {
  int *tiles, *lo, *rows, *height;
};

// Tile of a launch: expert, first row and rows, first feature. Every role, a whole warp, walks the tiles in
// increasing order, so the expert only moves forward, 32 at a look. (One by one, with the divisions of a
// common raster, a step over 25 experts took longer than the tile's 8 stages.) An expert's tiles go
// feature tile by feature tile, the weight's rows from the L2 for the second token tile on.
struct Fp4Tile {
  int e = 0, row0, rows, f0;
  int token_tile, feature_tile;  // of all experts
  __device__ __forceinline__ bool at(const Fp4Args &p, const Fp4Experts &x, int tile) {
    int tm, tn;
    if (p.offsets) {
      if (tile >= x.tiles[p.E] * p.ftiles) return false;
      const int lane = threadIdx.x & 31;
      for (int n = 32; n == 32;) {
        const int next = e + 1 + lane;
        n = __popc(__ballot_sync(0xFFFFFFFFu, next < p.E && x.tiles[next] * p.ftiles <= tile));
        e += n;
      }
      const int before = x.tiles[e], count = x.tiles[e + 1] - before, local = tile - before * p.ftiles;
      tn = count == 1 ? local : local / count;
      tm = local - tn * count;
      token_tile = before + tm;
      row0 = x.lo[e] + tm * x.height[e];
      rows = min(x.height[e], x.lo[e] + x.rows[e] - row0);
    } else {  // the tiles of the last rows, where they are fewer, behind all others
      if (tile >= p.units) return false;
      if (tile < p.whole * p.ftiles) {
        tile_coords(tile, p.whole, p.ftiles, tm, tn);
      } else {
        tm = p.whole;
        tn = tile - p.whole * p.ftiles;
      }
      token_tile = tm;
      row0 = tm * p.tile_tokens;
      rows = min(p.tile_tokens, static_cast<int>(p.R) - row0);
    }
    f0 = tn * kFp4PairFeatures;
    feature_tile = e * p.ftiles + tn;
    return true;
  }
};

// Atoms of 128 rows and 8 (NVFP4) or 16 slices (called stages here) per CTA; slices behind the end of K are zeros. The rows' bytes come in whole 16-byte pieces to shared memory
// (lines apart by an odd number of pieces, free of bank conflicts) and are cut out from there.
template <int FMT>
struct AtomCfg {
  static constexpr int kThreads = 256, kStages = fp4_atom_stages(FMT);
  static constexpr int kSpanBytes = kStages * Fp4<FMT>::kBytes;     // of a row: 128
  static constexpr int kPieces = kSpanBytes / 16 + 1;               // that hold them
  static_assert(kPieces % 2 == 1, "rows an odd number of 16-byte pieces apart");
};

template <int FMT>
__global__ void __launch_bounds__(AtomCfg<FMT>::kThreads) sq_fp4_atoms_kernel(const Fp4Args p) {
  using C = AtomCfg<FMT>;
  constexpr int W = Fp4<FMT>::kWords;
  __shared__ uint4 piece[128 * C::kPieces];
  static_assert(sizeof(TileSearch) <= sizeof(piece), "the search's memory");
  const int cnt = p.depth * p.slices, groups = (cnt + C::kStages - 1) / C::kStages;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int block = static_cast<int>(blockIdx.x) / groups;
  const int kb0 = (static_cast<int>(blockIdx.x) - block * groups) * C::kStages;
  dependency_wait();
  dependency_start();
  const bool tokens = block < p.token_blocks;
  const uint8_t *plane = p.w_scales;
  int64_t row0, plane_rows = static_cast<int64_t>(p.E) * p.N;
  int rows;
  uint4 *out;
  if (tokens) {
    if (p.offsets) {
      int e, r0;
      find_tile(p, *reinterpret_cast<TileSearch *>(piece), block >> 1, kFp4PairApart, 16, e, r0, rows);
      row0 = r0;
      __syncthreads();  // the search's memory is the pieces'
    } else {
      row0 = static_cast<int64_t>(block >> 1) * p.tile_tokens;
      rows = static_cast<int>(min(static_cast<int64_t>(p.tile_tokens), p.R - row0));
    }
    plane = p.x_scales;
    plane_rows = p.R;
    row0 += 128 * (block & 1);
    rows -= 128 * (block & 1);
    out = p.x_atoms + (static_cast<int64_t>(block >> 1) * cnt * 2 + (block & 1)) * (W * kAtom / 16);
  } else {
    block -= p.token_blocks;
    const int tile = block >> 1, e = tile / p.ftiles, f0 = (tile - e * p.ftiles) * kFp4PairFeatures + 128 * (block & 1);
    row0 = static_cast<int64_t>(e) * p.N + f0;
    rows = p.N - f0;
    out = p.w_atoms + static_cast<int64_t>(block) * cnt * (W * kAtom / 16);
  }
  rows = min(rows, 128);
  const uint8_t *first = plane + row0 * p.G, *end = plane + plane_rows * p.G;
  // Row r's bytes from stage kb0 on begin off(r) behind the 16-byte boundary `base`.
  const uint8_t *base = first + kb0 * Fp4<FMT>::kBytes;
  const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(base) % 16);
  base -= lead;
  auto off = [&](int r) { return static_cast<int64_t>(r) * p.G + lead; };
  constexpr int kLoads = (128 * C::kPieces + C::kThreads - 1) / C::kThreads;
  uint4 x[kLoads];
#pragma unroll
  for (int l = 0; l < kLoads; ++l) {
    const int i = threadIdx.x + l * C::kThreads, r = i / C::kPieces, j = i - r * C::kPieces;
    const uint8_t *from = base + (off(r) & ~int64_t(15)) + 16 * j;
    x[l] = make_uint4(0, 0, 0, 0);
    if (r < rows && from + 16 <= end) x[l] = *reinterpret_cast<const uint4 *>(from);
  }
  if (rows > 0 && base + off(rows - 1) + C::kPieces * 16 > end) {  // the plane's last rows: it may end inside a piece
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      const int i = threadIdx.x + l * C::kThreads, r = i / C::kPieces, j = i - r * C::kPieces;
      const uint8_t *from = base + (off(r) & ~int64_t(15)) + 16 * j;
      if (r < rows && from < end && from + 16 > end) {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int b = 0; b < 16; ++b)
          if (from + b < end) w[b / 4] |= static_cast<uint32_t>(from[b]) << (8 * (b % 4));
        x[l] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
#pragma unroll
  for (int l = 0; l < kLoads; ++l) {
    const int i = threadIdx.x + l * C::kThreads;
    if (i < rows * C::kPieces) piece[i] = x[l];
  }
  __syncthreads();
  uint32_t sign = 0;
  const bool level = p.G % 16 == 0;  // every row begins on a boundary
  for (int stage = warp; stage < C::kStages && kb0 + stage < cnt; stage += C::kThreads / 32) {
    const int kb = kb0 + stage;
    uint32_t w[4][W];
    if (level) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = lane + 32 * r;
        uint4 a = make_uint4(0, 0, 0, 0);
        if (row < rows) a = piece[row * C::kPieces + stage * Fp4<FMT>::kBytes / 16];
        if constexpr (FMT == 0) {
          w[r][0] = a.x, w[r][1] = a.y, w[r][2] = a.z, w[r][3] = a.w;
        } else {
          w[r][0] = stage & 1 ? a.z : a.x, w[r][1] = stage & 1 ? a.w : a.y;
        }
      }
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = lane + 32 * r;
        uint32_t y[8] = {};
        const int from = static_cast<int>(off(row) & 15) + stage * Fp4<FMT>::kBytes, shift = from % 16;  // in the row's pieces
        if (row < rows) {
          const uint4 *q = piece + row * C::kPieces + from / 16;
          const uint4 a = q[0];
          y[0] = a.x, y[1] = a.y, y[2] = a.z, y[3] = a.w;
          if (shift + Fp4<FMT>::kBytes > 16) {
            const uint4 b = q[1];
            y[4] = b.x, y[5] = b.y, y[6] = b.z, y[7] = b.w;
          }
        }
        if (shift & 8) {
#pragma unroll
          for (int i = 0; i < 6; ++i) y[i] = y[i + 2];
        }
        if (shift & 4) {
#pragma unroll
          for (int i = 0; i < 5; ++i) y[i] = y[i + 1];
        }
#pragma unroll
        for (int i = 0; i < W; ++i) w[r][i] = __funnelshift_r(y[i], y[i + 1], 8 * (shift & 3));
      }
    }
    const int valid = p.G - kb * Fp4<FMT>::kBytes;  // scale bytes of a row from the stage's first on
    if (valid < Fp4<FMT>::kBytes) {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const int b = valid - 4 * i;
        const uint32_t keep = b >= 4 ? 0xFFFFFFFFu : b <= 0 ? 0u : (1u << (8 * b)) - 1;
#pragma unroll
        for (int r = 0; r < 4; ++r) w[r][i] &= keep;
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < W; ++i) sign |= w[r][i];
    uint4 *dst = out + static_cast<int64_t>(kb) * (W * kAtom / 16) * (tokens ? 2 : 1) + lane;
#pragma unroll
    for (int i = 0; i < W; ++i) dst[i * (kAtom / 16)] = make_uint4(w[0][i], w[1][i], w[2][i], w[3][i]);
  }
  if (FMT == 0) {
    const int any = __syncthreads_or(sign & 0x80808080u);
    if (threadIdx.x == 0) p.negative[blockIdx.x] = any != 0;
  }
}

// H: slices of a stage. WIDE: a dense product in tiles of 240 or 256 tokens.
template <int FMT, int H, bool WIDE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Fp4PairCfg::kThreads, 1)
    sq_fp4_pair_kernel(const __grid_constant__ Fp4PairMaps maps, const Fp4Args p) {
  using C = Fp4PairCfg;
  constexpr int W = Fp4<FMT>::kWords;
  constexpr int kBlock = W * kAtom;  // the atoms of 128 rows and a stage
  constexpr int kB = (WIDE ? kFp4PairTokens : kFp4PairApart) / 2 * 128;  // codes of half the tokens
  constexpr int kBs = H * C::kA, kSf = kBs + H * kB, kXs = kSf + H * kBlock, kStage = fp4_pair_stage(FMT, H, WIDE), kSecond = WIDE ? kPairOver : kFp4PairApart;
  static_assert(kXs + 2 * H * kBlock <= kStage && kStage % 1024 == 0, "a stage");
  constexpr int kScaleCols = 12 * W, kScaleBufs = 48 / kScaleCols;
  extern __shared__ uint8_t fp4_smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(fp4_smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ uint64_t bars[3 * C::kMaxStages + 5];
  __shared__ uint32_t tmem_slot, sink;
  __shared__ int abort_word;
  volatile int *abort_flag = &abort_word;
  const int S = p.stages;
  uint64_t *full = bars;                    // [S] leader: both CTAs' stages are there              (1 arrival + tx)
  uint64_t *landed = full + C::kMaxStages;  // [S] with codes to mend: this CTA's copies have landed  (1 arrival + tx)
  uint64_t *empty = landed + C::kMaxStages;  // [S] the pair's MMAs have read the stage             (multicast commit)
  uint64_t *tfull = empty + C::kMaxStages;  // [2] accumulator complete                             (multicast commit)
  uint64_t *tempty = tfull + 2;             // [2] leader: both epilogues have read it              (8 warps of each; wide: and, of the tile behind, its shared columns)
  uint64_t *drain = tempty + 2;
  __shared__ __align__(16) float row_scale[C::kEpiWarps][32];
  __shared__ volatile uint32_t tile_n[C::kMaxStages];  // tokens of the tile that a stage belongs to, in whole 16
  Fp4Experts ex;
  ex.tiles = reinterpret_cast<int *>(smem + S * kStage + C::kEpiWarps * C::kBox);
  ex.lo = ex.tiles + p.E + 1;
  ex.rows = ex.lo + p.E;
  ex.height = ex.rows + p.E;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&landed[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], (WIDE ? 4 : 2) * C::kEpiWarps);
    }
    if (WIDE)  // no tile before the second one waits for its accumulator
      for (int i = 0; i < 2 * C::kEpiWarps; ++i) mbar_arrive(&tempty[1]);
    mbar_init(drain, 1);
    abort_word = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == C::kMmaWarp) tmem_alloc_pair(&tmem_slot, 512);
  dependency_wait();
  dependency_start();
  bool mend = false;  // some scale is negative
  if (FMT == 0)
    for (int i = threadIdx.x; i < p.atom_ctas; i += C::kThreads) mend |= p.negative[i] != 0;
  if (p.offsets) {
    for (int e = threadIdx.x; e < p.E; e += C::kThreads) {
      int lo, hi;
      expert_rows(p, e, lo, hi);
      ex.lo[e] = lo;
      ex.rows[e] = hi - lo;
      ex.height[e] = tile_height(hi - lo, kFp4PairApart, 16);
      ex.tiles[e + 1] = tile_count(hi - lo, kFp4PairApart);
    }
    __syncthreads();
    if (warp == 0) {
      // never more tiles than the launch has room for, which only offsets that descend ask for
      const int most = p.token_blocks >> 1;
      int before = 0;
      for (int e0 = 0; e0 < p.E; e0 += 32) {
        int v = e0 + lane < p.E ? ex.tiles[e0 + lane + 1] : 0;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
          const int u = __shfl_up_sync(0xFFFFFFFFu, v, d);
          if (lane >= d) v += u;
        }
        if (e0 + lane < p.E) ex.tiles[e0 + lane + 1] = min(before + v, most);
        before = min(before + __shfl_sync(0xFFFFFFFFu, v, 31), most);
      }
      if (lane == 0) ex.tiles[0] = 0;
    }
  }
  tc_fence_before();
  mend = __syncthreads_or(mend);
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = tmem_slot, ring = smem_u32(smem);
  const int cnt = p.depth;
  const int first = static_cast<int>(blockIdx.x >> 1), step = static_cast<int>(gridDim.x >> 1);
  const int tiles = p.offsets ? ex.tiles[p.E] * p.ftiles : static_cast<int>(p.units);
  const int pair_tiles = first < tiles ? (tiles - first + step - 1) / step : 0;  // of this pair
  Fp4Tile t;

  if (warp == C::kTmaWarp) {
    // ------------------------------------------------------ codes and atoms
    // Counted on the leader's barrier or, where codes have to be mended, on this CTA's own. Loops without
    // exits and uniform values here too (the loads of a stage took 590 cycles to issue, more than its MMAs):
    // after a wait that ran out nothing is loaded.
    const bool own = mend, counts = mend || rank == 0;
    const int mine = uniform(pair_tiles);
    int it = 0, s = 0;
    uint32_t ph = 1, go = 1;
    struct Job {
      int row, f, e, xa, wa, half, box;  // xa, wa: the atoms' rows of 512 bytes
      uint32_t bytes;
    };
    auto job = [&](int tc) {
      Job j;
      t.at(p, ex, first + tc * step);
      j.half = uniform(((t.rows + 15) & ~15) / 2);  // tokens of a CTA, in the smallest box that holds them
      int box = 0;
      while (box + 1 < kFp4PairBoxes && fp4_pair_box(box) < j.half) ++box;
      j.box = uniform(box);
      j.bytes = H * (C::kA + 3 * kBlock + fp4_pair_box(j.box) * 128);
      j.row = uniform(t.row0) + j.half * static_cast<int>(rank);
      j.f = uniform(t.f0) + 128 * static_cast<int>(rank);
      j.e = uniform(t.e);
      j.xa = uniform(t.token_tile) * cnt * H * 2 * W;
      j.wa = (2 * uniform(t.feature_tile) + static_cast<int>(rank)) * cnt * H * W;
      return j;
    };
    Job j = {};
    if (mine > 0) j = job(0);
    for (int tc = 0; tc < mine; ++tc) {
      Job next = j;
      for (int kb = 0; kb < cnt; ++kb, ++it) {
        if (kb == cnt - 1 && tc + 1 < mine) next = job(tc + 1);  // before the wait for a slot, in its shadow
        if (it >= S) go = warp_wait(&empty[s], ph, abort_flag, p.err) ? go : 0;
        const uint32_t at = ring + s * kStage;
        if (kb == 0) {
          tile_n[s] = 2 * j.half;
          __syncwarp();
        }
        const uint32_t count = smem_u32(own ? &landed[s] : &full[s]);
        expect_tx_elect(counts ? go : 0, count, own ? j.bytes : 2 * j.bytes);
        const uint32_t bar = mapa_shared(count, own ? rank : 0);
#pragma unroll
        for (int h = 0; h < H; ++h) {
          tma_load_3d_pair_elect(go, at + h * C::kA, &maps.w, bar, (kb * H + h) * (kDeep / 2), j.f, j.e);
          tma_load_2d_pair_elect(go, at + kBs + h * kB, &maps.x[j.box], bar, (kb * H + h) * (kDeep / 2), j.row);
        }
        tma_load_2d_pair_elect(go, at + kSf, &maps.w_atoms, bar, 0, j.wa + kb * H * W);
        tma_load_2d_pair_elect(go, at + kXs, &maps.x_atoms, bar, 0, j.xa + kb * H * 2 * W);
        if (++s == S) {
          s = 0;
          ph ^= 1u;
        }
      }
      j = next;
    }
    if (*abort_flag && (mend || rank == 0)) {
      uint64_t *bar = mend ? landed : full;
      for (int i = (it > S ? it - S : 0); i < it; ++i) mbar_drain(&bar[i % S], static_cast<uint32_t>(i / S) & 1u);
    }
  } else if (warp == C::kMmaWarp) {
    // ------------------------------------------------------ MMA issuer (leader; one elected lane)
    if (rank == 0) {
      const uint64_t ad0 = smem_desc_sw128(ring, 16, 1024), bd0 = smem_desc_sw128(ring + kBs, 16, 1024);
      const uint64_t sd0 = atom_desc(ring + kSf);
      // Behind the MMA that they run the tensor cores hold about two more: between the last MMA of a stage and
      // the first of the next there are 250 cycles for the barriers, the commit and the atoms.
      // The loop is there twice: a stage whose codes the peer has mended is waited for at cluster scope.
      const int mine = __reduce_max_sync(0xFFFFFFFFu, pair_tiles);
      auto issue = [&](auto mended) {
        constexpr bool kMended = decltype(mended)::value;
        int s = 0, it = 0;
        uint32_t ph = 0;
        bool there = false;  // the stage was found complete while the one before was issued
        for (int tc = 0; tc < mine; ++tc) {
          const int ab = tc & 1;
          if (tc >= (WIDE ? 1 : 2)) warp_wait<true>(&tempty[ab], (static_cast<uint32_t>(tc >> 1) & 1u) ^ (WIDE && ab ? 0u : 1u), abort_flag, p.err);
          // the tile's N comes with its first stage: looked up here it would bring its branches into the loop
          if (!there) warp_wait<kMended>(&full[s], ph, abort_flag, p.err);
          there = true;
          const uint32_t n16 = __reduce_max_sync(0xFFFFFFFFu, tile_n[s]);
          const uint32_t d = tmem + ab * kSecond;
          const uint32_t desc0 = idesc_fp4<FMT>(2 * 128, 0, 0) | n16 << 14, desc1 = idesc_fp4<FMT>(2 * 128, 0, FMT == 0 ? 0 : 2) | n16 << 14;
          for (int kb = 0; kb < cnt; ++kb, ++it) {
            if (!there) warp_wait<kMended>(&full[s], ph, abort_flag, p.err);
            tc_fence_after();
            const uint32_t so = static_cast<uint32_t>(s * kStage) >> 4;
            bool found = false;
#pragma unroll
            for (int h = 0; h < H; ++h) {
              const uint32_t sa = tmem + kPairScales + ((it * H + h) & (kScaleBufs - 1)) * kScaleCols, sb = sa + 4 * W;
#pragma unroll
              for (int i = 0; i < W; ++i) {
                atom_to_tmem_pair_elect(sa + 4 * i, sd0 + so + ((h * kBlock + i * kAtom) >> 4));
                atom_to_tmem_pair_elect(sb + 8 * i, sd0 + so + (((H + 2 * h) * kBlock + i * kAtom) >> 4));
                atom_to_tmem_pair_elect(sb + 8 * i + 4, sd0 + so + (((H + 2 * h + 1) * kBlock + i * kAtom) >> 4));
              }
              if (h == H - 1) found = warp_test<kMended>(&full[s + 1 == S ? 0 : s + 1], s + 1 == S ? ph ^ 1u : ph);
#pragma unroll
              for (int kk = 0; kk < 4; ++kk) {  // past the end of K: codes and scales are zeros
                const int word = FMT == 0 ? kk : kk / 2;
                umma_fp4_pair_elect<FMT>(d, ad0 + so + (h * C::kA >> 4) + 2 * kk, bd0 + so + (h * kB >> 4) + 2 * kk,
                                         kk & 1 ? desc1 : desc0, sa + 4 * word, sb + 8 * word, (kb > 0 || h > 0 || kk > 0) ? 1u : 0u);
              }
            }
            commit_pair_mc_elect(&empty[s]);
            if (++s == S) {
              s = 0;
              ph ^= 1u;
            }
            there = __all_sync(0xFFFFFFFFu, found);
          }
          commit_pair_mc_elect(&tfull[ab]);
        }
      };
      if (FMT == 0 && __any_sync(0xFFFFFFFFu, mend))
        issue(std::true_type());
      else
        issue(std::false_type());
      commit_pair_elect(drain);
      mbar_drain(drain, 0);
    }
  } else if (warp == C::kMendWarp) {
    // ------------------------------------------------------ codes of blocks with a negative scale
    if (FMT == 0 && mend) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int tile = first; ok && t.at(p, ex, tile); tile += step)
        for (int kb = 0; kb < cnt; ++kb) {
          if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(&landed[s], ph, abort_flag, p.err)))) break;
          const uint32_t at = ring + s * kStage;
          const int half = ((t.rows + 15) & ~15) / 2;
          for (int i = 0; i < 3 * W * H; ++i) {  // an atom of the features, then of the first 128 and the other tokens of a slice
            const bool of_w = i < W * H;
            const int j = of_w ? i : i - W * H, word = j % W, h = of_w ? j / W : j / (2 * W);
            const int lift = of_w ? 0 : 128 * (j / W % 2) - half * static_cast<int>(rank), rows = of_w ? 128 : half;
            const uint32_t line = at + kSf + i * kAtom + lane * 16, codes = at + (of_w ? h * C::kA : kBs + h * kB);
            const uint4 x = lds128(line);
            uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int row = lane + 32 * r + lift;
              if ((w[r] & 0x80808080u) && row >= 0 && row < rows) flip_codes(codes, row, word, w[r]);
            }
            st_shared_v4(line, w[0] & 0x7F7F7F7Fu, w[1] & 0x7F7F7F7Fu, w[2] & 0x7F7F7F7Fu, w[3] & 0x7F7F7F7Fu);
          }
          fence_proxy_async_smem();
          __syncwarp();
          // the peer reports by a store that waits for nothing (an arrival at cluster scope waits for all writes
          // before it, 1,000 cycles)
          if (lane == 0) {
            if (rank == 0)
              mbar_arrive_expect_tx(&full[s], 4);
            else
              st_async_signal(mapa_shared(smem_u32(&sink), 0), mapa_shared(smem_u32(&full[s]), 0));
          }
          if (++s == S) {
            s = 0;
            ph ^= 1u;
          }
        }
    }
  } else {
    // ------------------------------------------------------ epilogue
    // A lane has a feature's 32 tokens. Two neighbours exchange halves, so each has two features of 16
    // tokens, and put them into a box whose line t holds tokens t and t + 16, 64 bytes each: written and
    // read without bank conflicts.
    const int quad = warp & 3, share = warp >> 2;
    const uint32_t t_row = tmem + (static_cast<uint32_t>(quad * 32) << 16);
    const uint32_t box = ring + S * kStage + warp * C::kBox;
    float *scales = row_scale[warp];
    int tc = 0;
    bool ok = true;
    for (int tile = first; ok && t.at(p, ex, tile); tile += step, ++tc) {
      const int ab = tc & 1;
      const int groups = (t.rows + 31) / 32;  // of 32 tokens
      const float ws2 = p.w_ws2 ? p.w_ws2[t.e] : p.ws2;
      ok = WIDE ? warp_wait(&tfull[ab], static_cast<uint32_t>(tc >> 1) & 1u, abort_flag, p.err)
                : __all_sync(0xFFFFFFFFu, mbar_wait(&tfull[ab], static_cast<uint32_t>(tc >> 1) & 1u, abort_flag, p.err));
      if (!ok) break;
      tc_fence_after();
      auto release = [&] {  // the warp's part of the accumulator is read
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_cluster(mapa_shared(smem_u32(&tempty[ab]), 0));
      };
      auto release_over = [&] {
        if (!WIDE) return;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_cluster(mapa_shared(smem_u32(&tempty[ab ^ 1]), 0));
      };
      if (share >= groups) {
        release_over();
        release();
      }
#pragma unroll 1
      for (int n = share; n < groups; n += 2) {  // the first accumulator's shared columns are its last
        const int g = WIDE && ab == 0 ? groups - 1 - n : n;
        const int left = t.rows - 32 * g;  // tokens of the group
        uint32_t v[32];
        tmem_ld32(t_row + ab * kSecond + 32 * g, v);
        if (WIDE && n == share) {  // the next tile's MMAs wait for this
          tmem_ld_wait();
          release_over();
        }
        const float mine = lane < left ? (p.row_ws2 ? p.row_ws2[static_cast<int64_t>(t.row0) + 32 * g + lane] : p.x_ws2) : 0.f;
        __syncwarp();  // the box and the scales are read
        scales[lane] = mine;
        tmem_ld_wait();
        if (n + 2 >= groups) release();
        __syncwarp();
        uint32_t o[16];  // tokens 2 i and 2 i + 1
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          const float4 r = *reinterpret_cast<const float4 *>(scales + i);
          const __nv_bfloat162 a = __floats2bfloat162_rn(__uint_as_float(v[i]) * ws2 * r.x, __uint_as_float(v[i + 1]) * ws2 * r.y);
          const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float(v[i + 2]) * ws2 * r.z, __uint_as_float(v[i + 3]) * ws2 * r.w);
          o[i / 2] = *reinterpret_cast<const uint32_t *>(&a);
          o[i / 2 + 1] = *reinterpret_cast<const uint32_t *>(&b);
        }
        const bool odd = lane & 1;
        const int f = t.f0 + 128 * static_cast<int>(rank) + 32 * quad + 8 * (lane & 3);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          if (part > 0) __syncwarp();  // the box is read
#pragma unroll
          for (int i = 4 * part; i < 4 * part + 4; ++i) {  // even lanes keep tokens 0-15, odd ones 16-31, of both features
            const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, odd ? o[i] : o[i + 8], 1);
            const uint32_t even_f = odd ? other : o[i], odd_f = odd ? o[i + 8] : other;
            const uint32_t at = box + (2 * i - 8 * part) * 128 + (odd ? 64 : 0) + (lane >> 1) * 4;
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(prmt(even_f, odd_f, 0x5410u)) : "memory");
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + 128), "r"(prmt(even_f, odd_f, 0x7632u)) : "memory");
          }
          __syncwarp();
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int line = 4 * q + (lane >> 3), r = 8 * part + line + (lane & 4 ? 16 : 0);  // eight lanes a line
            const uint4 y = lds128(box + line * 128 + (lane & 7) * 16);
            if (r < left && f < p.N)
              *reinterpret_cast<uint4 *>(p.out + (static_cast<int64_t>(t.row0) + 32 * g + r) * p.N + f) = y;
          }
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  cluster_sync_all();
  if (warp == C::kMmaWarp) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
}

template <typename Maps>
cudaError_t launch_kernel(void (*kernel)(Maps, Fp4Args), int &done_mask, int most_smem, unsigned grid, int threads, size_t smem, int cluster,
                       cudaStream_t stream, const Maps &maps, const Fp4Args &p) {
  int dev = 0;
  cudaGetDevice(&dev);
  if (!(done_mask & (1 << (dev & 31)))) {
    cudaError_t e;
    if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem)) != cudaSuccess ||
        (e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout,
                                  cudaSharedmemCarveoutMaxShared)) != cudaSuccess)
      return e;
    done_mask |= 1 << (dev & 31);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, maps, p);
}

template <int FMT, bool RAW>
cudaError_t launch_few_fp4(const Fp4Maps &maps, const Fp4Args &p, cudaStream_t stream) {
  static int done_mask = 0;
  const size_t smem = static_cast<size_t>(p.stages) * fp4_few_stage(p.tile_tokens) + 1024;
  return launch_kernel(sq_fp4_few_kernel<FMT, RAW>, done_mask, kFp4SmemAlone,
                    static_cast<unsigned>(p.units * p.splits), Fp4FewCfg::kThreads, smem, p.splits, stream, maps, p);
}

}  // namespace

cudaError_t fp4_clusters(Fp4Clusters &fit) {
  const auto kernel = sq_fp4_few_kernel<0, true>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFp4SmemAlone);
  if (e != cudaSuccess) return e;
  for (int c = 8; c >= 1; --c) {
    for (int two = 0; two < 2; ++two) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(8 * c, 1, 1);
      cfg.blockDim = dim3(Fp4FewCfg::kThreads, 1, 1);
      cfg.dynamicSmemBytes = two ? kFp4SmemShared : kFp4SmemAlone;
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = c;
      attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
      cfg.attrs = attr;
      cfg.numAttrs = 1;
      if ((e = cudaOccupancyMaxActiveClusters(two ? &fit.shared[c] : &fit.alone[c], kernel, &cfg)) != cudaSuccess) return e;
    }
  }
  fit.alone[0] = 1;
  return cudaSuccess;
}

cudaError_t launch_fp4_few(int fmt, const Fp4Maps &maps, const Fp4Args &p, cudaStream_t stream) {
  const bool raw = p.G % kSpan == 0;
  if (fmt == 0) return raw ? launch_few_fp4<0, true>(maps, p, stream) : launch_few_fp4<0, false>(maps, p, stream);
  return raw ? launch_few_fp4<1, true>(maps, p, stream) : launch_few_fp4<1, false>(maps, p, stream);
}

template <int FMT, int H, bool WIDE>
static cudaError_t launch_pair(const Fp4PairMaps &maps, const Fp4Args &p, int sm_count, cudaStream_t stream) {
  static int done_mask = 0;
  const cudaError_t e = launch_after(sq_fp4_atoms_kernel<FMT>, static_cast<unsigned>(p.atom_ctas), AtomCfg<FMT>::kThreads, 0, stream, p);
  if (e != cudaSuccess) return e;
  const int clusters = static_cast<int>(std::min<int64_t>(p.units, sm_count / 2));
  return launch_kernel<const Fp4PairMaps>(sq_fp4_pair_kernel<FMT, H, WIDE>, done_mask, kFp4SmemMost, 2u * clusters, Fp4PairCfg::kThreads,
                                          fp4_pair_smem(FMT, H, WIDE, p.stages, p.offsets ? p.E : 0), 1, stream, maps, p);
}

cudaError_t launch_fp4_pair(int fmt, const Fp4PairMaps &maps, const Fp4Args &p, int sm_count, cudaStream_t stream) {
  const bool wide = p.tile_tokens > kFp4PairApart;
  if (fmt == 0 && wide) return launch_pair<0, 1, true>(maps, p, sm_count, stream);
  if (fmt == 0) return p.slices == 1 ? launch_pair<0, 1, false>(maps, p, sm_count, stream) : launch_pair<0, 2, false>(maps, p, sm_count, stream);
  if (wide) return p.slices == 1 ? launch_pair<1, 1, true>(maps, p, sm_count, stream) : launch_pair<1, 2, true>(maps, p, sm_count, stream);
  return p.slices == 1 ? launch_pair<1, 1, false>(maps, p, sm_count, stream) : launch_pair<1, 2, false>(maps, p, sm_count, stream);
}

}  // namespace sqi
