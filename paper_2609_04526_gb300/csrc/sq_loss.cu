// Softmax cross entropy of hidden rows against a frozen vocabulary projection, with the gradient
// of the rows (sm_103a):
//
//   z = X W^T,  loss = log sum_v exp z_v - z_label,  dX = g (softmax(z) - onehot(label)) W
//
// The logits exist only as accumulator tiles in tensor memory. Per piece of labelled tokens:
//
//   gather    the labelled tokens' rows, packed, and each row's label logit z_l (CUDA cores)
//   logits    z tile by tile; the epilogue forms e = 2^(z log2(e) - r), adds e over 64 columns
//             and, for the gradient, writes bf16 e of the piece
//   finalize  sums -> loss, log-sum-exp and the row's two gradient factors
//   gradient  (e W) over the vocabulary, cut into parts where few tiles would leave SMs idle
//   rows      dX = g (1 - p) (e W / Z - W[label]), p the label's share and Z the sum of e as it is in e W
//
// The reference r of a row is ceil(z_l log2(e)), known before the product: e then needs no
// maximum first, and e W no second pass over the logits once S is known. Where a tile holds a
// logit more than 2^100 above it (a label of probability below 2^-100), that quarter of
// it takes its own maximum as reference, and finalize rescales the row's e. References are whole
// powers of two, so such a change of reference is exact. Terms more than 2^126 below the label's
// own vanish.
//
// The label's own term is left out of e and of the sums and carried in fp32: 1 - p is (S - e_l) / S
// without cancellation, so confident tokens keep an accurate loss and gradient.
//
// e is rounded to bf16 once, as an operand of the tensor cores: at most 2^-9 of a term. The sum S, of
// the loss and of 1 - p, takes the unrounded values. e W is divided by the sum Z of the rounded ones: its
// weights so add up to 1, as the label's coefficient does, what the rows of W have in common cancels,
// and a term of share s among the others moves the result by 1 - s of its rounding. (Relative error
// of dX for 256 rows against 8000 x 512 where the rows of W share a part of ten times their own size and
// one competitor of the label has 0.6 of the others: 0.00167, of which the rounding of dX itself is
// 0.00166; with S in place of Z 0.0094.)
#include "sq_gemm_kernels.cuh"
#include "sq_launch.cuh"

namespace sqi {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr uint32_t kMinusInfinity = 0xFF800000u;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRefSlack = 100.f;  // a logit this far above the reference (in powers of two) moves it
constexpr float kFarSum = 0x1p100f;  // the sum of a quarter tile that may hold one

// What a product launch does.
enum HeadStep {
  HEAD_LOSS,       // logits, of a call without a gradient
  HEAD_KEEP,       // logits, whose exponentials are written for the gradient
  HEAD_GRAD,       // gradient, each sum in one accumulator
  HEAD_GRAD_LONG,  // gradient, sums longer than kHeadSegment products
};

// A pair's tile has 256 rows and NT columns, its stages are BK deep. Epilogue warp w takes TMEM lanes
// 32 (w % 4) .. + 31 and the w / 4-th 64 columns (which stay in registers) or, where a sum leaves tensor
// memory once, 128.
template <int STEP, int BK, int NT>
struct HeadCfg {
  static constexpr bool GRAD = STEP >= HEAD_GRAD;
  static constexpr int kEpiCols = STEP == HEAD_GRAD ? 128 : 64;
  static constexpr int kEpiWarps = NT / kEpiCols * 4;
  static constexpr int kTmaWarp = kEpiWarps;
  static constexpr int kMmaWarp = kTmaWarp + 1;
  static constexpr int kThreads = 32 * (kMmaWarp + 1);
  static constexpr int kBK = BK;
  static constexpr int kCols = NT / 2;             // columns of a CTA
  static constexpr int kB = kCols * kBK * 2;       // bytes of them in a stage
  static constexpr int kRing = 192 * 1024;         // 6 stages of 128 rows and 128 columns, 64 deep
  static constexpr int kMaxStages = 12;
  static constexpr int kUnit = GRAD ? 128 / kBK : 1;  // stages of a unit of the walk's contraction
  static constexpr int kRows = kHeadTile;
  static constexpr int kOffBox = kRing;
  static constexpr int kBoxCols = STEP == HEAD_GRAD_LONG ? 16 : 32;
  static constexpr int kBoxBytes = 32 * kBoxCols * (GRAD ? 4 : 2);  // 32 rows x kBoxCols columns of a warp
  // Stages added up in one accumulator. The tensor core truncates its running fp32 sum at every
  // step of 16, a bias that grows with the length: a sum of 4096 products in one accumulator left
  // the log-sum-exp, of 11 to 14, 1.6e-5 too small (1.6e-6 now). The logits therefore leave tensor memory every 512 products
  // and are added in registers, and so does the gradient, rounded to bf16 in the end, every
  // kHeadSegment.
  static constexpr int kSegment = STEP == HEAD_GRAD ? 1 << 30 : (GRAD ? kHeadSegment : 512) / kBK;
  static constexpr int kOffBar = kOffBox + kEpiWarps * kBoxBytes;
  static constexpr int kSmemBytes = kOffBar + 512 + 1024;
};
// The last stage's A, read to 128 rows of its second 64-wide chunk, ends within the shared memory (the
// smallest tiles: 12 stages of 16 KiB).
static_assert(11 * 16384 + 4096 + 16384 <= HeadCfg<HEAD_LOSS, 128, 64>::kOffBar, "operand rows past the shared memory");
static_assert(HeadCfg<HEAD_KEEP, 64, 256>::kSmemBytes <= 232448 && HeadCfg<HEAD_GRAD, 64, 256>::kSmemBytes <= 232448 &&
                  HeadCfg<HEAD_GRAD_LONG, 64, 256>::kSmemBytes <= 232448,
              "head kernel exceeds the opt-in shared memory of one CTA");

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 2^d of a whole d <= 0, exactly; 0 where it is not a normal number.
__device__ __forceinline__ float whole_exp2(float d) {
  return d < -126.f ? 0.f : __int_as_float((127 + static_cast<int>(d)) << 23);
}

// The pair's MMA and its commits from one elected lane of a converged warp (the same lane at every
// election): the descriptors stay in uniform registers. A single lane's are moved there for every
// MMA, which beside four epilogue warps on its scheduler takes longer than the MMA itself.
__device__ __forceinline__ void umma_pair_elect(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                                uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_commit_pair_mc_elect(uint64_t *bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(
          smem_u32(bar)),
      "h"(static_cast<unsigned short>(3))
      : "memory");
}
__device__ __forceinline__ void umma_commit_pair_elect(uint64_t *bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xFFFFFFFF;\n\t"
      "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar))
      : "memory");
}

// mbar_wait without a call, for a thread that holds many registers.
__device__ __forceinline__ bool mbar_wait_inline(uint64_t *bar, uint32_t parity, volatile int *abort_flag, int *err) {
  if (mbar_try_wait(bar, parity)) return true;
  const unsigned long long t0 = globaltimer();
  while (true) {
#pragma unroll 1
    for (int i = 0; i < 32; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
    if (globaltimer() - t0 > kWaitLimitNs) {
      *abort_flag = 1;
      atomicOr(err, kErrWaitTimeout);
      return false;
    }
  }
}

// 32 lanes x 16 consecutive fp32 columns.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
}

__device__ __forceinline__ float warp_total(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// Reference exponent of a row from its label logit in powers of two; never -inf, and a NaN logit
// leaves a number here (the row's NaN reaches its results through the label's own term).
__device__ __forceinline__ float row_reference(float label_z) { return fmaxf(ceilf(label_z * kLog2e), -1e30f); }

// Rows of the piece's chunk that starts at compact row `first`. The launches behind the logits read
// what gather wrote before their wait, from the L2: the launch ahead of them, having passed its own
// wait, shows that it is complete (64 rows of width 512 against 8000, loss and gradient: 22.2 us, 21.2
// so; 8 of 2312 against 3211: 26.6, 25.2).
__device__ __forceinline__ int chunk_rows(const HeadArgs &a, int first) {
  const int left = __ldcg(a.count) - first;
  return left < 0 ? 0 : (left < a.chunk ? left : a.chunk);
}

// ---------------------------------------------------------------- gather

// SHARE warps per token and 8 / SHARE tokens per CTA. The labelled tokens are packed in order
// (each CTA counts the labels before its own), so rows without a label cost nothing later and
// what they hold reaches no product. Few tokens take a whole CTA each: one warp walked a row of
// 4096 in 7.3 us.
template <int SHARE>
__global__ void __launch_bounds__(256) sq_head_gather_kernel(const HeadArgs a) {
  static_assert(SHARE == 1 || SHARE == 8, "a token's 256 lanes, or 32 that take their eight sums");
  constexpr int kTokens = 8 / SHARE;
  __shared__ int before[8];
  __shared__ float dots[8];
  dependency_wait();
  dependency_start();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t0 = blockIdx.x * kTokens, own = warp / SHARE, t = t0 + own;
  auto labelled = [&](int i) {
    const int64_t y = a.labels[i];
    return y >= 0 && y < a.V;
  };
  for (int i = blockIdx.x * 256 + threadIdx.x; i < a.chunk; i += gridDim.x * 256) a.moved[i] = 0;
  int seen = 0;
  for (int i = threadIdx.x; i < t0; i += 256) seen += labelled(i);
  const uint32_t here =  // the same in every warp
      __ballot_sync(0xFFFFFFFFu, lane < kTokens && t0 + lane < a.T && labelled(t0 + lane));
  seen = __reduce_add_sync(0xFFFFFFFFu, seen);
  if (lane == 0) before[warp] = seen;
  __syncthreads();
  int row = __popc(here & ((1u << own) - 1));
#pragma unroll
  for (int w = 0; w < 8; ++w) row += before[w];
  const bool target = (here >> own) & 1;
  const int first = (warp % SHARE) * 32 + lane;  // of this token's threads
  if (t == a.T - 1 && first == 0) *a.count = row + target;
  const int pieces = static_cast<int>(a.D / 8);
  float dot = 0.f;
  int64_t y = 0;
  if (t < a.T && !target) {
    if (a.dX) {
      uint4 *out = reinterpret_cast<uint4 *>(a.dX + static_cast<int64_t>(t) * a.D);
      for (int i = first; i < pieces; i += 32 * SHARE) out[i] = make_uint4(0, 0, 0, 0);
    }
    if (first == 0) {
      if (a.loss) a.loss[t] = 0.f;
      if (a.lse) a.lse[t] = 0.f;
    }
  } else if (t < a.T) {
    y = a.labels[t];
    const uint4 *x = reinterpret_cast<const uint4 *>(a.X + static_cast<int64_t>(t) * a.D);
    const uint4 *w = reinterpret_cast<const uint4 *>(a.W + y * a.D);
    uint4 *out = reinterpret_cast<uint4 *>(a.rows + static_cast<int64_t>(row) * a.width);
    // eight sums of every 256th 16 bytes, a warp's or, of one warp, each lane's own: one order for both
    float sums[kTokens] = {};
    constexpr int kFlight = kTokens < 4 ? kTokens : 4;  // 16-byte loads of each row in flight
    for (int i0 = first; i0 < pieces; i0 += 256) {
#pragma unroll
      for (int c0 = 0; c0 < kTokens; c0 += kFlight) {
        uint4 p[kFlight], q[kFlight];
#pragma unroll
        for (int c = 0; c < kFlight; ++c) {
          const int i = i0 + 32 * (c0 + c);
          p[c] = q[c] = make_uint4(0, 0, 0, 0);
          if (i < pieces) {
            p[c] = x[i];
            q[c] = w[i];
          }
        }
#pragma unroll
        for (int c = 0; c < kFlight; ++c) {
          const int i = i0 + 32 * (c0 + c);
          if (i < pieces) out[i] = p[c];
          const uint32_t pw[4] = {p[c].x, p[c].y, p[c].z, p[c].w}, qw[4] = {q[c].x, q[c].y, q[c].z, q[c].w};
          float &sum = sums[c0 + c];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sum = fmaf(__uint_as_float(pw[e] << 16), __uint_as_float(qw[e] << 16), sum);
            sum = fmaf(__uint_as_float(pw[e] & 0xFFFF0000u), __uint_as_float(qw[e] & 0xFFFF0000u), sum);
          }
        }
      }
    }
#pragma unroll
    for (int c = 0; c < kTokens; ++c) dot += warp_total(sums[c]);
  }
  if (SHARE > 1) {
    if (lane == 0) dots[warp] = dot;
    __syncthreads();
    dot = 0.f;
#pragma unroll
    for (int w = 0; w < SHARE; ++w) dot += dots[own * SHARE + w];
  }
  if (t < a.T && target && first == 0) {
    a.token[row] = t;
    a.label[row] = static_cast<int>(y);
    a.label_z[row] = dot;
  }
}

// ---------------------------------------------------------------- contractions
//
// Both contractions run as CTA pairs (tcgen05.mma.cta_group::2, tiles of 256 rows and NT columns, two
// fp32 accumulators in tensor memory, so a tile's epilogue runs under the next tile's MMAs).
//   logits:   D[t, v] = sum_d X[t, d] W[v, d]   both operands K-major
//   gradient: D[t, d] = sum_v e[t, v] W[v, d]   e K-major, W MN-major; a unit is a tile over a
//             part of the vocabulary and writes its own fp32 plane, added in order later. The
//             vocabulary goes backwards, the parts side by side: its end is in the L2 from the
//             logits (12 tokens against 21887 x 2720: 64 us, 62 so; 53 against 27534 x 3152: 82, 80)

// The tiles of one cluster in order: every step-th of a list that goes part by part, in panels of
// up to 8 row tiles, a panel column by column (so the CTAs resident at any moment share a few row
// and column tiles in the L2). Stepped without divisions: they took a thread 1,000 cycles a tile,
// in which the ring of loads ran dry and sixteen epilogue warps spent 600 issue slots each.
template <bool GRAD>
struct HeadWalk {
  int tm, tn, part;  // row tile, column tile, part of the vocabulary
  int k0, nk;        // its first stage and stages (gradient: every parts-th, backwards)
  int step, tiles_m, tiles_n, parts, stages;
  int panel, height, at;  // first row tile of the panel, its row tiles, place in it
  uint32_t by_height, by_parts;  // 2^32 / height and parts, rounded up: exact quotients below 2^26
  __device__ __forceinline__ HeadWalk(int first, int step_, int tiles_m_, int tiles_n_, int parts_, int stages_)
      : step(step_), tiles_m(tiles_m_), tiles_n(tiles_n_), parts(parts_), stages(stages_) {
    part = tiles_m > 0 ? 0 : parts;
    at = first;
    by_parts = inverse(parts);
    open(0);
    place();
  }
  __device__ __forceinline__ bool more() const { return part < parts; }
  __device__ __forceinline__ void advance() {
    at += step;
    place();
  }

 private:
  static __device__ __forceinline__ uint32_t inverse(int n) { return n > 1 ? 0xFFFFFFFFu / n + 1 : 0; }
  static __device__ __forceinline__ int quotient(int x, int n, uint32_t by) {
    return n > 1 ? static_cast<int>(__umulhi(static_cast<uint32_t>(x), by)) : x;
  }
  __device__ __forceinline__ void open(int first) {
    panel = first;
    height = min(8, tiles_m - first);
    by_height = inverse(height);
  }
  __device__ __forceinline__ void place() {
    while (part < parts && at >= height * tiles_n) {
      at -= height * tiles_n;
      if (panel + height < tiles_m) {
        open(panel + height);
      } else {
        ++part;
        if (panel > 0) open(0);
      }
    }
    tn = quotient(at, height, by_height);
    tm = panel + at - tn * height;
    k0 = GRAD ? stages - 1 - part : 0;
    nk = GRAD ? quotient(stages - part + parts - 1, parts, by_parts) : stages;
  }
};

template <int STEP, int BK, int NT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(HeadCfg<STEP, BK, NT>::kThreads, 1)
    sq_head_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                   const __grid_constant__ CUtensorMap tmO, const HeadArgs a, const int first) {
  using C = HeadCfg<STEP, BK, NT>;
  constexpr bool GRAD = C::GRAD, KEEP = STEP == HEAD_KEEP;
  // A stage holds box_rows rows of A; the MMAs read 128 all the same, the rest of them whatever
  // lies behind in the ring and the store boxes, and nothing reads those rows of the product. Few
  // tokens so leave the ring to the columns, which are all their traffic (one token against 128256
  // x 4096: 181 us with 96 KiB of columns in flight, 170 with 128). Without a gradient the store
  // boxes' room is part of the ring.
  constexpr int kMax = C::kMaxStages;
  const int a_bytes = a.box_rows * C::kBK * 2, stage_bytes = a_bytes + C::kB;
  const int S = min(kMax, (GRAD || KEEP ? C::kRing : C::kOffBar) / stage_bytes);
  const bool both = a.T > 128;  // else the peer's rows of A are past the last token
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t *full = reinterpret_cast<uint64_t *>(smem + C::kOffBar);  // [S] leader: both CTAs' tiles landed
  uint64_t *empty = full + kMax;    // [S] the pair's MMAs have read the stage        (multicast commit)
  uint64_t *tfull = empty + kMax;   // [2] accumulator complete                       (multicast commit)
  uint64_t *tempty = tfull + 2;  // [2] leader: both epilogues drained it (kEpiWarps arrivals + the peer's st.async)
  uint64_t *drain = tempty + 2;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(drain + 1);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
  uint32_t *sink = reinterpret_cast<uint32_t *>(drain + 2);  // [kEpiWarps] leader: st.async targets

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  auto stage_a = [&](int s) { return smem + s * stage_bytes; };
  auto stage_b = [&](int s) { return smem + s * stage_bytes + a_bytes; };

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&tfull[b], 1);
      mbar_init(&tempty[b], C::kEpiWarps);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == C::kMmaWarp) tmem_alloc_pair(tmem_slot, 2 * kTmemCols);
  if (warp == C::kTmaWarp && lane == 0) {
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
    tma_prefetch_desc(&tmO);
  }
  tc_fence_before();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  int rows = GRAD ? chunk_rows(a, first) : 0;
  dependency_wait();
  dependency_start();
  if (!GRAD) rows = chunk_rows(a, first);
  const int tiles_m = (rows + C::kRows - 1) / C::kRows;
  const int tiles_n = static_cast<int>(((GRAD ? a.D : a.V) + NT - 1) / NT);
  constexpr int kDepth = C::kBK * C::kUnit;
  const int stages = static_cast<int>(((GRAD ? a.V : a.D) + kDepth - 1) / kDepth);
  const int parts = GRAD && tiles_m > 0 ? a.parts[tiles_m - 1] + 1 : 1;
  HeadWalk<GRAD> t(blockIdx.x >> 1, gridDim.x >> 1, tiles_m, tiles_n, parts, stages);

  if (warp == C::kTmaWarp) {
    // ------------------------------------------------------ TMA producer (both CTAs)
    if (lane == 0) {
      int it = 0;
      bool ok = true;
      int s = 0;
      uint32_t ph = 1;  // parity of the phase that frees slot s: its first use finds it free
      for (; t.more() && ok; t.advance()) {
        const int32_t row0 = (GRAD ? 0 : first) + t.tm * C::kRows + 128 * static_cast<int32_t>(rank);
        const int32_t col0 = t.tn * NT + C::kCols * static_cast<int32_t>(rank);
        int kb = t.k0 * C::kUnit;
        for (int i = 0; i < t.nk * C::kUnit; ++i, ++it) {
          if (it >= S && !(ok = mbar_wait(&empty[s], ph, abort_flag, a.err))) break;
          if (rank == 0) mbar_arrive_expect_tx(&full[s], 2 * C::kB + (both ? 2 : 1) * a_bytes);
          const uint32_t bar = mapa_shared(smem_u32(&full[s]), 0);
          if (rank == 0 || both)
            for (int j = 0; j < C::kBK / 64; ++j)
              tma_load_2d_pair(smem_u32(stage_a(s)) + j * (a.box_rows * 128), &tmA, bar, kb * C::kBK + 64 * j, row0);
          if (GRAD) {  // 64 columns of D x kBK vocabulary rows
            for (int j = 0; j < 2; ++j)
              tma_load_2d_pair(smem_u32(stage_b(s)) + j * (C::kB / 2), &tmB, bar, col0 + 64 * j, kb * C::kBK);
          } else {  // kCols vocabulary rows x 64 columns of D
            for (int j = 0; j < C::kBK / 64; ++j)
              tma_load_2d_pair(smem_u32(stage_b(s)) + j * (C::kCols * 128), &tmB, bar, kb * C::kBK + 64 * j, col0);
          }
          ++kb;
          if (GRAD && kb % C::kUnit == 0) kb -= (parts + 1) * C::kUnit;
          if (++s == S) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
      if (*abort_flag && rank == 0) {
        for (int i = (it > S ? it - S : 0); i < it; ++i) mbar_drain(&full[i % S], static_cast<uint32_t>(i / S) & 1u);
      }
    }
  } else if (warp == C::kMmaWarp) {
    // ------------------------------------------------------ MMA issuer (leader CTA)
    // The whole warp walks the stages, so a wait that runs out for some lanes ends all of them.
    if (rank == 0) {
      constexpr uint32_t idesc = idesc_bf16(2 * 128, NT, 0, GRAD ? 1 : 0);
      // K-major: K step kk in 64-wide chunk kk / 4 (a box apart), byte 32 (kk % 4) of each row;
      // MN-major: 16 contraction rows (2 KiB) per step, 64-column atoms half the operand apart
      const uint64_t ad_base = smem_desc_sw128(smem_u32(stage_a(0)), 16, 1024);
      const uint64_t bd_base = smem_desc_sw128(smem_u32(stage_b(0)), GRAD ? C::kB / 2 : 16, 1024);
      int s = 0, tc = 0;  // tc: accumulators filled
      uint32_t ph = 0;
      bool ok = true;
      for (; t.more() && ok; t.advance()) {
        const int steps_all = t.nk * C::kUnit;
        for (int k0 = 0; k0 < steps_all && ok; k0 += C::kSegment, ++tc) {
          const int ab = tc & 1;
          const uint32_t au = static_cast<uint32_t>(tc >> 1);
          if (tc >= 2 &&
              !(ok = __all_sync(0xFFFFFFFFu, mbar_spin_cluster(&tempty[ab], (au & 1u) ^ 1u, abort_flag, a.err))))
            break;
          tc_fence_after();
          const uint32_t d_tmem = tmem_base + ab * kTmemCols;
          const int steps = min(C::kSegment, steps_all - k0);
          for (int kb = 0; kb < steps; ++kb) {
            if (!(ok = __all_sync(0xFFFFFFFFu, mbar_spin(&full[s], ph, abort_flag, a.err)))) break;
            const uint64_t so = static_cast<uint64_t>(s * (stage_bytes >> 4));
            const uint64_t a0 = ad_base + so, b0 = bd_base + so;
#pragma unroll
            for (int kk = 0; kk < C::kBK / 16; ++kk) {
              const uint32_t ka = (kk >> 2) * (a.box_rows * 8) + (kk & 3) * 2;
              const uint32_t kb_ = GRAD ? (kk * 2048) >> 4 : ((kk >> 2) * (C::kCols * 128) + (kk & 3) * 32) >> 4;
              umma_pair_elect(d_tmem, a0 + ka, b0 + kb_, idesc, (kb > 0 || kk > 0) ? 1u : 0u);
            }
            umma_commit_pair_mc_elect(&empty[s]);
            if (++s == S) {
              s = 0;
              ph ^= 1u;
            }
          }
          if (ok) umma_commit_pair_mc_elect(&tfull[ab]);
        }
      }
      umma_commit_pair_elect(drain);
      mbar_drain(drain, 0);
    }
  } else {
    // ------------------------------------------------------ epilogue (both CTAs)
    // (a wait that runs out for some lanes ends the warp's tiles as a whole)
    const int quad = warp & 3, share = warp >> 2;
    const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + share * C::kEpiCols;
    const uint32_t box = smem_u32(smem + C::kOffBox + warp * C::kBoxBytes);
    // accumulator drained: the leader's warps arrive (warp 0 arming the peer's bytes), the peer's
    // signal with a non-blocking async store
    auto release = [&](int ab) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (rank == 0) {
          if (warp == 0)
            mbar_arrive_expect_tx(&tempty[ab], 4 * C::kEpiWarps);
          else
            mbar_arrive(&tempty[ab]);
        } else {
          st_async_signal(mapa_shared(smem_u32(&sink[warp]), 0), mapa_shared(smem_u32(&tempty[ab]), 0));
        }
      }
    };
    int tc = 0;
    bool ok = true;
    int label = -1;  // of this lane's row in the next tile, and its logit
    float label_z = 0.f;
    auto labels = [&] {
      const int r = t.tm * C::kRows + 128 * static_cast<int>(rank) + 32 * quad + lane;
      label = -1;
      label_z = 0.f;
      if (!GRAD && r < rows) {
        label = a.label[first + r];
        label_z = a.label_z[first + r];
      }
    };
    if (t.more()) labels();
    while (t.more() && ok) {
      const int row32 = t.tm * C::kRows + 128 * static_cast<int>(rank) + 32 * quad;  // of the chunk
      const int col0 = t.tn * NT + C::kEpiCols * share;
      if constexpr (STEP == HEAD_GRAD) {
        const int ab = tc & 1;
        ok = __all_sync(0xFFFFFFFFu, mbar_wait(&tfull[ab], static_cast<uint32_t>(tc >> 1) & 1u, abort_flag, a.err));
        if (!ok) break;
        tc_fence_after();
        const uint32_t t_buf = t_row + ab * kTmemCols;
        const int32_t out_row = t.part * tiles_m * C::kRows + row32;
#pragma unroll 1
        for (int g = 0; g < C::kEpiCols / 32; ++g) {
          uint32_t v[32];
          tmem_ld32(t_buf + 32 * g, v);
          tmem_ld_wait();
          if (lane == 0) bulk_wait_read<0>();  // the previous box's store has read the buffer
          __syncwarp();
#pragma unroll
          for (int q = 0; q < 8; ++q)
            st_shared_v4(box + lane * 128 + ((q ^ (lane & 7)) << 4), v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
          fence_proxy_async_smem();  // the box -> async proxy (the TMA store)
          __syncwarp();
          if (lane == 0) {
            if (col0 + 32 * g < a.D && row32 < rows) tma_store_2d(&tmO, box, col0 + 32 * g, out_row);
            bulk_commit_group();
          }
        }
        release(ab);
        ++tc;
        t.advance();
      } else if constexpr (GRAD) {
        const int32_t out_row = t.part * tiles_m * C::kRows + row32;
        const int steps = t.nk * C::kUnit;
        float v[C::kEpiCols] = {};  // the row's sums
#pragma unroll 1
        for (int k0 = 0; k0 < steps; k0 += C::kSegment, ++tc) {
          const int ab = tc & 1;
          ok = __all_sync(0xFFFFFFFFu, mbar_wait_inline(&tfull[ab], static_cast<uint32_t>(tc >> 1) & 1u, abort_flag, a.err));
          if (!ok) break;
          tc_fence_after();
          // Added to zeros the first time too: with loads in place, as of the logits, or a call in the wait
          // 50 registers were saved in memory at every turn (2048 against 38912 x 2048, loss and gradient:
          // 394 us, 381 so).
#pragma unroll
          for (int g = 0; g < C::kEpiCols / 16; ++g) {
            uint32_t x[16];
            tmem_ld16(t_row + ab * kTmemCols + 16 * g, x);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) v[16 * g + i] += __uint_as_float(x[i]);
          }
          release(ab);
        }
        if (!ok) break;
#pragma unroll
        for (int g = 0; g < C::kEpiCols / 16; ++g) {
          if (lane == 0) bulk_wait_read<0>();  // the previous box's store has read the buffer
          __syncwarp();
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float *x = v + 16 * g + 4 * q;
            st_shared_v4(box + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4), __float_as_uint(x[0]), __float_as_uint(x[1]),
                         __float_as_uint(x[2]), __float_as_uint(x[3]));
          }
          fence_proxy_async_smem();  // the box -> async proxy (the TMA store)
          __syncwarp();
          if (lane == 0) {
            if (col0 + 16 * g < a.D && row32 < rows) tma_store_2d(&tmO, box, col0 + 16 * g, out_row);
            bulk_commit_group();
          }
        }
        t.advance();
      } else {
        const bool in = row32 + lane < rows;
        const int at = label - col0;  // the label's own column is left out
        float ref = row_reference(label_z);
        uint32_t z[2][32];  // the row's logits
        static_assert(C::kEpiCols == 64, "two 32-column loads");
        for (int k0 = 0; k0 < stages; k0 += C::kSegment, ++tc) {
          const int ab = tc & 1;
          ok = __all_sync(0xFFFFFFFFu, mbar_wait(&tfull[ab], static_cast<uint32_t>(tc >> 1) & 1u, abort_flag, a.err));
          if (!ok) break;
          tc_fence_after();
          if (k0 == 0) {
            tmem_ld32(t_row + ab * kTmemCols, z[0]);
            tmem_ld32(t_row + ab * kTmemCols + 32, z[1]);
            tmem_ld_wait_for(z[0]);
            tmem_ld_wait_for(z[1]);
          } else {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              uint32_t v[16];
              tmem_ld16(t_row + ab * kTmemCols + 16 * g, v);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                uint32_t &q = z[g / 2][16 * (g % 2) + i];
                q = __float_as_uint(__uint_as_float(q) + __uint_as_float(v[i]));
              }
            }
          }
          release(ab);
        }
        if (!ok) break;
        // the next tile's labels are on their way while this one's exponentials are formed
        const int64_t at_sum = static_cast<int64_t>(col0 / C::kEpiCols) * a.sum_rows + row32 + lane;
        t.advance();
        if (t.more()) labels();
        if (col0 >= a.V) continue;
        if (__any_sync(0xFFFFFFFFu, at >= 0 && at < C::kEpiCols)) {
#pragma unroll
          for (int i = 0; i < C::kEpiCols; ++i)
            if (i == at) z[i / 32][i % 32] = kMinusInfinity;
        }
        if (col0 + C::kEpiCols > a.V) {
#pragma unroll
          for (int i = 0; i < C::kEpiCols; ++i)
            if (col0 + i >= a.V) z[i / 32][i % 32] = kMinusInfinity;
        }
        // A logit far above the reference shows in the sum; the largest one then becomes the
        // reference and the exponentials are formed again.
        float sum = 0.f, sum_e = 0.f;
#pragma unroll 1
        for (bool again = false;; again = true) {
          float part[4] = {};
          sum_e = 0.f;
#pragma unroll
          for (int g = 0; g < C::kEpiCols / 32; ++g) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              uint32_t packed[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float e0 = exp2_fast(fmaf(__uint_as_float(z[g][8 * q + 2 * i]), kLog2e, -ref));
                const float e1 = exp2_fast(fmaf(__uint_as_float(z[g][8 * q + 2 * i + 1]), kLog2e, -ref));
                part[i] += e0 + e1;
                const __nv_bfloat162 h2 = __floats2bfloat162_rn(e0, e1);
                packed[i] = *reinterpret_cast<const uint32_t *>(&h2);
              }
              // The test at run time, always true, keeps the compiler from forming all exponentials
              // ahead of the first store and spilling them (2048 against 38912 x 512, logits and
              // gradient: 171 us without it and in groups of 32, 148 so).
              if (KEEP && a.e) {
                if (q == 0) {
                  if (lane == 0) bulk_wait_read<0>();  // the box's last store, half a tile ago, has read it
                  __syncwarp();
                }
                st_shared_v4(box + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4), packed[0], packed[1], packed[2], packed[3]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  sum_e += __uint_as_float(packed[i] << 16) + __uint_as_float(packed[i] & 0xFFFF0000u);
              }
            }
            if (KEEP && a.e) {
              fence_proxy_async_smem();  // the box -> async proxy (the TMA store)
              __syncwarp();
              if (lane == 0) {
                if (col0 + 32 * g < a.V && row32 < rows) tma_store_2d(&tmO, box, col0 + 32 * g, row32);
                bulk_commit_group();
              }
            }
          }
          sum = (part[0] + part[1]) + (part[2] + part[3]);
          if (again || !__any_sync(0xFFFFFFFFu, in && !(sum < kFarSum))) break;
          float most = -INFINITY;
#pragma unroll
          for (int i = 0; i < C::kEpiCols; ++i) most = fmaxf(most, __uint_as_float(z[i / 32][i % 32]));
          if (fmaf(most, kLog2e, -ref) > kRefSlack) {
            ref = ceilf(most * kLog2e);
            if (in) a.moved[row32 + lane] = 1;
          }
          if (lane == 0) bulk_wait_all();  // the first box is written before the second one
          __syncwarp();
        }
        if (in) {
          if constexpr (KEEP)
            reinterpret_cast<float2 *>(a.sums)[at_sum] = make_float2(sum, sum_e);
          else
            a.sums[at_sum] = sum;
          a.refs[at_sum] = ref;
        }
      }
    }
    if (lane == 0) bulk_wait_all();
  }

  __syncwarp();
  tc_fence_before();
  cluster_sync_all();
  if (warp == C::kMmaWarp) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 2 * kTmemCols);
  }
}

// ---------------------------------------------------------------- finalize and rows

__device__ __forceinline__ float from_lane(float v, int mask) { return __shfl_xor_sync(0xFFFFFFFFu, v, mask); }
__device__ __forceinline__ float2 from_lane(float2 v, int mask) {
  return make_float2(from_lane(v.x, mask), from_lane(v.y, mask));
}

// ROWS rows per CTA: each takes 32 / ROWS lanes of every warp, which take the quarter tiles in turn
// (neighbouring rows of one quarter tile lie side by side): 8 read whole sectors, 4 give few tokens
// twice the CTAs (32, whole lines, left most SMs without rows: 14 us for 2048). The order of a row's
// sum is the same in all, so it depends on nothing but the row: 256 sums of every 256th quarter
// tile, eight to a warp, then the warps'.
template <int ROWS, bool KEEP>
__global__ void __launch_bounds__(1024, ROWS == 4 ? 1 : 2) sq_head_finalize_kernel(const HeadArgs a, const int first) {
  constexpr int kShare = 32 / ROWS;
  __shared__ float parts[32][ROWS + 1], parts_e[32][ROWS + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rows = chunk_rows(a, first), r0 = blockIdx.x * ROWS;
  const int own = lane % ROWS;  // of the CTA's rows
  const int r = min(r0 + own, rows - 1), row = first + r;  // lanes past the last row repeat it
  const bool on = r0 < rows;
  const float z = on ? __ldcg(a.label_z + row) : 0.f;
  const int t = on ? __ldcg(a.token + row) : 0;
  const float g = on && KEEP ? __ldcg(a.dloss + t) : 0.f;
  dependency_wait();
  dependency_start();
  if (!on) return;
  constexpr int kCols = HeadCfg<HEAD_LOSS, 64, 256>::kEpiCols;
  const int filled = static_cast<int>((a.V + kCols - 1) / kCols);  // quarter tiles that hold columns
  const float *refs = a.refs + r;
  float top = row_reference(z);
  const bool moved = a.moved[r];
  const bool any = __any_sync(0xFFFFFFFFu, moved);  // the same rows in every warp
  // f over the row's quarter tiles of this warp
  constexpr int kOwn = 8 / kShare;  // of the warp's eight sums, those of this lane
  auto over_tiles = [&](auto start, auto value, auto f) {
    decltype(start) v[kOwn];
#pragma unroll
    for (int j = 0; j < kOwn; ++j) v[j] = start;
#pragma unroll kShare
    for (int i0 = 8 * warp + lane / ROWS * kOwn; i0 < filled; i0 += 256) {
#pragma unroll
      for (int j = 0; j < kOwn; ++j)
        if (i0 + j < filled) v[j] = f(v[j], value(static_cast<int64_t>(i0 + j) * a.sum_rows));
    }
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) {  // the eight sums in one order, over lanes or in the lane
      if (d >= kOwn) {
#pragma unroll
        for (int j = 0; j < kOwn; ++j) v[j] = f(v[j], from_lane(v[j], d / kOwn * ROWS));
      } else {
#pragma unroll
        for (int j = 0; j < d; ++j) v[j] = f(v[j], v[j + d]);
      }
    }
    return v[0];
  };
  auto larger = [](float x, float y) { return fmaxf(x, y); };
  auto plus = [](float x, float y) { return x + y; };
  auto plus2 = [](float2 x, float2 y) { return make_float2(x.x + y.x, x.y + y.y); };
  // the sums, or with a gradient both kinds, each times `by` of its place
  auto add_up = [&](auto by) {
    if constexpr (KEEP) {
      const float2 *sums = reinterpret_cast<const float2 *>(a.sums) + r;
      const float2 both = over_tiles(
          make_float2(0.f, 0.f),
          [&](int64_t at) {
            const float2 v = sums[at];
            const float f = by(at);
            return make_float2(v.x * f, v.y * f);
          },
          plus2);
      parts[warp][own] = both.x;
      parts_e[warp][own] = both.y;
    } else {
      const float *sums = a.sums + r;
      parts[warp][own] = over_tiles(0.f, [&](int64_t at) { return sums[at] * by(at); }, plus);
    }
  };
  if (any) {  // references differ: the largest of them first
    parts[warp][own] = over_tiles(top, [&](int64_t at) { return refs[at]; }, larger);
    __syncthreads();
    for (int w = 0; w < 32; ++w) top = fmaxf(top, parts[w][own]);
    __syncthreads();
    add_up([&](int64_t at) { return whole_exp2(refs[at] - top); });
  } else {
    add_up([](int64_t) { return 1.f; });
  }
  __syncthreads();
  if (KEEP && any) {  // the exponentials of moved rows follow their reference
    for (int i = warp; i < filled; i += 32)
      for (int l = 0; l < ROWS && r0 + l < rows; ++l) {
        if (!__shfl_sync(0xFFFFFFFFu, moved, l)) continue;
        const float by = whole_exp2(a.refs[static_cast<int64_t>(i) * a.sum_rows + r0 + l] - __shfl_sync(0xFFFFFFFFu, top, l));
        if (by == 1.f) continue;
        __nv_bfloat16 *e = reinterpret_cast<__nv_bfloat16 *>(a.e) + static_cast<int64_t>(r0 + l) * a.pitch;
        for (int64_t c = i * kCols + lane; c < a.V && c < (i + 1) * kCols; c += 32)
          e[c] = __float2bfloat16_rn(__bfloat162float(e[c]) * by);
      }
  }
  if (warp > 0 || lane >= ROWS || r0 + lane >= rows) return;
  float others = 0.f, others_e = 0.f;
  for (int w = 0; w < 32; ++w) others += parts[w][own];
  if constexpr (KEEP)
    for (int w = 0; w < 32; ++w) others_e += parts_e[w][own];
  a.moved[r] = 0;  // for the next chunk
  const float above = fmaf(z, kLog2e, -top);  // once rounded, as the others' exponents are
  const float label = exp2_fast(above), total = others + label;
  // log(total / label): where label underflows against a far larger logit, from the exponents
  const bool near = above > -60.f;
  const float loss = near ? log1pf(others / label) : logf(total) - above * kLn2;
  if (a.loss) a.loss[t] = loss;
  if (a.lse) a.lse[t] = near ? z + loss : top * kLn2 + logf(total);
  if constexpr (KEEP) a.factors[row] = make_float2(g * (others / total), others_e > 0.f ? 1.f / others_e : 0.f);
}

// dX[token] = f.x (f.y sum over the parts - W[label]). A warp per 256 columns of a row, or, where
// there are many parts (SHARE = 8), a CTA whose warps add up every eighth part each.
template <int SHARE>
__global__ void __launch_bounds__(256) sq_head_rows_kernel(const HeadArgs a, const int first) {
  __shared__ float sums[SHARE > 1 ? 7 : 1][256];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t pieces = static_cast<uint32_t>((a.D + 255) / 256);
  const uint32_t unit = SHARE > 1 ? blockIdx.x : blockIdx.x * 8 + warp;
  const int r = unit / pieces, row = first + r;
  const int rows = chunk_rows(a, first);
  const int64_t c = static_cast<int64_t>(unit % pieces) * 256 + lane * 8;
  const int tiles_m = (rows + kHeadTile - 1) / kHeadTile;
  const int parts = tiles_m > 0 ? a.parts[tiles_m - 1] + 1 : 0;
  const int64_t plane = static_cast<int64_t>(tiles_m) * kHeadTile * a.width;
  float2 f = make_float2(0.f, 0.f);
  int64_t token = 0;
  uint4 w = make_uint4(0, 0, 0, 0);
  if (r < rows) {  // what the launch before the one ahead wrote, and the weights
    f = __ldcg(a.factors + row);
    token = __ldcg(a.token + row);
    if (c < a.D && warp % SHARE == 0)
      w = __ldcg(reinterpret_cast<const uint4 *>(a.W + static_cast<int64_t>(__ldcg(a.label + row)) * a.D + c));
  }
  dependency_wait();
  dependency_start();
  if (r >= rows || (SHARE == 1 && c >= a.D)) return;
  float s[8] = {};
  if (c < a.D) {
    const float *p = a.partial + static_cast<int64_t>(r) * a.width + c + warp % SHARE * plane;
#pragma unroll 4
    for (int i = warp % SHARE; i < parts; i += SHARE, p += SHARE * plane) {
      const float4 u = reinterpret_cast<const float4 *>(p)[0], v = reinterpret_cast<const float4 *>(p)[1];
      s[0] += u.x, s[1] += u.y, s[2] += u.z, s[3] += u.w;
      s[4] += v.x, s[5] += v.y, s[6] += v.z, s[7] += v.w;
    }
  }
  if (SHARE > 1) {
    if (warp > 0)
#pragma unroll
      for (int q = 0; q < 8; ++q) sums[warp - 1][q * 32 + lane] = s[q];
    __syncthreads();
    if (warp > 0) return;
#pragma unroll
    for (int i = 0; i < SHARE - 1; ++i)
#pragma unroll
      for (int q = 0; q < 8; ++q) s[q] += sums[i][q * 32 + lane];
    if (c >= a.D) return;
  }
  const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
  uint32_t o[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const __nv_bfloat162 h2 =
        __floats2bfloat162_rn(f.x * fmaf(f.y, s[2 * q], -__uint_as_float(ww[q] << 16)),
                              f.x * fmaf(f.y, s[2 * q + 1], -__uint_as_float(ww[q] & 0xFFFF0000u)));
    o[q] = *reinterpret_cast<const uint32_t *>(&h2);
  }
  *reinterpret_cast<uint4 *>(a.dX + token * a.D + c) = make_uint4(o[0], o[1], o[2], o[3]);
}

// As many two-CTA clusters as fit on the GPU at once, or one per tile (most: no number of tiles
// that the host knows).
template <int STEP, int BK, int NT>
cudaError_t launch_head_product(const CUtensorMap &tmA, const CUtensorMap &tmB, const CUtensorMap &tmO,
                                const HeadArgs &a, int first, int64_t most, int sm_count, cudaStream_t stream) {
  using C = HeadCfg<STEP, BK, NT>;
  static int done_mask = 0;  // per device ordinal (first 31)
  static int max_clusters[32] = {0};
  int dev = 0;
  cudaGetDevice(&dev);
  if (!(done_mask & (1 << (dev & 31)))) {
    cudaError_t e =
        cudaFuncSetAttribute(sq_head_kernel<STEP, BK, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * (sm_count / 2), 1, 1);
    cfg.blockDim = dim3(C::kThreads, 1, 1);
    cfg.dynamicSmemBytes = C::kSmemBytes;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, sq_head_kernel<STEP, BK, NT>, &cfg) != cudaSuccess || n <= 0) {
      cudaGetLastError();
      n = sm_count / 2;
    }
    max_clusters[dev & 31] = n;
    done_mask |= 1 << (dev & 31);
  }
  const int64_t clusters = std::min<int64_t>(most, max_clusters[dev & 31]);
  return launch_after(sq_head_kernel<STEP, BK, NT>, static_cast<unsigned>(2 * clusters), C::kThreads, C::kSmemBytes, stream, tmA,
                      tmB, tmO, a, first);
}

}  // namespace

cudaError_t launch_head_gather(const HeadArgs &a, cudaStream_t stream) {
  if (a.T <= 1024) return launch_after(sq_head_gather_kernel<8>, static_cast<unsigned>(a.T), 256, 0, stream, a);
  return launch_after(sq_head_gather_kernel<1>, static_cast<unsigned>((a.T + 7) / 8), 256, 0, stream, a);
}

cudaError_t launch_head_chunk(const HeadArgs &a, const HeadMaps &m, int first, int sm_count, cudaStream_t stream) {
  const int rows = a.T - first < a.chunk ? a.T - first : a.chunk;
  const int64_t tiles_m = (rows + kHeadTile - 1) / kHeadTile;
  // Few tokens are bound by the weights' way from memory: stages of 128, whose rows are read 256 bytes
  // at a time. More are bound by the MMAs: stages of 64, of which five wait behind the one in work
  // (2048 against 38912 x 2048 in 163 us, 175 with 128).
  auto logits = [&](auto step) {
    constexpr int k = decltype(step)::value;
    return a.columns == 64    ? launch_head_product<k, 128, 64>
           : a.columns == 128 ? launch_head_product<k, 128, 128>
           : a.few            ? launch_head_product<k, 128, 256>
                              : launch_head_product<k, 64, 256>;
  };
  const auto product = a.dX ? logits(std::integral_constant<int, HEAD_KEEP>{}) : logits(std::integral_constant<int, HEAD_LOSS>{});
  cudaError_t e = product(m.rows, m.weights, m.e_store, a, first, tiles_m * ((a.V + a.columns - 1) / a.columns), sm_count,
                          stream);
  if (e != cudaSuccess) return e;
  auto finalize = [&](auto keep) {
    constexpr bool k = decltype(keep)::value;
    return rows <= 4 * sm_count
               ? launch_after(sq_head_finalize_kernel<4, k>, (rows + 3) / 4, 1024, 0, stream, a, first)
               : launch_after(sq_head_finalize_kernel<8, k>, (rows + 7) / 8, 1024, 0, stream, a, first);
  };
  e = a.dX ? finalize(std::true_type{}) : finalize(std::false_type{});
  if (e != cudaSuccess || !a.dX) return e;
  const int64_t tiles_d = (a.D + kHeadTile - 1) / kHeadTile;
  int64_t units = 0, parts = 0;  // the most of any number of labelled rows
  for (int64_t t = 1; t <= tiles_m; ++t) {
    units = std::max(units, t * tiles_d * (a.parts[t - 1] + 1));
    parts = std::max<int64_t>(parts, a.parts[t - 1] + 1);
  }
  const auto gradient = a.few ? a.long_sums ? launch_head_product<HEAD_GRAD_LONG, 128, 256>
                                            : launch_head_product<HEAD_GRAD, 128, 256>
                        : a.long_sums ? launch_head_product<HEAD_GRAD_LONG, 64, 256>
                                      : launch_head_product<HEAD_GRAD, 64, 256>;
  if ((e = gradient(m.e_load, m.weights_grad, m.partial, a, first, units, sm_count, stream)) != cudaSuccess) return e;
  const int64_t pieces = rows * ((a.D + 255) / 256);
  if (parts >= 8 && pieces <= 16 * static_cast<int64_t>(sm_count))  // too few warps for loads one after the other
    return launch_after(sq_head_rows_kernel<8>, static_cast<unsigned>(pieces), 256, 0, stream, a, first);
  return launch_after(sq_head_rows_kernel<1>, static_cast<unsigned>((pieces + 7) / 8), 256, 0, stream, a, first);
}

}  // namespace sqi
