// Token routing around the grouped expert linears: top-k of the router's logits with its
// gradient, the tokens sorted by expert, and the rows that travel to the experts and back.
#include <cuda_bf16.h>
#include <float.h>
#include <limits.h>

#include <algorithm>

#include "sq_internal.h"
#include "sq_launch.cuh"

namespace sqi {
namespace {

constexpr uint32_t kAll = 0xFFFFFFFFu;

// ---------------------------------------------------------------- router
//
// z[T, E] -> the k largest logits of each token, ties to the lowest expert. A NaN or -inf logit
// is never chosen; +inf counts as the largest finite number.
//
// LANES lanes of a warp take a token, PER logits each, in groups of four that every lane sorts
// (stably, so equal logits stay in the order of their experts). Each of k rounds takes the
// largest of the lanes' largest and shifts it out of its group. Bound by instructions: with a
// warp per token and the logits as ordered integers, 522 of them a token (32768 tokens, top-8
// of 128: 19 us); eight lanes a token share them among four, about 260 a token (14.7 us, both
// profiled from a cold cache).

// A logit as it is ranked; -inf, and so NaN, is never chosen.
__device__ __forceinline__ float rank_value(float z) { return fminf(fmaxf(z, -INFINITY), FLT_MAX); }

__device__ __forceinline__ float load_logit(const float *p) { return *p; }
__device__ __forceinline__ float load_logit(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void load_logits4(const float *p, float *v) {
  const float4 q = *reinterpret_cast<const float4 *>(p);
  v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
}
__device__ __forceinline__ void load_logits4(const __nv_bfloat16 *p, float *v) {
  const uint2 q = *reinterpret_cast<const uint2 *>(p);
  v[0] = __uint_as_float(q.x << 16), v[1] = __uint_as_float(q.x & 0xFFFF0000u);
  v[2] = __uint_as_float(q.y << 16), v[3] = __uint_as_float(q.y & 0xFFFF0000u);
}
__device__ __forceinline__ void store_logits4(float *p, const float *v) {
  *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store_logits4(__nv_bfloat16 *p, const float *v) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
  *reinterpret_cast<uint2 *>(p) =
      make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}
__device__ __forceinline__ void store_logit(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_logit(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// e^d for d <= 0. The product's rounding adds |d| 2^-24 of the value: less than 1e-6 where it counts.
__device__ __forceinline__ float exp_of(float d) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(d * 1.4426950408889634f));
  return y;
}

// The same to 2^-22 for any d, of the weights themselves: what the product and the constant round off
// comes back to first order.
__device__ __forceinline__ float exp_close(float d) {
  constexpr float kLog2e = 1.44269504f, kRest = 1.92596299e-8f;  // log2(e) = kLog2e + kRest
  d = fmaxf(d, -200.f);  // 0 from there on
  const float t = d * kLog2e, rest = fmaf(d, kRest, fmaf(d, kLog2e, -t));
  const float y = exp_of(d);
  return fmaf(y, rest * 0.6931471805599453f, y);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
  return v;
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int d = LANES / 2; d > 0; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
  return v;
}
template <int LANES>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int d = LANES / 2; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, d));
  return v;
}

// Expert of a lane's element i: four neighbours at a time (WIDE, where E % 4 == 0), or one.
template <int LANES, bool WIDE>
__device__ __forceinline__ int expert_of(int i, int lane) {
  return WIDE ? (i / 4) * 4 * LANES + lane * 4 + i % 4 : i * LANES + lane;
}
// The ranked logits of one token; -inf past the last expert.
template <int LANES, bool WIDE, int PER, typename T>
__device__ __forceinline__ void load_row(const T *row, int E, int lane, bool on, float (&z)[PER]) {
#pragma unroll
  for (int i = 0; i < PER; i += WIDE ? 4 : 1) {
    const int e = expert_of<LANES, WIDE>(i, lane);
    if (WIDE) {
      float v[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (on && e < E) load_logits4(row + e, v);
#pragma unroll
      for (int c = 0; c < 4; ++c) z[i + c] = rank_value(v[c]);
    } else {
      z[i] = on && e < E ? rank_value(load_logit(row + e)) : -INFINITY;
    }
  }
}

// k <= LANES: lane j of a token keeps its slot j.
template <int LANES, bool WIDE, int PER, typename T>
__global__ void __launch_bounds__(256)
    sq_route_kernel(int64_t tokens, int E, int k, const T *logits, const uint8_t *valid,
                    bool normalize, int *__restrict__ experts, float *__restrict__ weights) {
  constexpr int kGroups = PER / 4;
  dependency_wait();
  dependency_start();
  const int lane = threadIdx.x % LANES, base = threadIdx.x & 31 & ~(LANES - 1);
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
  const bool on = t < tokens && (!valid || valid[t]);
  float z[PER];
  load_row<LANES, WIDE, PER>(logits + (on ? t * E : 0), E, lane, on, z);
  float top = z[0];
#pragma unroll
  for (int i = 1; i < PER; ++i) top = fmaxf(top, z[i]);
  top = lanes_max<LANES>(top);
  float total = 0.f;
  if (!normalize) {
#pragma unroll
    for (int i = 0; i < PER; ++i) total += exp_of(z[i] - top);  // not a number without any logit, and unused
    total = lanes_sum<LANES>(total);
  }
  uint32_t order[kGroups];  // places within the group of its sorted logits, two bits each
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    uint32_t at[4] = {0, 1, 2, 3};
    float *v = z + 4 * g;
#pragma unroll
    for (int n = 3; n > 0; --n)
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const bool swap = v[i + 1] > v[i];
        const float x = swap ? v[i + 1] : v[i];
        const uint32_t p = swap ? at[i + 1] : at[i];
        v[i + 1] = swap ? v[i] : v[i + 1];
        at[i + 1] = swap ? at[i] : at[i + 1];
        v[i] = x;
        at[i] = p;
      }
    order[g] = at[0] | at[1] << 2 | at[2] << 4 | at[3] << 6;
  }
  int my_expert = -1;
  float my_value = -INFINITY;
  for (int j = 0; j < k; ++j) {
    float best = z[0];
    uint32_t places = order[0];
    int group = 0;
#pragma unroll
    for (int g = 1; g < kGroups; ++g) {
      const bool more = z[4 * g] > best;
      best = more ? z[4 * g] : best;
      places = more ? order[g] : places;
      group = more ? g : group;
    }
    const float won = lanes_max<LANES>(best);
    if (!__any_sync(kAll, won > -INFINITY)) break;
    int e = expert_of<LANES, WIDE>(4 * group + static_cast<int>(places & 3u), lane);
    bool mine = best == won;
    const uint32_t same = (__ballot_sync(kAll, mine) >> base) & (LANES == 32 ? kAll : (1u << LANES % 32) - 1u);
    if (__any_sync(kAll, (same & (same - 1)) != 0)) {  // equal logits in several lanes: the lowest expert
      int lowest = mine ? e : INT_MAX;
#pragma unroll
      for (int d = LANES / 2; d > 0; d >>= 1) lowest = min(lowest, __shfl_xor_sync(kAll, lowest, d));
      mine = mine && e == lowest;
      e = lowest;
    } else {
      e = __shfl_sync(kAll, e, base + __ffs(same) - 1);
    }
    if (lane == j && won > -INFINITY) {
      my_expert = e;
      my_value = won;
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const bool pop = mine && group == g;
      z[4 * g] = pop ? z[4 * g + 1] : z[4 * g];
      z[4 * g + 1] = pop ? z[4 * g + 2] : z[4 * g + 1];
      z[4 * g + 2] = pop ? z[4 * g + 3] : z[4 * g + 2];
      z[4 * g + 3] = pop ? -INFINITY : z[4 * g + 3];
      order[g] = pop ? order[g] >> 2 : order[g];
    }
  }
  const float w = my_expert >= 0 ? exp_close(my_value - top) : 0.f;
  if (normalize) total = lanes_sum<LANES>(w);
  if (t < tokens && lane < k) {
    experts[t * k + lane] = my_expert;
    weights[t * k + lane] = my_expert >= 0 ? w / total : 0.f;
  }
}

// dz_e = q_e (dw_e - sum_j q_j dw_j), q the weights over the chosen experts (normalize) or the
// softmax over all; dw_e is 0 for an expert that was not chosen. The softmax is formed again
// from the logits: keeping it would cost a write and the same read.
template <int LANES, bool WIDE, int PER, typename T>
__global__ void __launch_bounds__(256)
    sq_route_grad_kernel(int64_t tokens, int E, int k, const T *logits, const int *experts,
                         const float *dweights, bool normalize, T *__restrict__ dlogits) {
  dependency_wait();
  dependency_start();
  const int lane = threadIdx.x % LANES;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
  const bool slot = t < tokens && lane < k;
  const int64_t row = t < tokens ? t * E : 0;
  int e = slot ? experts[t * k + lane] : -1;
  if (e >= E) e = -1;
  const float dw = e >= 0 ? dweights[t * k + lane] : 0.f;
  const float z = e >= 0 ? rank_value(load_logit(logits + row + e)) : -INFINITY;
  const bool any = lanes_max<LANES>(z) > -INFINITY;  // the token has an expert
  float dense[PER], top = lanes_max<LANES>(z);
  if (!normalize) {
    load_row<LANES, WIDE, PER>(logits + row, E, lane, any, dense);
    top = dense[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) top = fmaxf(top, dense[i]);
    top = lanes_max<LANES>(top);
  }
  const float mine = z > -INFINITY ? exp_close(z - top) : 0.f;
  float total = 0.f;
  if (normalize) {
    total = mine;
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      dense[i] = exp_of(dense[i] - top);
      total += dense[i];
    }
  }
  total = lanes_sum<LANES>(total);
  const float by = any ? 1.f / total : 0.f;
  const float share = mine * by;
  const float inner = lanes_sum<LANES>(share > 0.f ? share * dw : 0.f);
  const float scale = -by * inner;
  if (t < tokens) {
#pragma unroll
    for (int i = 0; i < PER; i += WIDE ? 4 : 1) {
      const int at = expert_of<LANES, WIDE>(i, lane);
      if (at >= E) continue;
      float v[4];
#pragma unroll
      for (int c = 0; c < (WIDE ? 4 : 1); ++c) v[c] = normalize || !any ? 0.f : dense[i + c] * scale;
      if (WIDE)
        store_logits4(dlogits + row + at, v);
      else
        store_logit(dlogits + row + at, v[0]);
    }
  }
  __syncwarp();  // the chosen experts' values go over the row's
  if (z > -INFINITY) store_logit(dlogits + row + e, share * (dw - inner));
}

// ---------------------------------------------------------------- tokens by expert
//
// Stable counting sort of the n slots t * k + j by expert. Each warp owns a run of neighbouring
// slots and a histogram row; the prefix over warps, CTAs and experts gives each its first row, and
// rows are handed out in slot order, so the order never depends on timing. Up to kSortOne slots
// take one CTA; more take a launch that counts per CTA and one that adds up the counts and places
// the slots (each CTA reads all CTAs' counts: G x E words from the L2).

constexpr int kSortStep = 2;  // loads of 32 slots in flight
constexpr int64_t kSortOne = 4096;
constexpr int64_t kSortMany = 2048;  // slots of a CTA at least, of several
constexpr int kSortThreads = 1024;   // of a CTA, of several

// EARLY: ahead of the launch's wait, from the L2, where older launches' results are.
template <bool EARLY = false>
__device__ __forceinline__ void load_slots(const int *experts, int64_t at, int64_t end, int E, int lane,
                                           int (&e)[kSortStep]) {
#pragma unroll
  for (int s = 0; s < kSortStep; ++s) {
    const int64_t i = at + 32 * s + lane;
    e[s] = i < end ? (EARLY ? __ldcg(experts + i) : experts[i]) : -1;
    if (e[s] >= E) e[s] = -1;
  }
}

// The lanes with the same expert (of `bits` bits) as this one, among those that have one: a vote per
// bit (0.5 us less than __match_any_sync over 262144 slots of 128 experts).
__device__ __forceinline__ uint32_t same_expert(int e, int bits) {
  uint32_t same = __ballot_sync(kAll, e >= 0);
  for (int b = 0; b < bits; ++b) {
    const uint32_t set = __ballot_sync(kAll, (e >> b) & 1);
    same &= (e >> b) & 1 ? set : ~set;
  }
  return same;
}

__global__ void __launch_bounds__(kSortThreads)
    sq_sort_count_kernel(int64_t n, int E, int64_t per, const int *experts, int *__restrict__ counts) {
  extern __shared__ int sort_smem[];
  dependency_wait();
  dependency_start();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = kSortThreads / 32;
  for (int i = threadIdx.x; i < E; i += kSortThreads) sort_smem[i] = 0;
  __syncthreads();
  const int64_t begin = blockIdx.x * per, end = min(n, begin + per);
  for (int64_t at = begin + warp * 32 * kSortStep; at < end; at += warps * 32 * kSortStep) {
    int e[kSortStep];
    load_slots(experts, at, end, E, lane, e);
#pragma unroll
    for (int s = 0; s < kSortStep; ++s)
      if (e[s] >= 0) atomicAdd(sort_smem + e[s], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < E; i += kSortThreads) counts[static_cast<int64_t>(blockIdx.x) * E + i] = sort_smem[i];
}

// counts: [gridDim.x, E] of the launch before, or null for the one CTA that takes all slots.
__global__ void __launch_bounds__(1024)
    sq_sort_kernel(int64_t n, int E, int64_t per, const int *experts, const int *counts,
                   int64_t *__restrict__ offsets, int *__restrict__ row_of, int *__restrict__ slot_of) {
  extern __shared__ int sort_smem[];
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int *hist = sort_smem;           // [warps][E]
  int *all = hist + warps * E;     // [E] slots of an expert
  int *first = all + E;            // [E] those of earlier CTAs, then the first row of this one's
  __shared__ int scan[32];
  const int64_t cta_end = min(n, (blockIdx.x + 1) * per);
  const int64_t per_warp = (per + warps * 32 - 1) / (warps * 32) * 32;
  const int64_t begin = min(cta_end, blockIdx.x * per + warp * per_warp);
  const int64_t end = min(cta_end, begin + per_warp);
  for (int i = threadIdx.x; i < (warps + 2) * E; i += blockDim.x) hist[i] = 0;
  // behind a count launch `experts` is complete already; each CTA counts its own slots meanwhile
  if (!counts) {
    dependency_wait();
    dependency_start();
  }
  __syncthreads();
  int *mine = hist + warp * E;
  for (int64_t at = begin; at < end; at += 32 * kSortStep) {
    int e[kSortStep];
    load_slots<true>(experts, at, end, E, lane, e);
#pragma unroll
    for (int s = 0; s < kSortStep; ++s)
      if (e[s] >= 0) atomicAdd(mine + e[s], 1);
  }
  if (counts) {
    dependency_wait();  // the counts are complete
    dependency_start();
    // a group of threads takes every groups-th CTA's counts, a thread one expert of them
    const int width = min(static_cast<int>(blockDim.x), (E + 31) / 32 * 32);
    const int groups = blockDim.x / width, group = threadIdx.x / width;
    for (int e = threadIdx.x % width; e < E && group < groups; e += width) {
      int sum = 0, before = 0;
      for (int b0 = group; b0 < gridDim.x; b0 += groups * 8) {
        int c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int b = b0 + i * groups;
          c[i] = b < gridDim.x ? counts[b * E + e] : 0;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sum += c[i];
          before += b0 + i * groups < blockIdx.x ? c[i] : 0;
        }
      }
      atomicAdd(all + e, sum);
      atomicAdd(first + e, before);
    }
  }
  __syncthreads();
  int carry = 0;
  for (int e0 = 0; e0 < E; e0 += blockDim.x) {  // the experts' prefix, a block width at a time
    const int e = e0 + threadIdx.x;
    int here = 0;
    if (e < E) {
      for (int w = 0; w < warps; ++w) {
        const int c = hist[w * E + e];
        hist[w * E + e] = here;
        here += c;
      }
      if (counts) here = all[e];
    }
    int incl = here;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(kAll, incl, d);
      if (lane >= d) incl += v;
    }
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    if (warp == 0) {
      int v = lane < warps ? scan[lane] : 0;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(kAll, v, d);
        if (lane >= d) v += u;
      }
      scan[lane] = v;
    }
    __syncthreads();
    const int start = carry + incl - here + (warp > 0 ? scan[warp - 1] : 0);
    carry += scan[31];
    if (e < E) {
      first[e] += start;
      if (blockIdx.x == 0) offsets[e] = start;
    }
    __syncthreads();
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) offsets[E] = carry;
  const int bits = 32 - __clz(E - 1);  // of the largest expert (none for one expert)
  for (int64_t at = begin; at < end; at += 32 * kSortStep) {
    int e[kSortStep];
    load_slots(experts, at, end, E, lane, e);
#pragma unroll
    for (int s = 0; s < kSortStep; ++s) {
      const int64_t i = at + 32 * s + lane;
      const uint32_t same = same_expert(e[s], bits);
      int row = -1;
      if (e[s] >= 0) row = first[e[s]] + mine[e[s]] + __popc(same & ((1u << lane) - 1));
      __syncwarp();
      if (e[s] >= 0 && (same >> lane) == 1u) mine[e[s]] += __popc(same);  // its last slot here
      __syncwarp();
      if (i < end) {
        row_of[i] = row;
        if (row >= 0) slot_of[row] = static_cast<int>(i);
      }
    }
  }
  for (int64_t r = carry + static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; r < n;
       r += static_cast<int64_t>(gridDim.x) * blockDim.x)
    slot_of[r] = -1;
}

// ---------------------------------------------------------------- rows to the experts and back
//
// bf16 rows of D elements, moved 8 (16 bytes) per lane. A row index outside [0, rows) marks a
// slot that no expert serves.

// 16 bytes, or zeros where not `on`. Loads of several rows are issued one after the other in both
// forms; with a branch around each the backward pass of 2677 tokens of width 1496 from 4 experts
// took 29.1 us, 24.7 without. load_or_first reads the tensor's first elements instead, in fewer
// registers: the sum of eight rows stays below 64 (2048 tokens of width 2048: 15.2 us, 16.4 with
// predicates; of one row, 32768 of width 4096, 82.3 and 80.7).
__device__ __forceinline__ uint4 load_row16(const uint16_t *p, bool on) {
  uint4 v;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
      "@p ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
      : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w)
      : "l"(p), "r"(static_cast<int>(on))
      : "memory");
  return v;
}
__device__ __forceinline__ uint4 load_or_first(const uint16_t *p, int64_t at, bool on) {
  const uint4 v = *reinterpret_cast<const uint4 *>(p + (on ? at : 0));
  return make_uint4(on ? v.x : 0, on ? v.y : 0, on ? v.z : 0, on ? v.w : 0);
}
__device__ __forceinline__ void store_row16(uint16_t *p, const uint4 &v) { *reinterpret_cast<uint4 *>(p) = v; }
__device__ __forceinline__ void unpack8(const uint4 &q, float (&v)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t *>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

constexpr int kMoveVecs = 2;  // 16-byte loads of a lane in flight
constexpr int kMoveCols = 32 * 8 * kMoveVecs;

// Xs[row_of[t, j]] = X[t]; rows whose slot_of is negative are zero. A warp takes kMoveCols
// columns of one token, read once and written k times.
__global__ void __launch_bounds__(256)
    sq_dispatch_kernel(uint32_t units, uint32_t pieces, int k, int64_t D, int64_t rows, const uint16_t *X,
                       const int *row_of, const int *slot_of, uint16_t *__restrict__ Xs) {
  const int lane = threadIdx.x & 31;
  const uint32_t unit = blockIdx.x * 8 + (threadIdx.x >> 5);
  dependency_wait();
  dependency_start();
  if (unit >= units) return;
  const int64_t t = unit / pieces;
  const int64_t c0 = static_cast<int64_t>(unit % pieces) * kMoveCols + lane * 8;
  const int64_t slot = t * k + lane;
  int64_t row = -1;
  bool empty = false;
  if (lane < k) {
    row = row_of[slot];
    if (row >= rows) row = -1;
    empty = slot < rows && slot_of[slot] < 0;
  }
  uint4 v[kMoveVecs];
  const bool read = __any_sync(kAll, row >= 0);
#pragma unroll
  for (int i = 0; i < kMoveVecs; ++i)
    v[i] = load_row16(X + t * D + c0 + 256 * i, read && c0 + 256 * i < D);
  for (int j = 0; j < k; ++j) {
    const int64_t to = __shfl_sync(kAll, row, j);
    if (to < 0) continue;
#pragma unroll
    for (int i = 0; i < kMoveVecs; ++i)
      if (c0 + 256 * i < D) store_row16(Xs + to * D + c0 + 256 * i, v[i]);
  }
  for (uint32_t m = __ballot_sync(kAll, empty); m; m &= m - 1) {
    const int64_t to = t * k + __ffs(m) - 1;
#pragma unroll
    for (int i = 0; i < kMoveVecs; ++i)
      if (c0 + 256 * i < D) store_row16(Xs + to * D + c0 + 256 * i, make_uint4(0, 0, 0, 0));
  }
}

// Rows that a warp has in flight (ROWS of the token's k) and 256-column pieces of each (COLS): 8
// loads of 16 bytes a lane where k > 4, 4 below. With the rows of one piece alone, k = 1 left one
// load in flight (17182 tokens of width 1544, backward: 92 us instead of 47). The gradient, whose
// stores keep the next piece's loads back, takes two pieces of four rows (8192 tokens of width 2880:
// 68 us, 73 with one).
template <bool GRAD, typename F>
cudaError_t with_flight(int k, F f) {
  using std::integral_constant;
  if (k == 1) return f(integral_constant<int, 1>{}, integral_constant<int, 4>{});
  if (k == 2) return f(integral_constant<int, 2>{}, integral_constant<int, 2>{});
  if (k <= 4) return f(integral_constant<int, 4>{}, integral_constant<int, GRAD ? 2 : 1>{});
  return f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
}

// Y[t] = sum_j w[t, j] Ys[row_of[t, j]] in fp32 in the order of j, rounded once (without
// weights: the plain sum, the gradient of the dispatch). `share` warps per token, which take its
// columns in turn. Bound by memory; at most 64 registers a thread, so 32 warps per SM (with 97
// registers and 16 warps a 2880-wide batch of 1999 tokens took 19 us instead of 12).
template <int ROWS, int COLS>
__global__ void __launch_bounds__(256, 4)
    sq_combine_kernel(int64_t tokens, int k, int D, int rows, int share, const uint16_t *Ys,
                      const int *row_of, const float *weights, uint16_t *__restrict__ Y) {
  dependency_wait();
  dependency_start();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (8 / share) + warp / share;
  if (t >= tokens) return;
  int row = -1;  // lanes past k hold none
  float w = 0.f;
  if (lane < k) {
    row = row_of[t * k + lane];
    if (row >= rows) row = -1;
    if (row >= 0) w = weights ? weights[t * k + lane] : 1.f;  // a slot without a row adds 0 * 0
  }
  for (int c0 = (warp % share) * 256 * COLS; c0 < D; c0 += share * 256 * COLS) {
    const int c = c0 + lane * 8;
    float sum[COLS][8] = {};
    for (int j0 = 0; j0 < k; j0 += ROWS) {
      uint4 v[ROWS][COLS];
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const int at = __shfl_sync(kAll, row, j0 + i);
#pragma unroll
        for (int q = 0; q < COLS; ++q) {
          const int64_t from = static_cast<int64_t>(at) * D + (c + 256 * q);
          const bool on = at >= 0 && c + 256 * q < D;
          v[i][q] = ROWS > 1 ? load_or_first(Ys, from, on) : load_row16(Ys + from, on);
        }
      }
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const float wi = __shfl_sync(kAll, w, j0 + i);
#pragma unroll
        for (int q = 0; q < COLS; ++q) {
          float x[8];
          unpack8(v[i][q], x);
#pragma unroll
          for (int e = 0; e < 8; ++e) sum[q][e] = fmaf(wi, x[e], sum[q][e]);
        }
      }
    }
#pragma unroll
    for (int q = 0; q < COLS; ++q)
      if (c + 256 * q < D) store_row16(Y + t * D + c + 256 * q, pack8(sum[q]));
  }
}

// dYs[row_of[t, j]] = w[t, j] dY[t] and dw[t, j] = sum_d dY[t, d] Ys[row_of[t, j], d]. One token
// per `share` warps of the CTA, which take its columns in turn; their sums are added in order.
// Bound by memory: 32768 tokens of width 2048 to 8 experts move 2.2 GB in 328 us.
template <int ROWS, int COLS>
__global__ void __launch_bounds__(256)
    sq_combine_grad_kernel(int64_t tokens, int k, int D, int rows, int share, const uint16_t *dY,
                           const uint16_t *Ys, const int *row_of,
                           const int *slot_of, const float *weights,
                           uint16_t *__restrict__ dYs, float *__restrict__ dweights) {
  __shared__ float partial[8][32];
  dependency_wait();
  dependency_start();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int part = warp % share;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (8 / share) + warp / share;
  float dw = 0.f;  // lane j: this warp's part of dw[t, j]
  if (t < tokens) {
    const int64_t slot = t * k + lane;
    int row = -1;
    float w = 0.f;
    bool empty = false;
    if (lane < k) {
      row = row_of[slot];
      if (row >= rows) row = -1;
      w = weights[slot];
      empty = slot < rows && slot_of[slot] < 0;
    }
    const uint32_t clear = __ballot_sync(kAll, empty);
    for (int j0 = 0; j0 < k; j0 += ROWS) {
      int at[ROWS];
      float wj[ROWS], acc[ROWS];
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {  // lanes past k hold row -1
        at[i] = __shfl_sync(kAll, row, j0 + i);
        wj[i] = __shfl_sync(kAll, w, j0 + i);
        acc[i] = 0.f;
      }
      for (int c = part * 256 * COLS + lane * 8; c < D; c += share * 256 * COLS) {
        uint4 g[COLS], v[ROWS][COLS];
#pragma unroll
        for (int q = 0; q < COLS; ++q) {
          const bool in = c + 256 * q < D;
#pragma unroll
          for (int i = 0; i < ROWS; ++i)
            v[i][q] = load_row16(Ys + static_cast<int64_t>(at[i]) * D + (c + 256 * q), in && at[i] >= 0);
          g[q] = load_row16(dY + t * D + c + 256 * q, in);
        }
#pragma unroll
        for (int q = 0; q < COLS; ++q) {
          if (c + 256 * q >= D) break;
          float d[8];
          unpack8(g[q], d);
#pragma unroll
          for (int i = 0; i < ROWS; ++i) {
            if (at[i] < 0) continue;
            float x[8], o[8];
            unpack8(v[i][q], x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              acc[i] = fmaf(d[e], x[e], acc[i]);
              o[e] = wj[i] * d[e];
            }
            store_row16(dYs + static_cast<int64_t>(at[i]) * D + (c + 256 * q), pack8(o));
          }
        }
      }
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const float s = warp_sum(acc[i]);
        if (lane == j0 + i) dw = s;
      }
    }
    for (uint32_t m = clear; m; m &= m - 1) {
      const int64_t to = t * k + __ffs(m) - 1;
      for (int c = part * 256 + lane * 8; c < D; c += share * 256)
        store_row16(dYs + to * D + c, make_uint4(0, 0, 0, 0));
    }
  }
  if (share > 1) {
    partial[warp][lane] = dw;
    __syncthreads();
    if (part == 0)
      for (int i = 1; i < share; ++i) dw += partial[warp + i][lane];
  }
  if (part == 0 && t < tokens && lane < k) dweights[t * k + lane] = dw;
}

// Lanes of a token and logits of a lane: as few lanes as hold the slots and at most 16 logits each
// (32768 tokens, router, sort and gradient: top-16 of 128 in 39.0 us with 16 lanes, 45.8 with 32;
// top-8 of 256 in 41.0, 43.3; with 32 logits for eight lanes 38.4, but 1000 tokens 20.3 instead of
// 19.4). Not a rule on the tokens: a softmax keeps its bits in any batch.
template <bool WIDE, typename F>
void with_row_shape(int E, int k, F f) {
  auto go = [&](auto lanes, auto per) { f(lanes, std::integral_constant<bool, WIDE>{}, per); };
  using std::integral_constant;
  if (k <= 8 && E <= 32)
    go(integral_constant<int, 8>{}, integral_constant<int, 4>{});
  else if (k <= 8 && E <= 64)
    go(integral_constant<int, 8>{}, integral_constant<int, 8>{});
  else if (k <= 8 && E <= 128)
    go(integral_constant<int, 8>{}, integral_constant<int, 16>{});
  else if (k <= 16 && E <= 128)
    go(integral_constant<int, 16>{}, integral_constant<int, 8>{});
  else if (k <= 16 && E <= 256)
    go(integral_constant<int, 16>{}, integral_constant<int, 16>{});
  else if (E <= 128)
    go(integral_constant<int, 32>{}, integral_constant<int, 4>{});
  else if (E <= 256)
    go(integral_constant<int, 32>{}, integral_constant<int, 8>{});
  else if (E <= 512)
    go(integral_constant<int, 32>{}, integral_constant<int, 16>{});
  else
    go(integral_constant<int, 32>{}, integral_constant<int, 32>{});
}

// f(logits pointer of their type, lanes, wide, per) for this launch.
template <typename F>
void with_route(bool bf16, const void *logits, int E, int k, F f) {
  auto typed = [&](auto *z) {
    auto shaped = [&](auto lanes, auto wide, auto per) { f(z, lanes, wide, per); };
    if (E % 4 == 0)
      with_row_shape<true>(E, k, shaped);
    else
      with_row_shape<false>(E, k, shaped);
  };
  if (bf16)
    typed(static_cast<const __nv_bfloat16 *>(logits));
  else
    typed(static_cast<const float *>(logits));
}

}  // namespace

cudaError_t launch_route(int64_t T, int E, int k, bool bf16, const void *logits, const uint8_t *valid, bool normalize,
                         int *experts, float *weights, cudaStream_t stream) {
  cudaError_t status = cudaSuccess;
  with_route(bf16, logits, E, k, [&](auto *z, auto lanes, auto wide, auto per) {
    using L = std::remove_const_t<std::remove_pointer_t<decltype(z)>>;
    constexpr int kTokens = 256 / lanes.value;
    status = launch_after(sq_route_kernel<lanes.value, wide.value, per.value, L>,
                          static_cast<unsigned>((T + kTokens - 1) / kTokens), 256, 0, stream, T, E, k, z, valid,
                          normalize, experts, weights);
  });
  return status;
}

cudaError_t launch_route_grad(int64_t T, int E, int k, bool bf16, const void *logits, const int *experts,
                              const float *dweights, bool normalize, void *dlogits, cudaStream_t stream) {
  cudaError_t status = cudaSuccess;
  with_route(bf16, logits, E, k, [&](auto *z, auto lanes, auto wide, auto per) {
    using L = std::remove_const_t<std::remove_pointer_t<decltype(z)>>;
    constexpr int kTokens = 256 / lanes.value;
    status = launch_after(sq_route_grad_kernel<lanes.value, wide.value, per.value, L>,
                          static_cast<unsigned>((T + kTokens - 1) / kTokens), 256, 0, stream, T, E, k, z, experts,
                          dweights, normalize, static_cast<L *>(dlogits));
  });
  return status;
}

static int64_t sort_per_cta(int64_t n, int sm_count) {
  if (n <= kSortOne) return n;
  const int64_t even = (n + sm_count - 1) / sm_count;
  return std::max(kSortMany, (even + kSortThreads - 1) / kSortThreads * kSortThreads);
}

size_t sort_workspace(int64_t n, int E, int sm_count) {
  if (n <= kSortOne) return 0;
  const int64_t per = sort_per_cta(n, sm_count);
  return static_cast<size_t>((n + per - 1) / per) * E * sizeof(int);
}

cudaError_t launch_sort(int64_t n, int E, const int *experts, int64_t *offsets, int *row_of, int *slot_of,
                        int *workspace, int sm_count, cudaStream_t stream) {
  const bool one = n <= kSortOne;
  const int64_t per = sort_per_cta(n, sm_count);
  const unsigned ctas = one ? 1 : static_cast<unsigned>((n + per - 1) / per);
  // few slots: eight warps, whose prefix is short
  const int threads = one ? (n <= 1024 ? 256 : 1024) : kSortThreads;
  if (!one) {
    const cudaError_t e =
        launch_after(sq_sort_count_kernel, ctas, kSortThreads, E * sizeof(int), stream, n, E, per, experts, workspace);
    if (e != cudaSuccess) return e;
  }
  const size_t smem = (static_cast<size_t>(threads / 32) + 2) * E * sizeof(int);
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(sq_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               34 * kRouteMaxExperts * static_cast<int>(sizeof(int)));
    if (e != cudaSuccess) return e;
  }
  return launch_after(sq_sort_kernel, ctas, threads, smem, stream, n, E, per, experts, one ? nullptr : workspace, offsets,
                      row_of, slot_of);
}

// Warps of a token: as many as it takes for `warps` in all, at most one per 256 columns.
static int warps_of_token(int64_t T, int64_t D, int64_t warps) {
  int share = 1;
  while (share < 8 && T * share < warps && share * 256 < D) share *= 2;
  return share;
}

cudaError_t launch_dispatch(int64_t T, int k, int64_t D, int64_t rows, const uint16_t *X, const int *row_of,
                            const int *slot_of, uint16_t *Xs, cudaStream_t stream) {
  const uint32_t pieces = static_cast<uint32_t>((D + kMoveCols - 1) / kMoveCols);
  const uint32_t units = static_cast<uint32_t>(T) * pieces;
  return launch_after(sq_dispatch_kernel, (units + 7) / 8, 256, 0, stream, units, pieces, k, D, rows, X, row_of, slot_of,
                      Xs);
}

cudaError_t launch_combine(int64_t T, int k, int64_t D, int64_t rows, const uint16_t *Ys, const int *row_of,
                           const float *weights, uint16_t *Y, int sm_count, cudaStream_t stream) {
  const int share = warps_of_token(T, D, 32 * static_cast<int64_t>(sm_count));
  const int64_t per = 8 / share;
  if (rows == 0) Ys = Y;  // no rows and perhaps no tensor: load_or_first still needs one to read
  return with_flight<false>(k, [&](auto r, auto c) {
    return launch_after(sq_combine_kernel<r.value, c.value>, static_cast<unsigned>((T + per - 1) / per), 256, 0, stream, T,
                        k, D, rows, share, Ys, row_of, weights, Y);
  });
}

cudaError_t launch_combine_grad(int64_t T, int k, int64_t D, int64_t rows, const uint16_t *dY, const uint16_t *Ys,
                                const int *row_of, const int *slot_of, const float *weights, uint16_t *dYs,
                                float *dweights, int sm_count, cudaStream_t stream) {
  const int share = warps_of_token(T, D, 16 * static_cast<int64_t>(sm_count));
  const int64_t per = 8 / share;
  return with_flight<true>(k, [&](auto r, auto c) {
    return launch_after(sq_combine_grad_kernel<r.value, c.value>, static_cast<unsigned>((T + per - 1) / per), 256, 0,
                        stream, T, k, D, rows, share, dY, Ys, row_of, slot_of, weights, dYs, dweights);
  });
}

}  // namespace sqi
