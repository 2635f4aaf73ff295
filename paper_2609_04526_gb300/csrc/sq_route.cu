// Token routing around the grouped expert linears: top-k of the router's logits with its
// gradient, the tokens sorted by expert, and the rows that travel to the experts and back.
#include <cuda_bf16.h>
#include <float.h>
#include <limits.h>

#include <algorithm>

#include "sq_internal.h"

namespace sqi {
namespace {

constexpr uint32_t kAll = 0xFFFFFFFFu;

// ---------------------------------------------------------------- router
//
// z[T, E] -> the k largest logits of each token, ties to the lowest expert. A NaN or -inf logit
// is never chosen; +inf counts as the largest finite number. One warp per token.

// A logit as an unsigned key with the order of the numbers; 0 for one that is never chosen.
__device__ __forceinline__ uint32_t order_key(float z) {
  if (!(z > -INFINITY)) return 0u;
  const uint32_t u = __float_as_uint(fminf(z, FLT_MAX) + 0.0f);  // -0 becomes +0
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

__device__ __forceinline__ float load_logit(const float *p) { return __ldg(p); }
__device__ __forceinline__ float load_logit(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void load_logits4(const float *p, float (&v)[4]) {
  const float4 q = __ldg(reinterpret_cast<const float4 *>(p));
  v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
}
__device__ __forceinline__ void load_logits4(const __nv_bfloat16 *p, float (&v)[4]) {
  const uint2 q = __ldg(reinterpret_cast<const uint2 *>(p));
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

// Expert of element i of a lane: lanes take VEC neighbours at a time.
template <int VEC>
__device__ __forceinline__ int expert_of(int i, int lane) {
  return (i / VEC) * 32 * VEC + lane * VEC + i % VEC;
}
// The logits of one token, PER per lane; absent experts as NaN.
template <int VEC, int PER, typename T>
__device__ __forceinline__ void load_row(const T *row, int E, int lane, float (&z)[PER]) {
#pragma unroll
  for (int i = 0; i < PER; i += VEC) {
    const int e = expert_of<VEC>(i, lane);
    if (VEC == 4) {
      float v[4] = {NAN, NAN, NAN, NAN};
      if (e < E) load_logits4(row + e, v);
#pragma unroll
      for (int c = 0; c < 4; ++c) z[i + c] = v[c];
    } else {
      z[i] = e < E ? load_logit(row + e) : NAN;
    }
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
  return v;
}

// The winners of a lane in descending order: up to 8 logits are sorted first (stably, so equal
// ones stay in the order of their experts) and a winner is shifted out; more are searched again
// after each. 32768 tokens of 128 logits, top-8: 22.3 us with the search.
template <int VEC, int PER>
struct LaneTop {
  static constexpr bool kSorted = PER <= 8;
  uint32_t key[PER];
  int expert[PER];
  __device__ __forceinline__ LaneTop(const float (&z)[PER], int lane) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      key[i] = order_key(z[i]);
      expert[i] = expert_of<VEC>(i, lane);
    }
    if (kSorted) {
#pragma unroll
      for (int n = PER - 1; n > 0; --n)
#pragma unroll
        for (int i = 0; i < n; ++i) {
          const bool swap = key[i + 1] > key[i];
          const uint32_t k = swap ? key[i + 1] : key[i];
          const int e = swap ? expert[i + 1] : expert[i];
          key[i + 1] = swap ? key[i] : key[i + 1];
          expert[i + 1] = swap ? expert[i] : expert[i + 1];
          key[i] = k;
          expert[i] = e;
        }
    } else {
      search();
    }
  }
  uint32_t best_key;
  int best_expert;
  __device__ __forceinline__ uint32_t top() const { return kSorted ? key[0] : best_key; }
  __device__ __forceinline__ int top_expert() const { return kSorted ? expert[0] : best_expert; }
  __device__ __forceinline__ void pop() {
    if (kSorted) {
#pragma unroll
      for (int i = 0; i + 1 < PER; ++i) {
        key[i] = key[i + 1];
        expert[i] = expert[i + 1];
      }
      key[PER - 1] = 0;
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (expert[i] == best_expert) key[i] = 0;
      search();
    }
  }
  __device__ __forceinline__ void search() {
    best_key = 0;
    best_expert = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (key[i] > best_key) {
        best_key = key[i];
        best_expert = expert[i];
      }
  }
};

template <int VEC, int PER, typename T>
__global__ void __launch_bounds__(256)
    sq_route_kernel(int64_t tokens, int E, int k, const T *__restrict__ logits, const uint8_t *__restrict__ valid,
                    bool normalize, int *__restrict__ experts, float *__restrict__ weights) {
  const int lane = threadIdx.x & 31;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  if (t >= tokens) return;
  const bool on = !valid || valid[t];
  int my_expert = -1;
  float my_value = 0.f, top = 0.f, total = 0.f;
  if (on) {
    float z[PER];
    load_row<VEC, PER>(logits + t * E, E, lane, z);
    LaneTop<VEC, PER> own(z, lane);
    for (int j = 0; j < k; ++j) {
      const uint32_t won = __reduce_max_sync(kAll, own.top());
      if (won == 0) break;
      if (j == 0) {
        top = key_value(won);
        if (!normalize) {
#pragma unroll
          for (int i = 0; i < PER; ++i)
            if (z[i] > -INFINITY) total += expf(fminf(z[i], FLT_MAX) - top);
          total = warp_sum(total);
        }
      }
      const uint32_t same = __ballot_sync(kAll, own.top() == won);
      int winner = __ffs(same) - 1;
      int e = __shfl_sync(kAll, own.top_expert(), winner);
      if (same & (same - 1)) {  // equal logits in several lanes: the lowest expert
        e = __reduce_min_sync(kAll, own.top() == won ? own.top_expert() : INT_MAX);
        winner = __ffs(__ballot_sync(kAll, own.top() == won && own.top_expert() == e)) - 1;
      }
      if (lane == winner) own.pop();
      if (lane == j) {
        my_expert = e;
        my_value = key_value(won);
      }
    }
  }
  float w = my_expert >= 0 ? expf(my_value - top) : 0.f;
  if (normalize) total = warp_sum(w);
  if (lane < k) {
    experts[t * k + lane] = my_expert;
    weights[t * k + lane] = my_expert >= 0 ? w / total : 0.f;
  }
}

// dz_e = q_e (dw_e - sum_j q_j dw_j), q the weights over the chosen experts (normalize) or the
// softmax over all; dw_e is 0 for an expert that was not chosen. The softmax is formed again
// from the logits: keeping it would cost a write and the same read.
template <int VEC, int PER, typename T>
__global__ void __launch_bounds__(256)
    sq_route_grad_kernel(int64_t tokens, int E, int k, const T *__restrict__ logits, const int *__restrict__ experts,
                         const float *__restrict__ dweights, bool normalize, T *__restrict__ dlogits) {
  const int lane = threadIdx.x & 31;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  if (t >= tokens) return;
  const T *row = logits + t * E;
  T *out = dlogits + t * E;
  int e = lane < k ? experts[t * k + lane] : -1;
  if (e >= E) e = -1;
  const float dw = e >= 0 ? dweights[t * k + lane] : 0.f;
  const float z = e >= 0 ? load_logit(row + e) : NAN;
  const uint32_t key = e >= 0 ? order_key(z) : 0u;
  const bool any = __any_sync(kAll, key != 0);
  float share = 0.f, inner = 0.f, top = 0.f, total = 1.f;
  float dense[PER];
  if (any) {
    if (normalize) {
      top = key_value(__reduce_max_sync(kAll, key));
      share = key ? expf(key_value(key) - top) : 0.f;
      total = warp_sum(share);
    } else {
      float zs[PER];
      load_row<VEC, PER>(row, E, lane, zs);
      uint32_t best = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) best = max(best, order_key(zs[i]));
      top = key_value(__reduce_max_sync(kAll, best));
      total = 0.f;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const uint32_t q = order_key(zs[i]);
        dense[i] = q ? expf(key_value(q) - top) : 0.f;
        total += dense[i];
      }
      total = warp_sum(total);
      share = key ? expf(key_value(key) - top) : 0.f;
    }
    share /= total;
    inner = warp_sum(share * dw);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) dense[i] = any && !normalize ? -(dense[i] / total) * inner : 0.f;
#pragma unroll
  for (int i = 0; i < PER; i += VEC) {
    const int at = expert_of<VEC>(i, lane);
    if (at >= E) continue;
    if (VEC == 4)
      store_logits4(out + at, dense + i);
    else
      store_logit(out + at, dense[i]);
  }
  __syncwarp();  // the chosen experts' values go over the row's
  if (key) store_logit(out + e, share * (dw - inner));
}

// ---------------------------------------------------------------- tokens by expert
//
// Stable counting sort of the n slots t * k + j by expert. Each warp owns a run of neighbouring
// slots and a histogram row; the prefix over warps, CTAs and experts gives each its first row, and
// rows are handed out in slot order, so the order never depends on timing. Up to kSortOne slots
// take one CTA; more take a launch that counts per CTA and one that adds up the counts and places
// the slots (each CTA reads all CTAs' counts: G x E words from the L2).

constexpr int kSortStep = 4;  // loads of 32 slots in flight
constexpr int64_t kSortOne = 4096;
constexpr int64_t kSortMany = 2048;  // slots of a CTA at least, of several
constexpr int kSortThreads = 512;    // of a CTA, of several

__device__ __forceinline__ void load_slots(const int *experts, int64_t at, int64_t end, int E, int lane,
                                           int (&e)[kSortStep]) {
#pragma unroll
  for (int s = 0; s < kSortStep; ++s) {
    const int64_t i = at + 32 * s + lane;
    e[s] = i < end ? __ldg(experts + i) : -1;
    if (e[s] >= E) e[s] = -1;
  }
}

__global__ void __launch_bounds__(kSortThreads)
    sq_sort_count_kernel(int64_t n, int E, int64_t per, const int *__restrict__ experts, int *__restrict__ counts) {
  extern __shared__ int sort_smem[];
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
    sq_sort_kernel(int64_t n, int E, int64_t per, const int *__restrict__ experts, const int *__restrict__ counts,
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
  __syncthreads();
  int *mine = hist + warp * E;
  for (int64_t at = begin; at < end; at += 32 * kSortStep) {
    int e[kSortStep];
    load_slots(experts, at, end, E, lane, e);
#pragma unroll
    for (int s = 0; s < kSortStep; ++s)
      if (e[s] >= 0) atomicAdd(mine + e[s], 1);
  }
  if (counts) {
    const int cells = gridDim.x * E, before = blockIdx.x * E;
#pragma unroll 4
    for (int i = threadIdx.x; i < cells; i += blockDim.x) {
      const int c = counts[i];
      if (c == 0) continue;
      const int e = i % E;
      atomicAdd(all + e, c);
      if (i < before) atomicAdd(first + e, c);
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
  for (int64_t at = begin; at < end; at += 32 * kSortStep) {
    int e[kSortStep];
    load_slots(experts, at, end, E, lane, e);
#pragma unroll
    for (int s = 0; s < kSortStep; ++s) {
      const int64_t i = at + 32 * s + lane;
      const uint32_t same = __match_any_sync(kAll, e[s]);
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

__device__ __forceinline__ uint4 load_row16(const uint16_t *p) {
  return __ldg(reinterpret_cast<const uint4 *>(p));
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
    sq_dispatch_kernel(uint32_t units, uint32_t pieces, int k, int64_t D, int64_t rows, const uint16_t *__restrict__ X,
                       const int *__restrict__ row_of, const int *__restrict__ slot_of, uint16_t *__restrict__ Xs) {
  const int lane = threadIdx.x & 31;
  const uint32_t unit = blockIdx.x * 8 + (threadIdx.x >> 5);
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
    if (read && c0 + 256 * i < D) v[i] = load_row16(X + t * D + c0 + 256 * i);
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

// Y[t] = sum_j w[t, j] Ys[row_of[t, j]] in fp32 in the order of j, rounded once (without
// weights: the plain sum, the gradient of the dispatch). `share` warps per token, which take its
// 256-column pieces in turn.
constexpr int kCombineFlight = 8;  // rows in flight
__global__ void __launch_bounds__(256)
    sq_combine_kernel(int64_t tokens, int k, int64_t D, int64_t rows, int share, const uint16_t *__restrict__ Ys,
                      const int *__restrict__ row_of, const float *__restrict__ weights, uint16_t *__restrict__ Y) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (8 / share) + warp / share;
  if (t >= tokens) return;
  int64_t row = -1;
  float w = 1.f;
  if (lane < k) {
    row = row_of[t * k + lane];
    if (row >= rows) row = -1;
    if (weights) w = weights[t * k + lane];
  }
  int64_t at[kCombineFlight];
  float wj[kCombineFlight];
  auto batch = [&](int j0) {
#pragma unroll
    for (int i = 0; i < kCombineFlight; ++i) {
      at[i] = __shfl_sync(kAll, row, j0 + i);
      wj[i] = __shfl_sync(kAll, w, j0 + i);
      if (j0 + i >= k) at[i] = -1;
    }
  };
  batch(0);
  for (int64_t c0 = (warp % share) * 256; c0 < D; c0 += share * 256) {
    const int64_t c = c0 + lane * 8;
    float sum[8] = {};
    for (int j0 = 0; j0 < k; j0 += kCombineFlight) {
      if (k > kCombineFlight) batch(j0);
      uint4 v[kCombineFlight];
#pragma unroll
      for (int i = 0; i < kCombineFlight; ++i)
        if (at[i] >= 0 && c < D) v[i] = load_row16(Ys + at[i] * D + c);
#pragma unroll
      for (int i = 0; i < kCombineFlight; ++i) {
        if (at[i] < 0) continue;
        float x[8];
        unpack8(v[i], x);
#pragma unroll
        for (int q = 0; q < 8; ++q) sum[q] = fmaf(wj[i], x[q], sum[q]);
      }
    }
    if (c < D) store_row16(Y + t * D + c, pack8(sum));
  }
}

// dYs[row_of[t, j]] = w[t, j] dY[t] and dw[t, j] = sum_d dY[t, d] Ys[row_of[t, j], d]. One token
// per `share` warps of the CTA, which take its 256-column pieces in turn.
constexpr int kGradFlight = 8;
__global__ void __launch_bounds__(256)
    sq_combine_grad_kernel(int64_t tokens, int k, int64_t D, int64_t rows, int share, const uint16_t *__restrict__ dY,
                           const uint16_t *__restrict__ Ys, const int *__restrict__ row_of,
                           const int *__restrict__ slot_of, const float *__restrict__ weights,
                           uint16_t *__restrict__ dYs, float *__restrict__ dweights) {
  __shared__ float partial[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int part = warp % share;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (8 / share) + warp / share;
  float dw = 0.f;  // lane j: this warp's part of dw[t, j]
  if (t < tokens) {
    const int64_t slot = t * k + lane;
    int64_t row = -1;
    float w = 0.f;
    bool empty = false;
    if (lane < k) {
      row = row_of[slot];
      if (row >= rows) row = -1;
      w = weights[slot];
      empty = slot < rows && slot_of[slot] < 0;
    }
    const uint32_t clear = __ballot_sync(kAll, empty);
    for (int j0 = 0; j0 < k; j0 += kGradFlight) {
      int64_t at[kGradFlight];
      float wj[kGradFlight], acc[kGradFlight];
#pragma unroll
      for (int i = 0; i < kGradFlight; ++i) {
        at[i] = __shfl_sync(kAll, row, j0 + i);
        wj[i] = __shfl_sync(kAll, w, j0 + i);
        if (j0 + i >= k) at[i] = -1;
        acc[i] = 0.f;
      }
      for (int64_t c = part * 256 + lane * 8; c < D; c += share * 256) {
        float g[8];
        uint4 v[kGradFlight];
#pragma unroll
        for (int i = 0; i < kGradFlight; ++i)
          if (at[i] >= 0) v[i] = load_row16(Ys + at[i] * D + c);
        unpack8(load_row16(dY + t * D + c), g);
#pragma unroll
        for (int i = 0; i < kGradFlight; ++i) {
          if (at[i] < 0) continue;
          float x[8], o[8];
          unpack8(v[i], x);
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            acc[i] = fmaf(g[q], x[q], acc[i]);
            o[q] = wj[i] * g[q];
          }
          store_row16(dYs + at[i] * D + c, pack8(o));
        }
      }
#pragma unroll
      for (int i = 0; i < kGradFlight; ++i) {
        const float s = warp_sum(acc[i]);
        if (lane == j0 + i) dw = s;
      }
    }
    for (uint32_t m = clear; m; m &= m - 1) {
      const int64_t to = t * k + __ffs(m) - 1;
      for (int64_t c = part * 256 + lane * 8; c < D; c += share * 256)
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

template <typename T, typename F>
void with_row_shape(int E, F f) {
  auto per = [&](auto vec) {
    constexpr int V = decltype(vec)::value;
    if (E <= 32 * V)
      f(vec, std::integral_constant<int, V>{});
    else if (E <= 128)
      f(vec, std::integral_constant<int, 4>{});
    else if (E <= 256)
      f(vec, std::integral_constant<int, 8>{});
    else if (E <= 512)
      f(vec, std::integral_constant<int, 16>{});
    else
      f(vec, std::integral_constant<int, 32>{});
  };
  if (E % 4 == 0)
    per(std::integral_constant<int, 4>{});
  else
    per(std::integral_constant<int, 1>{});
}

}  // namespace

cudaError_t launch_route(int64_t T, int E, int k, bool bf16, const void *logits, const uint8_t *valid, bool normalize,
                         int *experts, float *weights, cudaStream_t stream) {
  const unsigned grid = static_cast<unsigned>((T + 7) / 8);
  auto go = [&](auto *z) {
    using L = std::remove_const_t<std::remove_pointer_t<decltype(z)>>;
    with_row_shape<L>(E, [&](auto vec, auto per) {
      sq_route_kernel<decltype(vec)::value, decltype(per)::value, L>
          <<<grid, 256, 0, stream>>>(T, E, k, z, valid, normalize, experts, weights);
    });
  };
  if (bf16)
    go(static_cast<const __nv_bfloat16 *>(logits));
  else
    go(static_cast<const float *>(logits));
  return cudaGetLastError();
}

cudaError_t launch_route_grad(int64_t T, int E, int k, bool bf16, const void *logits, const int *experts,
                              const float *dweights, bool normalize, void *dlogits, cudaStream_t stream) {
  const unsigned grid = static_cast<unsigned>((T + 7) / 8);
  auto go = [&](auto *z) {
    using L = std::remove_const_t<std::remove_pointer_t<decltype(z)>>;
    with_row_shape<L>(E, [&](auto vec, auto per) {
      sq_route_grad_kernel<decltype(vec)::value, decltype(per)::value, L>
          <<<grid, 256, 0, stream>>>(T, E, k, z, experts, dweights, normalize, static_cast<L *>(dlogits));
    });
  };
  if (bf16)
    go(static_cast<const __nv_bfloat16 *>(logits));
  else
    go(static_cast<const float *>(logits));
  return cudaGetLastError();
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
    sq_sort_count_kernel<<<ctas, kSortThreads, E * sizeof(int), stream>>>(n, E, per, experts, workspace);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  const size_t smem = (static_cast<size_t>(threads / 32) + 2) * E * sizeof(int);
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(sq_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               34 * kRouteMaxExperts * static_cast<int>(sizeof(int)));
    if (e != cudaSuccess) return e;
  }
  sq_sort_kernel<<<ctas, threads, smem, stream>>>(n, E, per, experts, one ? nullptr : workspace, offsets, row_of,
                                                  slot_of);
  return cudaGetLastError();
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
  sq_dispatch_kernel<<<(units + 7) / 8, 256, 0, stream>>>(units, pieces, k, D, rows, X, row_of, slot_of, Xs);
  return cudaGetLastError();
}

cudaError_t launch_combine(int64_t T, int k, int64_t D, int64_t rows, const uint16_t *Ys, const int *row_of,
                           const float *weights, uint16_t *Y, int sm_count, cudaStream_t stream) {
  const int share = warps_of_token(T, D, 32 * static_cast<int64_t>(sm_count));
  const int64_t per = 8 / share;
  sq_combine_kernel<<<static_cast<unsigned>((T + per - 1) / per), 256, 0, stream>>>(T, k, D, rows, share, Ys, row_of,
                                                                                   weights, Y);
  return cudaGetLastError();
}

cudaError_t launch_combine_grad(int64_t T, int k, int64_t D, int64_t rows, const uint16_t *dY, const uint16_t *Ys,
                                const int *row_of, const int *slot_of, const float *weights, uint16_t *dYs,
                                float *dweights, int sm_count, cudaStream_t stream) {
  const int share = warps_of_token(T, D, 16 * static_cast<int64_t>(sm_count));
  const int64_t per = 8 / share;
  sq_combine_grad_kernel<<<static_cast<unsigned>((T + per - 1) / per), 256, 0, stream>>>(
      T, k, D, rows, share, dY, Ys, row_of, slot_of, weights, dYs, dweights);
  return cudaGetLastError();
}

}  // namespace sqi
