// Token routing around the grouped expert linears: top-k of the router's logits with its
// gradient, the tokens sorted by expert, and the rows that travel to the experts and back.
#include <cuda_bf16.h>
#include <float.h>

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
    uint32_t key[PER], best = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      key[i] = order_key(z[i]);
      best = max(best, key[i]);
    }
    for (int j = 0; j < k; ++j) {
      const uint32_t won = __reduce_max_sync(kAll, best);
      if (won == 0) break;
      if (j == 0) {
        top = key_value(won);
        if (!normalize) {
#pragma unroll
          for (int i = 0; i < PER; ++i)
            if (key[i]) total += expf(key_value(key[i]) - top);
          total = warp_sum(total);
        }
      }
      uint32_t mine = 0xFFFFFFFFu;  // the lowest expert of this lane with the winning logit
      if (best == won) {
#pragma unroll
        for (int i = PER - 1; i >= 0; --i)
          if (key[i] == won) mine = expert_of<VEC>(i, lane);
      }
      const uint32_t e = __reduce_min_sync(kAll, mine);
      if (mine == e) {
        best = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          if (expert_of<VEC>(i, lane) == static_cast<int>(e)) key[i] = 0;
          best = max(best, key[i]);
        }
      }
      if (lane == j) {
        my_expert = static_cast<int>(e);
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
  for (int i = 0; i < PER; ++i) {
    const int at = expert_of<VEC>(i, lane);
    if (at < E) store_logit(out + at, dense[i]);
  }
  __syncwarp();  // the chosen experts' values go over the row's
  if (key) store_logit(out + e, share * (dw - inner));
}

// ---------------------------------------------------------------- tokens by expert
//
// Stable counting sort of the n slots t * k + j by expert. One cluster of CTAs: each warp owns a
// run of neighbouring slots and a histogram row, the prefix over warps, CTAs (through
// distributed shared memory) and experts gives each its first row, and a second pass hands the
// rows out in slot order, so the order never depends on timing.

constexpr int kSortStep = 8;  // loads of 32 slots in flight

__device__ __forceinline__ uint32_t sort_cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t sort_cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void sort_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int remote_int(const int *p, uint32_t rank) {
  uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(p)), r;
  int v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(r) : "memory");
  return v;
}

__global__ void __launch_bounds__(1024)
    sq_sort_kernel(int64_t n, int E, const int *__restrict__ experts, int64_t *__restrict__ offsets,
                   int *__restrict__ row_of, int *__restrict__ slot_of) {
  extern __shared__ int sort_smem[];
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int *hist = sort_smem;             // [warps][E]
  int *counts = hist + warps * E;    // [E] slots of this CTA
  int *first = counts + E;           // [E] first row of this CTA's slots of an expert
  __shared__ int scan[32];
  __shared__ int routed;
  const uint32_t rank = sort_cluster_rank(), ctas = sort_cluster_size();
  const int64_t per_warp = ((n + ctas * warps - 1) / (ctas * warps) + 31) / 32 * 32;
  const int64_t begin = min(n, (static_cast<int64_t>(rank) * warps + warp) * per_warp);
  const int64_t end = min(n, begin + per_warp);
  for (int i = threadIdx.x; i < warps * E; i += blockDim.x) hist[i] = 0;
  __syncthreads();
  int *mine = hist + warp * E;
  auto load = [&](int64_t at, int (&e)[kSortStep]) {
#pragma unroll
    for (int s = 0; s < kSortStep; ++s) {
      const int64_t i = at + 32 * s + lane;
      e[s] = i < end ? __ldg(experts + i) : -1;
      if (e[s] >= E) e[s] = -1;
    }
  };
  for (int64_t at = begin; at < end; at += 32 * kSortStep) {
    int e[kSortStep];
    load(at, e);
#pragma unroll
    for (int s = 0; s < kSortStep; ++s)
      if (e[s] >= 0) atomicAdd(mine + e[s], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += blockDim.x) {
    int sum = 0;
    for (int w = 0; w < warps; ++w) {
      const int c = hist[w * E + e];
      hist[w * E + e] = sum;
      sum += c;
    }
    counts[e] = sum;
  }
  sort_cluster_sync();
  // rows of all CTAs per expert, scanned over the experts a block width at a time
  int carry = 0;
  for (int e0 = 0; e0 < E; e0 += blockDim.x) {
    const int e = e0 + threadIdx.x;
    int before = 0, all = 0;
    if (e < E)
      for (uint32_t r = 0; r < ctas; ++r) {
        const int c = remote_int(counts + e, r);
        before += r < rank ? c : 0;
        all += c;
      }
    int incl = all;
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
    const int start = carry + incl - all + (warp > 0 ? scan[warp - 1] : 0);
    carry += scan[31];
    if (e < E) {
      first[e] = start + before;
      if (rank == 0) offsets[e] = start;
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    routed = carry;
    if (rank == 0) offsets[E] = carry;
  }
  sort_cluster_sync();  // every CTA has read the others' counts; first and routed are visible
  for (int64_t at = begin; at < end; at += 32 * kSortStep) {
    int e[kSortStep];
    load(at, e);
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
  for (int64_t r = routed + static_cast<int64_t>(rank) * blockDim.x + threadIdx.x; r < n;
       r += static_cast<int64_t>(ctas) * blockDim.x)
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
// weights: the plain sum, the gradient of the dispatch). A warp takes 256 columns of one token.
constexpr int kCombineFlight = 8;  // rows in flight
__global__ void __launch_bounds__(256)
    sq_combine_kernel(uint32_t units, uint32_t pieces, int k, int64_t D, int64_t rows, const uint16_t *__restrict__ Ys,
                      const int *__restrict__ row_of, const float *__restrict__ weights, uint16_t *__restrict__ Y) {
  const int lane = threadIdx.x & 31;
  const uint32_t unit = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (unit >= units) return;
  const int64_t t = unit / pieces;
  const int64_t c = static_cast<int64_t>(unit % pieces) * 256 + lane * 8;
  int64_t row = -1;
  float w = 1.f;
  if (lane < k) {
    row = row_of[t * k + lane];
    if (row >= rows) row = -1;
    if (weights) w = weights[t * k + lane];
  }
  float sum[8] = {};
  for (int j0 = 0; j0 < k; j0 += kCombineFlight) {
    uint4 v[kCombineFlight];
    int64_t from[kCombineFlight];
#pragma unroll
    for (int i = 0; i < kCombineFlight; ++i) {
      from[i] = __shfl_sync(kAll, row, j0 + i);
      if (j0 + i >= k || c >= D) from[i] = -1;
      if (from[i] >= 0) v[i] = load_row16(Ys + from[i] * D + c);
    }
#pragma unroll
    for (int i = 0; i < kCombineFlight; ++i) {
      const float wi = __shfl_sync(kAll, w, j0 + i);
      if (from[i] < 0) continue;
      float x[8];
      unpack8(v[i], x);
#pragma unroll
      for (int q = 0; q < 8; ++q) sum[q] = fmaf(wi, x[q], sum[q]);
    }
  }
  if (c < D) store_row16(Y + t * D + c, pack8(sum));
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

cudaError_t launch_sort(int64_t n, int E, const int *experts, int64_t *offsets, int *row_of, int *slot_of,
                        cudaStream_t stream) {
  // few slots: one CTA of eight warps, whose prefix over the warps is short
  const int ctas = n <= 8192 ? 1 : 8, threads = n <= 2048 ? 256 : 1024;
  const size_t smem = (static_cast<size_t>(threads / 32) + 2) * E * sizeof(int);
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(sq_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               34 * kRouteMaxExperts * static_cast<int>(sizeof(int)));
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas, 1, 1);
  cfg.blockDim = dim3(threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, sq_sort_kernel, n, E, experts, offsets, row_of, slot_of);
}

cudaError_t launch_dispatch(int64_t T, int k, int64_t D, int64_t rows, const uint16_t *X, const int *row_of,
                            const int *slot_of, uint16_t *Xs, cudaStream_t stream) {
  const uint32_t pieces = static_cast<uint32_t>((D + kMoveCols - 1) / kMoveCols);
  const uint32_t units = static_cast<uint32_t>(T) * pieces;
  sq_dispatch_kernel<<<(units + 7) / 8, 256, 0, stream>>>(units, pieces, k, D, rows, X, row_of, slot_of, Xs);
  return cudaGetLastError();
}

cudaError_t launch_combine(int64_t T, int k, int64_t D, int64_t rows, const uint16_t *Ys, const int *row_of,
                           const float *weights, uint16_t *Y, cudaStream_t stream) {
  const uint32_t pieces = static_cast<uint32_t>((D + 255) / 256), units = static_cast<uint32_t>(T) * pieces;
  sq_combine_kernel<<<(units + 7) / 8, 256, 0, stream>>>(units, pieces, k, D, rows, Ys, row_of, weights, Y);
  return cudaGetLastError();
}

cudaError_t launch_combine_grad(int64_t T, int k, int64_t D, int64_t rows, const uint16_t *dY, const uint16_t *Ys,
                                const int *row_of, const int *slot_of, const float *weights, uint16_t *dYs,
                                float *dweights, int sm_count, cudaStream_t stream) {
  // warps of a token: as many as keep the SMs busy, at most one per 256 columns
  int share = 1;
  while (share < 8 && T * share < 16 * static_cast<int64_t>(sm_count) && share * 256 < D) share *= 2;
  const int64_t per = 8 / share;
  sq_combine_grad_kernel<<<static_cast<unsigned>((T + per - 1) / per), 256, 0, stream>>>(
      T, k, D, rows, share, dY, Ys, row_of, slot_of, weights, dYs, dweights);
  return cudaGetLastError();
}

}  // namespace sqi
