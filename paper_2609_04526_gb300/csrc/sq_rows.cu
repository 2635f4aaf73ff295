// Rows of activations to microscaled FP4 and back (sm_103a):
//
//   NVFP4  u = x / row,  s_b = max(2^-9, E4M3(max_b |u| / 6)),  code = E2M1(u / s_b)
//   MXFP4  s_b = 2^(floor(log2 max_b |x|) - 2),                 code = E2M1(x / s_b)
//
// over blocks b of 16 or 32 values, every rounding to nearest, ties to even, and saturating at 448
// and 6. `row` is a scale given for all rows (then u = fl32(x * fl32(1 / row))) or each row's own
// power of two: the smallest 2^e >= 2^-116 with max |x| <= 6 * 448 * 2^e, so x / row is exact, nothing
// saturates, and a decoded value is a normal bf16. Of a row's own scale the E4M3 scales carry what is
// not a power of two.
//
// The decisions are exact. u / s_b is the product with a reciprocal and one correction by the exact
// remainder (Markstein's method). On a border m between two codes u is m s_b exactly, the remainder
// brings the quotient to m exactly, and the tie goes to the even code. Off it, u and m s_b are
// different numbers of 24 bits, and a quotient of two such numbers never rounds to m: their relative
// distance is at least 2^-23 / Mu, Mu < 2 the significand of u, against half a step of 2^-24 / Mm
// around m. The same holds for max / 6 and the borders of E4M3.
//
// Bound by memory (2 + 9/16 bytes a value, either way): 32768 x 4096 NVFP4 quantised in 57 us, 6.0 TB/s, back
// in 50 us, 6.9 TB/s. A thread takes 16 values, 32 bytes of the row.
#include <type_traits>

#include "sq_gemm_kernels.cuh"
#include "sq_launch.cuh"

namespace sqi {
namespace {

constexpr int kRowsThreads = 256;
constexpr int kRowsHold = 4;  // chunks of 16 values that a thread keeps in registers

// The 16 values of a chunk as bf16 pairs: one 32-byte load where the row starts on 32 bytes.
__device__ __forceinline__ void load_chunk(const uint16_t *p, bool wide, uint32_t (&v)[8]) {
  if (wide) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "l"(p));
  } else {
    const uint4 a = reinterpret_cast<const uint4 *>(p)[0], b = reinterpret_cast<const uint4 *>(p)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
}

// The largest magnitude of a chunk as bf16 bits; infinities and NaN are above every finite value.
__device__ __forceinline__ uint32_t chunk_max(const uint32_t (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = __vmaxu2(m, v[i] & 0x7FFF7FFFu);
  return max(m & 0xFFFFu, m >> 16);
}

__device__ __forceinline__ float bf16_bits_float(uint32_t bits) { return __uint_as_float(bits << 16); }

__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Two quotients x / s from -x, with neg_r = -fl32(1 / s), their remainders carried out. (From x a
// zero would lose its sign.)
__device__ __forceinline__ uint64_t quotients(uint64_t neg_x, uint64_t s, uint64_t neg_r) {
  const uint64_t q = mul_f32x2(neg_x, neg_r);
  return fma_f32x2(fma_f32x2(q, s, neg_x), neg_r, q);
}
__device__ __forceinline__ uint64_t both(float x) { return pack_f32x2(__float_as_uint(x), __float_as_uint(x)); }

// Eight values (four pairs, the earlier value in the low half) to a word of E2M1 codes.
__device__ __forceinline__ uint32_t e2m1x8_rn(const uint64_t (&q)[4]) {
  uint32_t w;
  asm("{\n\t.reg .b8 c0, c1, c2, c3;\n\t.reg .f32 l0, h0, l1, h1, l2, h2, l3, h3;\n\t"
      "mov.b64 {l0, h0}, %1;\n\tmov.b64 {l1, h1}, %2;\n\tmov.b64 {l2, h2}, %3;\n\tmov.b64 {l3, h3}, %4;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c0, h0, l0;\n\tcvt.rn.satfinite.e2m1x2.f32 c1, h1, l1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c2, h2, l2;\n\tcvt.rn.satfinite.e2m1x2.f32 c3, h3, l3;\n\t"
      "mov.b32 %0, {c0, c1, c2, c3};\n\t}"
      : "=r"(w)
      : "l"(q[0]), "l"(q[1]), "l"(q[2]), "l"(q[3]));
  return w;
}

// Exponent of a row's own scale: 2688 = 1.3125 * 2^11 is 6 * 448, and 1.3125 has the bf16
// significand 0x28. `bits` is the largest finite magnitude.
__device__ __forceinline__ int row_exponent(uint32_t bits) {
  const int e = static_cast<int>(bits >> 7) - 127 - 11 + ((bits & 0x7Fu) > 0x28u ? 1 : 0);
  return max(e, -116);  // subnormal magnitudes end here too
}

// One chunk to codes and a scale byte. row: exponent of the row's own scale (OWN); fixed_inv:
// fl32(1 / the scale of all rows). `top` is the block's largest magnitude.
template <int FMT, bool OWN>
__device__ __forceinline__ uint32_t encode_chunk(const uint32_t (&v)[8], uint32_t top, int row, float fixed_inv,
                                                 uint2 &codes) {
  uint32_t byte;
  uint64_t q[8];
  if (FMT == 1) {
    byte = max(static_cast<int>(top >> 7) - 2, 0);
    const uint64_t r = both(__uint_as_float((254u - byte) << 23));
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = mul_f32x2(pack_f32x2(v[i] << 16, v[i] & 0xFFFF0000u), r);
    if (top >= 0x7F80u) byte = 0xFF;
  } else {
    const float inv = OWN ? __uint_as_float(static_cast<uint32_t>(127 - row) << 23) : fixed_inv;
    // far above what a fixed scale reaches, where the remainders would overflow
    constexpr float kFar = 0x1p20f;
    const float u = fminf(bf16_bits_float(top) * inv, kFar);
    constexpr float kSixth = 1.f / 6.f;
    const float t = u * kSixth;
    const float sixth = fmaf(fmaf(t, -6.f, u), kSixth, t);
    unsigned short e4m3;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(e4m3) : "f"(0.f), "f"(sixth));
    byte = max(e4m3 & 0xFFu, 1u);
    const float s = __uint_as_float(byte << 20) * 0x1p120f;
    const float rs = __frcp_rn(s);
    if (OWN) {  // x / (s * row): scaled by powers of two, nothing else is rounded
      const uint64_t sr = both(s * __uint_as_float(static_cast<uint32_t>(127 + row) << 23)), nr = both(-rs * inv);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t n = v[i] ^ 0x80008000u;
        q[i] = quotients(pack_f32x2(n << 16, n & 0xFFFF0000u), sr, nr);
      }
    } else {
      const uint64_t ss = both(s), nr = both(-rs), by = both(-fixed_inv);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint64_t n = mul_f32x2(pack_f32x2(v[i] << 16, v[i] & 0xFFFF0000u), by);
        if (u == kFar) {
          const float lo = __uint_as_float(static_cast<uint32_t>(n)), hi = __uint_as_float(static_cast<uint32_t>(n >> 32));
          n = pack_f32x2(__float_as_uint(fminf(fmaxf(lo, -kFar), kFar)), __float_as_uint(fminf(fmaxf(hi, -kFar), kFar)));
        }
        q[i] = quotients(n, ss, nr);
      }
    }
    if (top >= 0x7F80u) byte = 0x7F;
  }
  const uint64_t lo[4] = {q[0], q[1], q[2], q[3]}, hi[4] = {q[4], q[5], q[6], q[7]};
  codes = make_uint2(e2m1x8_rn(lo), e2m1x8_rn(hi));
  return byte;
}

// TPR threads per row, 256 / TPR rows per CTA. With OWN a row of at most TPR * kRowsHold chunks
// stays in registers between its maximum and its codes; a longer one is read again.
template <int FMT, bool OWN, int TPR>
__global__ void __launch_bounds__(kRowsThreads) sq_quantize_kernel(const QuantArgs a) {
  __shared__ uint32_t warp_top[kRowsThreads / 32];
  dependency_wait();
  dependency_start();
  const int t = threadIdx.x % TPR;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * (kRowsThreads / TPR) + threadIdx.x / TPR;
  const int chunks = (!OWN && r == a.R - 1 ? a.last : a.K) / 16;
  int64_t src = r < a.R ? r : -1;
  if (a.slot_of) {
    const int slot = r < a.R ? a.slot_of[r] : -1;
    src = slot >= 0 && slot < a.slots ? slot / a.k : -1;
  }
  const uint16_t *x = a.X + (src < 0 ? 0 : src) * a.K;
  uint32_t v[kRowsHold][8];
  auto load = [&](int c0) {
#pragma unroll
    for (int j = 0; j < kRowsHold; ++j) {
      const int c = c0 + j * TPR + t;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] = 0;
      if (src >= 0 && c < chunks) load_chunk(x + 16 * static_cast<int64_t>(c), a.wide, v[j]);
    }
  };
  constexpr int kSpan = TPR * kRowsHold;
  int row = 0;
  load(0);
  if (OWN) {
    uint32_t top = 0;
    for (int c0 = 0;;) {
#pragma unroll
      for (int j = 0; j < kRowsHold; ++j) {
        const uint32_t m = chunk_max(v[j]);
        if (m < 0x7F80u) top = max(top, m);  // a block with infinities or NaN has no part in the scale
      }
      if ((c0 += kSpan) >= chunks) break;
      load(c0);
    }
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    if (TPR > 32) {
      if (threadIdx.x % 32 == 0) warp_top[threadIdx.x / 32] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < TPR / 32; ++w) top = max(top, warp_top[threadIdx.x / TPR * (TPR / 32) + w]);
    }
    row = row_exponent(top);
    if (t == 0 && r < a.R) a.row_ws2[r] = __uint_as_float(static_cast<uint32_t>(127 + row) << 23);
    if (chunks > kSpan) load(0);
  }
  uint2 *codes = reinterpret_cast<uint2 *>(a.codes + r * (a.K / 2));
  uint8_t *scales = a.scales + r * (a.K / (FMT == 0 ? 16 : 32));
  for (int c0 = 0;;) {
#pragma unroll
    for (int j = 0; j < kRowsHold; ++j) {
      if (c0 + j * TPR >= chunks) break;
      const int c = c0 + j * TPR + t;
      uint32_t top = chunk_max(v[j]);
      if (FMT == 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));  // K % 32 == 0: both or neither in the row
      uint2 w;
      const uint32_t byte = encode_chunk<FMT, OWN>(v[j], top, row, a.inv, w);
      if (r < a.R && c < chunks) {
        codes[c] = w;
        if (FMT == 0)
          scales[c] = static_cast<uint8_t>(byte);
        else if ((c & 1) == 0)
          scales[c >> 1] = static_cast<uint8_t>(byte);
      }
    }
    if ((c0 += kSpan) >= chunks) break;
    load(c0);
  }
}

// Rows by slot from the 4-bit rows of the tokens, a warp each: 16384 rows of 2048 values
// NVFP4 (19 MB, from the L2) in 6 us. A row of no token is what a row of zeros gives: the smallest scales. Codes move in 16-byte pieces;
// scale bytes too, or, where a row is not whole pieces, in the units that divide it. All of a row's loads are
// in flight before its first store.
__device__ __forceinline__ void fill_bytes(uint4 &u, uint32_t word) { u = make_uint4(word, word, word, word); }
template <typename Unit>
__device__ __forceinline__ void fill_bytes(Unit &u, uint32_t word) { u = static_cast<Unit>(word); }

template <typename Unit>
__global__ void __launch_bounds__(kRowsThreads) sq_spread_kernel(const QuantArgs a, const QuantArgs tokens, const int G,
                                                                 const uint32_t least) {
  dependency_wait();
  dependency_start();
  const int lane = threadIdx.x % 32;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * (kRowsThreads / 32) + threadIdx.x / 32;
  if (r >= a.R) return;
  const int slot = a.slot_of[r];
  const bool on = slot >= 0 && slot < a.slots;
  const int64_t t = on ? slot / a.k : 0;
  const int pieces = a.K / 32, units = G / static_cast<int>(sizeof(Unit));
  const uint4 *codes = reinterpret_cast<const uint4 *>(tokens.codes + t * (a.K / 2));
  uint4 *codes_to = reinterpret_cast<uint4 *>(a.codes + r * (a.K / 2));
  const Unit *scales = reinterpret_cast<const Unit *>(tokens.scales + t * G);
  Unit *scales_to = reinterpret_cast<Unit *>(a.scales + r * G);
  if (!on) {
    for (int c = lane; c < pieces; c += 32) codes_to[c] = make_uint4(0, 0, 0, 0);
    Unit s;
    fill_bytes(s, least);
    for (int c = lane; c < units; c += 32) scales_to[c] = s;
    if (a.row_ws2 && lane == 0) a.row_ws2[r] = 0x1p-116f;
    return;
  }
  const float row = a.row_ws2 ? tokens.row_ws2[t] : 0.f;
  for (int c0 = lane; c0 < max(pieces, units); c0 += 32 * kRowsHold) {
    uint4 v[kRowsHold];
    Unit s[kRowsHold];
#pragma unroll
    for (int j = 0; j < kRowsHold; ++j) {
      const int c = c0 + 32 * j;
      if (c < pieces) v[j] = codes[c];
      if (c < units) s[j] = scales[c];
    }
#pragma unroll
    for (int j = 0; j < kRowsHold; ++j) {
      const int c = c0 + 32 * j;
      if (c < pieces) codes_to[c] = v[j];
      if (c < units) scales_to[c] = s[j];
    }
  }
  if (a.row_ws2 && lane == 0) a.row_ws2[r] = row;
}

// 16 values of a thread: code x block scale exactly in bf16, times the row's scale in fp32, rounded once.
template <int FMT, int TPR>
__global__ void __launch_bounds__(kRowsThreads) sq_dequantize_kernel(const QuantArgs a, uint16_t *X, const bool wide) {
  dependency_wait();
  dependency_start();
  const int t = threadIdx.x % TPR, chunks = a.K / 16;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * (kRowsThreads / TPR) + threadIdx.x / TPR;
  if (r >= a.R) return;
  const float row = a.row_ws2 ? a.row_ws2[r] : a.ws2;
  const uint2 *codes = reinterpret_cast<const uint2 *>(a.codes + r * (a.K / 2));
  const uint8_t *scales = a.scales + r * (a.K / (FMT == 0 ? 16 : 32));
  uint16_t *out = X + r * a.K;
  for (int c0 = t; c0 < chunks; c0 += TPR * kRowsHold) {
    uint2 w[kRowsHold];
    uint32_t b[kRowsHold];
#pragma unroll
    for (int j = 0; j < kRowsHold; ++j) {
      const int c = c0 + j * TPR;
      if (c < chunks) {
        w[j] = codes[c];
        b[j] = scales[FMT == 0 ? c : c >> 1];
      }
    }
#pragma unroll
    for (int j = 0; j < kRowsHold; ++j) {
      const int c = c0 + j * TPR;
      if (c >= chunks) break;
      const uint32_t s = scale_bf16x2<FMT>(b[j]);
      uint32_t o[8];
      uint32_t half[4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        e2m1x8_to_bf16(h ? w[j].y : w[j].x, half);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t p = bf16x2_mul(half[i], s);
          const __nv_bfloat162 y = __floats2bfloat162_rn(__uint_as_float(p << 16) * row, __uint_as_float(p & 0xFFFF0000u) * row);
          o[4 * h + i] = *reinterpret_cast<const uint32_t *>(&y);
        }
      }
      uint16_t *dst = out + 16 * static_cast<int64_t>(c);
      if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(o[0]), "r"(o[1]), "r"(o[2]),
                     "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7])
                     : "memory");
      } else {
        reinterpret_cast<uint4 *>(dst)[0] = make_uint4(o[0], o[1], o[2], o[3]);
        reinterpret_cast<uint4 *>(dst)[1] = make_uint4(o[4], o[5], o[6], o[7]);
      }
    }
  }
}

// Threads of a row. Many rows: as few as hold it in registers, each with kRowsHold chunks in flight (32768 x
// 4096 quantised with 256 threads of one chunk 105 us, with 64 of four 57; back 69, 50). Few
// rows: as many as it has chunks.
template <typename F>
cudaError_t by_width(int64_t R, int K, int sm_count, F f) {
  const int chunks = K / 16, want = R >= 8 * static_cast<int64_t>(sm_count) ? (chunks + kRowsHold - 1) / kRowsHold : chunks;
  if (want <= 32) return f(std::integral_constant<int, 32>());
  if (want <= 64) return f(std::integral_constant<int, 64>());
  if (want <= 128) return f(std::integral_constant<int, 128>());
  return f(std::integral_constant<int, 256>());
}
unsigned row_ctas(int64_t R, int tpr) { return static_cast<unsigned>((R + kRowsThreads / tpr - 1) / (kRowsThreads / tpr)); }

// Without scales of the rows' own a block knows nothing of its row. Many are cut evenly, into rows of what 64 threads
// hold (2048 x 14336 NVFP4, whose rows leave an eighth of 256 threads idle, 14.1 -> 12.8 us; 8111 x 2880 MXFP4 7.2 ->
// 6.6). Read back, which waits for memory alone, they gain nothing.
void even_rows(QuantArgs &a, int sm_count) {
  constexpr int kEven = 64 * kRowsHold * 16;
  const int64_t values = a.R * a.K;
  if (a.row_ws2 || a.slot_of || values < int64_t(4) * sm_count * kRowsThreads * kRowsHold * 16) return;
  a.R = (values + kEven - 1) / kEven;
  a.K = kEven;
  a.last = static_cast<int>(values - (a.R - 1) * kEven);
}

}  // namespace

cudaError_t launch_quantize(int fmt, const QuantArgs &rows, int sm_count, cudaStream_t stream) {
  QuantArgs a = rows;
  even_rows(a, sm_count);
  return by_width(a.R, a.K, sm_count, [&](auto tpr) {
    constexpr int kTpr = decltype(tpr)::value;
    const auto kernel = fmt == 1       ? sq_quantize_kernel<1, false, kTpr>
                        : a.row_ws2 ? sq_quantize_kernel<0, true, kTpr>
                                    : sq_quantize_kernel<0, false, kTpr>;
    return launch_after(kernel, row_ctas(a.R, kTpr), kRowsThreads, 0, stream, a);
  });
}

cudaError_t launch_spread(int fmt, const QuantArgs &a, const QuantArgs &tokens, cudaStream_t stream) {
  const int G = a.K / (fmt == 0 ? 16 : 32);
  const auto kernel = G % 16 == 0  ? sq_spread_kernel<uint4>
                      : G % 4 == 0 ? sq_spread_kernel<uint32_t>
                      : G % 2 == 0 ? sq_spread_kernel<uint16_t>
                                   : sq_spread_kernel<uint8_t>;
  return launch_after(kernel, row_ctas(a.R, 32), kRowsThreads, 0, stream, a, tokens, G, fmt == 0 ? 0x01010101u : 0u);
}

cudaError_t launch_dequantize(int fmt, const QuantArgs &a, uint16_t *X, int sm_count, cudaStream_t stream) {
  const bool wide = reinterpret_cast<uintptr_t>(X) % 32 == 0;
  return by_width(a.R, a.K, sm_count, [&](auto tpr) {
    constexpr int kTpr = decltype(tpr)::value;
    const auto kernel = fmt == 1 ? sq_dequantize_kernel<1, kTpr> : sq_dequantize_kernel<0, kTpr>;
    return launch_after(kernel, row_ctas(a.R, kTpr), kRowsThreads, 0, stream, a, X, wide);
  });
}

}  // namespace sqi
