// Internal declarations shared by the host layer (sq_api.cu) and the kernel
// translation units of libscaleqlora. Not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

namespace sqi {

enum GemmMode : int {
  MODE_FWD = 0,    // Y  = X  . W^T   (GEMM M=tokens, N=out, contraction=in)
  MODE_DX = 1,     // dX = dY . W     (GEMM M=tokens, N=in,  contraction=out)
  MODE_SGRAD = 2   // g  = blockreduce(code * dY^T X)  (GEMM M=out, N=in, contraction=tokens)
};

// Rows of one activation TMA box of the pair kernels (the rows a CTA holds of a tile half).
constexpr int kBM = 128;
// Tokens per shared-memory stage of the scale-gradient kernel (also the height of its TMA boxes).
constexpr int kSgradBK = 128;

struct GemmArgs {
  int mode;
  int fmt;               // 0 NVFP4, 1 MXFP4
  int64_t M, N, K;       // tokens, out features, in features
  const uint8_t *codes;  // [N, K/2]
  const uint8_t *scales; // [N, K/B]
  float ws2;
  void *out;             // Y [M,N] bf16 | dX [M,K] bf16 | g [N,K/B] f32
  const uint8_t *mask;   // [N, K/B] or null (MODE_SGRAD only)
  int *err;              // device error word
  int splits = 1;            // MODE_SGRAD: token splits (sgrad_splits)
  float *partial = nullptr;  // MODE_SGRAD with splits > 1: [splits, N, K/B] fp32 partial sums
};

// Expert table of a grouped launch, built by the host for each call and copied
// to the device ahead of the kernel (64-byte aligned):
//   GroupMaps[E]         two TMA descriptors per expert, each addressing only that
//                        expert's token rows: FWD / DX the streamed activations and
//                        the output; SGRAD dY and X
//   int32 tile_start[E+1] first tile of each expert in the launch's tile list
//   int32 rows[E]        the expert's token count M_e
//   float ws2[E]         the expert's tensor scale (1.0 for MXFP4)
//   int32 id[E]          the expert of each entry: the scale gradient lists the experts
//                        longest first (its units last M_e tokens; dealt round-robin to
//                        the clusters, equal-length units then share a round), the
//                        forward and input gradient in order (their tiles are all K long)
struct GroupMaps {
  CUtensorMap m[2];
};
static_assert(sizeof(GroupMaps) == 256, "two 128-byte tensor maps per expert");
__host__ __device__ constexpr size_t group_off_tiles(int E) { return static_cast<size_t>(E) * sizeof(GroupMaps); }
__host__ __device__ constexpr size_t group_off_rows(int E) { return group_off_tiles(E) + static_cast<size_t>(E + 1) * 4; }
__host__ __device__ constexpr size_t group_off_ws2(int E) { return group_off_rows(E) + static_cast<size_t>(E) * 4; }
__host__ __device__ constexpr size_t group_off_ids(int E) { return group_off_ws2(E) + static_cast<size_t>(E) * 4; }
__host__ __device__ constexpr size_t group_table_bytes(int E) { return group_off_ids(E) + static_cast<size_t>(E) * 4; }

// Output rows of one FWD / DX tile and tokens of one scale-gradient stage: the
// host sizes the grouped tile list with these.
constexpr int kPairMTile = 512;
constexpr int kPairNTile = 256;
constexpr int kSgradTile = 256;

// Token splits of a dense scale-gradient launch. Each 256 x 256 tile contracts over
// all M tokens, so a launch with few tiles (q/k/v/o of the layer: 256 or 64) leaves
// much of its last wave idle, and a launch with many tiles streams every dY and X
// panel past the L2 once per wave of tiles that reads it. The tokens are then cut
// into up to kMaxSgradSplits parts of at least kMinSplitTokens each, one unit per
// (part, tile), walked part by part; every part writes a partial gradient plane and
// a second kernel adds the parts in order. A shorter part keeps the panels its
// waves share resident in L2 (measured on the 8B layer's shapes at M = 32768: 8
// parts read 1.3-2.0x the algorithmic bytes from DRAM against 2.2-3.5x for 5 parts
// or none), and each extra part adds ~0.2 % to the launch (the part sum's reads).
// Rule: with w(s) = ceil(tiles * s / clusters) / s, the launch's length in
// full-M tiles per cluster, take the largest s whose w(s) is within 1 % of the
// smallest w and no longer than the unsplit launch.
constexpr int kMaxSgradSplits = 8;
constexpr int64_t kMinSplitTokens = 2048;
inline int sgrad_splits(int64_t tiles, int clusters, int64_t M) {
  if (tiles <= 0 || clusters <= 0) return 1;
  auto waves = [&](int s) { return static_cast<double>((tiles * s + clusters - 1) / clusters) / s; };
  int top = 1;
  while (top < kMaxSgradSplits && M >= (top + 1) * kMinSplitTokens) ++top;
  double best = waves(1);
  for (int s = 2; s <= top; ++s) best = waves(s) < best ? waves(s) : best;
  const double limit = best * 1.01 < waves(1) ? best * 1.01 : waves(1);
  for (int s = top; s > 1; --s)
    if (waves(s) <= limit + 1e-9) return s;
  return 1;
}

// Forward / input gradient over few tokens (sq_few.cu): tiles of kFewFeatures output
// features x up to kFewTokens tokens. A grouped call lists its token tiles in device
// memory (an expert's rows cut into equal tiles); a CTA takes a token tile and a feature
// tile.
constexpr int kFewFeatures = 128;
constexpr int kFewTokens = 256;        // of a tile, where every CTA has an SM alone
constexpr int kFewTokensShared = 192;  // ... where two CTAs share an SM
constexpr int kFewBoxRows = 32;        // tokens of the smallest TMA box
constexpr int kFewSmemBytes = 111 * 1024;  // of a CTA: two share an SM
constexpr int kFewSmemAlone = 224 * 1024;  // ... where the launch has at most one CTA per SM
constexpr int kFewSlotBytes = 128 * 64;    // packed codes of 128 x 128 weights
constexpr int kFewMaxStages = 4, kFewMaxSlots = 12;
constexpr int kFewGroups = 2;        // sets of decode warps, which take the stages in turn
constexpr int kFewGroupsNarrow = 4;  // ... of tiles of kFewNarrow features
constexpr int kFewNarrow = 64;       // features of a tile where twice the tiles still have an SM each
constexpr int kFewTokensNarrow = 96; // ... and few enough tokens for four stages

// Tokens of the equal tiles (whole MMA steps of 16) that `rows` tokens are cut into.
inline int few_tile_tokens(int64_t rows, int limit) {
  const int64_t tiles = (rows + limit - 1) / limit;
  return static_cast<int>(((rows + tiles - 1) / tiles + 15) / 16 * 16);
}
// Token rows of a stage's activations: whole boxes.
inline int few_box_rows(int tile_tokens) {
  return (tile_tokens + kFewBoxRows - 1) / kFewBoxRows * kFewBoxRows;
}

// Shared memory of a CTA: `stages` stages of `depth` contraction indices (decoded weights
// and activations) and `slots` code slots, so the codes run ahead of the MMAs by the slots
// less the stages' share of them. The epilogue's bf16 tile reuses the stages.
//
// A code slot holds 128 / depth stages, and a set of decode warps waits by parity for the
// slot of its next stage. That wait can only be told from one for an earlier use of the slot
// if the use before is known to have landed: because the same set read it (a slot's uses lie
// slots * 128 / depth stages apart), or because its MMAs are done (a set that starts on stage
// i has seen those of stage i - sets - stages). A slot count that gives neither is reduced.
// (Four stages, three slots and four sets for up to 32 tokens gave neither.)
struct FewRing {
  int depth, stage_bytes, stages, slots;
  int bytes;  // with 1 KiB for the alignment
};
inline FewRing few_ring(int tile_tokens, bool alone, int features = kFewFeatures) {
  FewRing r;
  const int rows = few_box_rows(tile_tokens);
  const int room = (alone ? kFewSmemAlone : kFewSmemBytes) - 1024;
  r.depth = alone ? 128 : 64;
  r.stage_bytes = (features + rows) * r.depth * 2;
  if (features == kFewNarrow)
    r.stages = 4;
  else if (alone)
    r.stages = rows <= 96 ? 3 : 2;
  else
    r.stages = rows <= 64 ? 3 : 2;
  r.slots = (room - r.stages * r.stage_bytes) / kFewSlotBytes;
  if (r.slots > kFewMaxSlots) r.slots = kFewMaxSlots;
  const int sets = features == kFewNarrow ? kFewGroupsNarrow : kFewGroups, per = 128 / r.depth;
  while (r.slots * per % sets != 0 && r.slots * per < sets + r.stages) --r.slots;
  r.bytes = r.stages * r.stage_bytes + r.slots * kFewSlotBytes + 1024;
  return r;
}

struct FewTile {
  int expert, row0, rows;
  float ws2;
};
// Features of a tile. A CTA that decodes half as many weights per stage, in four sets of
// warps with a stage each, takes 0.43 us for one where 128 features take 0.56, so tiles of 64
// where twice as many still have an SM of their own (4096 x 4096 at 187 tokens 22.6 -> 18.5
// us); with more tokens than four stages have room for they were no faster.
inline int few_features(int64_t token_tiles, int tile_tokens, int64_t features, int sm_count) {
  return tile_tokens <= kFewTokensNarrow && token_tiles * ((features + kFewNarrow - 1) / kFewNarrow) <= sm_count
             ? kFewNarrow
             : kFewFeatures;
}
struct FewArgs {
  int mode, fmt;
  int64_t M, N, K;
  const uint8_t *scales;
  float ws2;
  uint16_t *out;
  int *err;
  const FewTile *tiles;  // device list of a grouped call, or null: tiles of tile_tokens over M
  int tile_tokens;       // tokens of the largest tile (<= kFewTokens)
  int features;          // output features of a tile (few_features)
  int64_t units;
};
// Which kernel runs a forward or input gradient, by estimates of both in microseconds that
// were fitted to measured launches (weights of 4096 x 4096, 1024 x 4096, 14336 x 4096, 768 x
// 2048 and 256 x 512 at 16 to 4096 tokens; 128 experts of 768 x 2048 and 2880 x 2880 with 2 to
// 1024 rows each). Over 346 launches of these and a few more shapes that ran on both kernels,
// the estimates above 15 us lie within 30 % of the times (half of them within 10 %), and the
// choice was the faster kernel or at most 7 % slower than it. Both sides of the line, few-token
// against pair kernel, in us: 4096 x 4096 19 against 43 at 16 to 192 tokens, 31 against 45 at
// 1024, 78 against 45 at 2048; 1024 x 4096 25 against 44 at 2048; 768 x 2048 experts 77 against
// 127 with 64 rows each, 139 against 148 with 256, 223 against 198 with 512; 2880 x 2880
// experts 271 against 566 with 16 rows each, 345 against 520 with 128, 581 against 567 with 256.
//
// few_us, for token tiles of `tokens` tokens on average and `largest` at most (0: all alike): a
// CTA alone on its SM takes 0.56 us per 128-deep stage (of 64 features 0.43), more above 128
// tokens (two stages in flight), and the launch lasts as long as its largest tile; CTAs that
// share an SM 0.27 us and up with the tokens per 64-deep stage, and 1.5 us to start and drain.
inline double few_us(int64_t token_tiles, double tokens, int64_t features, int64_t contraction, int sm_count,
                     int largest = 0) {
  const int64_t ctas = token_tiles * ((features + kFewFeatures - 1) / kFewFeatures);
  const double most = largest > 0 ? largest : tokens;
  if (most <= kFewTokensNarrow && token_tiles * ((features + kFewNarrow - 1) / kFewNarrow) <= sm_count)
    return 4.8 + ((contraction + 127) / 128) * 0.43;
  if (ctas <= sm_count)
    return 4.8 + ((contraction + 127) / 128) * (0.56 + (most > 128 ? 0.0015 * (most - 128) : 0.0));
  const double per_sm = ctas > 4 * sm_count ? static_cast<double>(ctas) / sm_count
                                            : static_cast<double>((ctas + sm_count - 1) / sm_count);
  return 4.8 + per_sm * (((contraction + 63) / 64) * (0.27 + 0.0006 * tokens) + 1.5);
}
// A wave of 512 x 256 pair tiles lasts 1.08 us per 128-deep k-step and 4 us at its end.
inline double pair_us(int64_t tiles, int64_t contraction, int sm_count) {
  const int64_t clusters = sm_count / 2, waves = (tiles + clusters - 1) / clusters;
  return 9.5 + waves * (1.08 * ((contraction + 127) / 128)) + 4.0 * (waves - 1);
}
// The limit of a token tile (few_tile_tokens) of the few-token launch over `rows` tokens in
// all, or 0 where the pair kernel's `pair_tiles` tiles are the faster launch. `tiles_at`
// counts the token tiles at a limit, `largest_at` gives the tokens of the largest of them
// (where experts differ).
template <class TilesAt, class LargestAt>
inline int few_limit(TilesAt tiles_at, int64_t rows, int64_t features, int64_t contraction, int64_t pair_tiles,
                     int sm_count, LargestAt largest_at) {
  if (sm_count < 2) return 0;
  double best_us = 0.97 * pair_us(pair_tiles, contraction, sm_count);
  int best = 0;
  for (int limit : {kFewTokens / 2, kFewTokensShared, kFewTokens}) {
    const int64_t tiles = tiles_at(limit);
    const int64_t ctas = tiles * ((features + kFewFeatures - 1) / kFewFeatures);
    if (ctas > (int64_t(1) << 24) || (limit > kFewTokensShared && ctas > sm_count)) continue;
    const double us =
        few_us(tiles, static_cast<double>(rows) / tiles, features, contraction, sm_count, largest_at(limit));
    if (us < best_us) {
      best_us = us;
      best = limit;
    }
  }
  return best;
}
template <class TilesAt>
inline int few_limit(TilesAt tiles_at, int64_t rows, int64_t features, int64_t contraction, int64_t pair_tiles,
                     int sm_count) {
  return few_limit(tiles_at, rows, features, contraction, pair_tiles, sm_count, [](int) { return 0; });
}

// tmX: the activations [M, contraction] in boxes of 64 x kFewBoxRows, 2 kFewBoxRows
// and 4 kFewBoxRows (a dense launch: the first in boxes of 64 x few_box_rows), 128-byte
// swizzle; tmCodes: the packed codes in boxes of 64 bytes x 128
// rows, 64-byte swizzle.
cudaError_t launch_few(const FewArgs &a, const CUtensorMap (&tmX)[3], const CUtensorMap &tmCodes, int sm_count,
                       cudaStream_t stream);

struct GroupedArgs {
  int mode;
  int fmt;
  int E;                 // experts
  int64_t N, K;          // per expert: out features, in features
  const uint8_t *codes;  // [E, N, K/2]
  const uint8_t *scales; // [E, N, K/B]
  void *out;             // MODE_SGRAD: g [E, N, K/B] f32 (FWD / DX write through the table's maps)
  const uint8_t *mask;   // [E, N, K/B] or null (MODE_SGRAD only)
  int *err;
  const uint8_t *table;  // device copy of the expert table
  int total_tiles;       // tile_start[E]
};

// Launch one grouped contraction. tmCodes is the descriptor of all experts'
// packed codes as one [E * N, K/2] tensor.
cudaError_t launch_grouped(const GroupedArgs &a, const CUtensorMap &tmCodes, int sm_count, cudaStream_t stream);

// The contractions of the full-precision multiplicative control (a.fmt ignored):
// a.codes is the bf16 weight W [N, K], a.scales the fp32 coefficients dS [N, K/16];
// tmB the descriptor of W in 64 x 128 boxes with the 128-byte swizzle (FWD / DX),
// or of X (SGRAD, as launch_gemm).
cudaError_t launch_control(const GemmArgs &a, const CUtensorMap &tmA, const CUtensorMap &tmB,
                           const CUtensorMap *tmOut, int sm_count, cudaStream_t stream);
// out = alpha_over_r * B A (B [N, r], A [r, G] bf16), through `workspace`
// (lowrank_product_workspace bytes): the control's low-rank coefficient plane.
size_t lowrank_product_workspace(int64_t N, int64_t G, int r, int sm_count);
cudaError_t launch_lowrank_product(int64_t N, int64_t G, int r, float alpha_over_r, const uint16_t *B,
                                   const uint16_t *A, float *out, float *workspace, int sm_count, cudaStream_t stream);

// Launch one contraction. tmA is the TMA descriptor of the streamed bf16
// activations; tmB that of the packed codes (MODE_FWD / MODE_DX) or of the second
// bf16 operand (MODE_SGRAD); tmC that of the bf16 output (MODE_FWD / MODE_DX:
// 32-row x 32-column boxes, 64-byte swizzle) or of the packed codes (MODE_SGRAD). Codes
// come in boxes of 64 bytes x 128 rows, 64-byte swizzle.
cudaError_t launch_gemm(const GemmArgs &a, const CUtensorMap &tmA, const CUtensorMap &tmB, const CUtensorMap &tmC,
                        int sm_count, cudaStream_t stream);
// One thread waiting on a barrier nothing arrives on, bounded like every kernel wait:
// records kErrWaitTimeout in *err and returns (the failure-path self-test).
cudaError_t launch_wait_probe(int *err, cudaStream_t stream);

// Projection / merge of `count` latents. With ws2_per (device, one float per
// expert; NVFP4 only) the latents are the planes of several experts, `plane` (a
// multiple of 16) elements each, and element i uses ws2_per[i / plane] instead of ws2.
cudaError_t launch_project(int fmt, int64_t count, float ws2, const float *latent, uint8_t *bytes_out,
                           uint8_t *mask_out, int32_t *nonfinite, int sm_count, cudaStream_t stream,
                           const float *ws2_per = nullptr, int64_t plane = 0);

cudaError_t launch_merge(int fmt, int64_t count, float ws2, const float *latent, uint8_t *scales_inout,
                         float *ongrid_delta, int64_t *changed, int sm_count, cudaStream_t stream,
                         const float *ws2_per = nullptr, int64_t plane = 0);

// Projection / merge of several scale planes of different shapes in one launch
// (the planes of all linears of a layer). The table travels by value in the
// kernel's parameters; each plane's N * G is a multiple of 16. Counters are summed
// per CTA into `acc` (kMaxPlanes int64 plus a uint32 ticket, zero between calls:
// the last CTA writes each plane's count to its counter and clears them).
constexpr int kMaxPlanes = 16;
struct PlaneArgs {
  int64_t count;     // scale blocks (N * G)
  float ws2;         // NVFP4 tensor scale (1 for MXFP4)
  const float *latent;
  uint8_t *bytes;    // projection: bytes out; merge: the scale plane, in place
  uint8_t *mask;     // projection: mask out or null
  float *delta;      // merge: on-grid delta or null
  void *counter;     // projection: int32 NaN count; merge: int64 changed bytes; or null
};
struct PlaneTable {
  int n;
  PlaneArgs p[kMaxPlanes];
};
constexpr size_t kPlaneAccBytes = kMaxPlanes * sizeof(int64_t) + 16;
cudaError_t launch_project_planes(int fmt, const PlaneTable &t, int64_t *acc, cudaStream_t stream);
cudaError_t launch_merge_planes(int fmt, const PlaneTable &t, int64_t *acc, cudaStream_t stream);

// Rollback of a merge by its on-grid delta (in place, counting changed bytes), and
// copy a -> b (write) or only count the bytes in which a and b differ.
cudaError_t launch_rollback(int fmt, int64_t count, float ws2, const float *delta, uint8_t *scales_inout,
                            int64_t *changed, int sm_count, cudaStream_t stream);
cudaError_t launch_swap_or_diff(int64_t count, const uint8_t *a, uint8_t *b, bool write, int64_t *differing,
                                int sm_count, cudaStream_t stream);

// Low-rank scale adapter (Sec. 3 "Scale-QLoRA forward"): latent eff + (alpha/r) B A
// projected onto the grid; and the gradients of B and A from the masked scale
// gradient, through `workspace` (lowrank_grad_workspace bytes). With experts > 1
// the planes and factors of that many experts follow each other in memory (one
// launch for all); ws2_per (device, NVFP4) gives each expert's tensor scale.
cudaError_t launch_project_lowrank(int fmt, int64_t N, int64_t G, int r, float ws2, float alpha_over_r,
                                   const uint8_t *base, const uint16_t *B, const uint16_t *A, uint8_t *bytes_out,
                                   uint8_t *mask_out, int32_t *nonfinite, float *latent_out, int sm_count,
                                   cudaStream_t stream, int experts = 1, const float *ws2_per = nullptr);
// Ranks up to 128 run on the tensor cores (sq_adapter_tc.cu), larger ones on CUDA
// cores; `err` is the device error word (bounded waits of the tensor-core path).
size_t lowrank_grad_workspace(int64_t N, int64_t G, int r, int sm_count, int experts = 1);
cudaError_t launch_lowrank_grad(int64_t N, int64_t G, int r, float alpha_over_r, const float *g, const uint16_t *B,
                                const uint16_t *A, float *dB, float *dA, float *workspace, int sm_count,
                                cudaStream_t stream, int *err, int experts = 1);
bool lowrank_grad_tc_supported(int r);
size_t lowrank_grad_tc_workspace(int64_t N, int64_t G, int r, int experts, int sm_count);
cudaError_t launch_lowrank_grad_tc(int64_t N, int64_t G, int r, float alpha_over_r, const float *g,
                                   const uint16_t *B, const uint16_t *A, float *dB, float *dA, float *workspace,
                                   int *err, int sm_count, cudaStream_t stream, int experts);
constexpr int kMaxLowRank = 256;  // r limit of the adapter kernels

// Scale-family variants (ablation appendix): the least-squares code-preserving fit
// of a weight update per block; the group gradient and the group-delta projection
// of the granularity ladder (gd groups of G / gd blocks per row).
cudaError_t launch_fit(int fmt, int64_t N, int64_t K, float ws2, const uint8_t *codes, const uint8_t *scales,
                       const uint16_t *dW, float *delta, float *captured, float *total, float *latent, int sm_count,
                       cudaStream_t stream);
cudaError_t launch_group_reduce(int64_t N, int64_t G, int64_t gd, const float *g, float *out, int sm_count,
                                cudaStream_t stream);
cudaError_t launch_project_group_delta(int fmt, int64_t N, int64_t G, int64_t gd, float ws2, const uint8_t *base,
                                       const float *delta, uint8_t *bytes_out, uint8_t *mask_out, int32_t *nonfinite,
                                       float *latent_out, int sm_count, cudaStream_t stream);

// Token routing (sq_route.cu): router logits [T, E] (fp32 or bf16) to the top-k experts and
// weights, and their gradient; the n = T * k slots sorted by expert; rows to the experts and back.
constexpr int kRouteMaxExperts = 1024;  // 32 logits a lane; the sort's histograms fit shared memory
constexpr int kRouteMaxK = 32;          // a token's slots are the lanes of a warp
constexpr int64_t kMaxMoveUnits = (int64_t(1) << 31) - 8;  // 256-column pieces of all tokens
cudaError_t launch_route(int64_t T, int E, int k, bool bf16, const void *logits, const uint8_t *valid, bool normalize,
                         int *experts, float *weights, cudaStream_t stream);
cudaError_t launch_route_grad(int64_t T, int E, int k, bool bf16, const void *logits, const int *experts,
                              const float *dweights, bool normalize, void *dlogits, cudaStream_t stream);
size_t sort_workspace(int64_t n, int E, int sm_count);
cudaError_t launch_sort(int64_t n, int E, const int *experts, int64_t *offsets, int *row_of, int *slot_of,
                        int *workspace, int sm_count, cudaStream_t stream);
cudaError_t launch_dispatch(int64_t T, int k, int64_t D, int64_t rows, const uint16_t *X, const int *row_of,
                            const int *slot_of, uint16_t *Xs, cudaStream_t stream);
cudaError_t launch_combine(int64_t T, int k, int64_t D, int64_t rows, const uint16_t *Ys, const int *row_of,
                           const float *weights, uint16_t *Y, int sm_count, cudaStream_t stream);
cudaError_t launch_combine_grad(int64_t T, int k, int64_t D, int64_t rows, const uint16_t *dY, const uint16_t *Ys,
                                const int *row_of, const int *slot_of, const float *weights, uint16_t *dYs,
                                float *dweights, int sm_count, cudaStream_t stream);

// Cross entropy against a vocabulary projection W [V, D] (sq_loss.cu). A call runs over pieces of
// kHeadPiece tokens, a piece's labelled tokens over chunks of whole tiles whose exponentials (or, without
// a gradient, sums) fit kHeadPieceBytes of scratch, or of one tile; their partial planes fit it too.
constexpr int kHeadTile = 256;
constexpr int kHeadPiece = 16384;
constexpr int64_t kHeadPieceBytes = int64_t(512) << 20;
constexpr int kMaxHeadParts = 64;
// Products of the gradient added up in one accumulator. (2048 rows against 50257 x 1024 whose rows share a
// part of 30 times their own size, relative error of dX with its bf16 rounding of 0.00166: 0.00175; with
// 8192 0.0021, unbroken 0.0046. 2048 takes 3 % of the call.)
constexpr int kHeadSegment = 4096;
constexpr int kMinHeadPartStages = 2;  // a part of the vocabulary is at least 2 x 128 entries long

// Vocabulary parts of a gradient launch over `rows` rows of D columns, `stages` 128 deep: the s with
// the least estimate of the launch, ceil(tiles s / clusters) / s tiles per cluster at 0.56 us a
// stage, and of the s fp32 planes it writes and the row kernel reads back, at 5 TB/s. (The longest
// waves alone as the rule gave 2048 rows against 38912 x 2048 19 parts: product and rows 184 + 38
// us; unsplit 170 + 9.)
inline int head_parts(int64_t rows, int64_t D, int stages, int clusters) {
  const int most = std::max(1, std::min(stages / kMinHeadPartStages, kMaxHeadParts));
  const int64_t tiles = (rows + kHeadTile - 1) / kHeadTile * ((D + kHeadTile - 1) / kHeadTile);
  const double plane_us = static_cast<double>(rows) * static_cast<double>(D) * 8 / 5e6;
  auto us = [&](int s) {
    return static_cast<double>((tiles * s + clusters - 1) / clusters) / s * stages * 0.56 + s * plane_us;
  };
  int best = 1;
  for (int s = 2; s <= most; ++s)
    if (us(s) < us(best)) best = s;
  return best;
}

// Columns of a tile of the logits: 256, or fewer where the call is one row of tiles and they would
// leave clusters idle, by the waves of the launch, a tile of 128 columns lasting 0.54 and one of 64
// lasting 0.4 of one of 256 (8 tokens against 3211 x 2312, loss and gradient: 32.7 us with 256, 26.6
// with 64; 32 against 64000 x 2048: 57.7, 51.3 with 128). Where the MMAs bound the launch, only if
// it is one wave (200 tokens against 64000 x 2048: 61.3, 64.7).
inline int head_columns(int64_t T, int64_t V, bool few, int clusters) {
  auto waves = [&](int64_t columns) {
    return static_cast<double>(((V + columns - 1) / columns + clusters - 1) / clusters);
  };
  if (T > kHeadTile || (!few && waves(256) > 1)) return 256;
  const double wide = waves(256), half = 0.54 * waves(128), quarter = 0.4 * waves(64);
  if (quarter < wide && quarter < half) return 64;
  return half < wide ? 128 : 256;
}

struct HeadArgs {
  int T;                  // tokens of the piece
  int64_t D, V;
  const uint16_t *X;      // [T, D] bf16
  const uint16_t *W;      // [V, D] bf16
  const int64_t *labels;  // [T]; outside [0, V): no label
  const float *dloss;     // [T] (gradient)
  float *loss, *lse;      // [T] or null
  uint16_t *dX;           // [T, D] bf16, or null: no gradient
  int box_rows;           // rows of A in a shared-memory stage: 16, 32, 64 or 128, all that few tokens have
  bool few;               // box_rows < 128: stages of 128 instead of 64
  int columns;            // of a tile of the logits
  bool long_sums;         // the gradient's parts are longer than kHeadSegment
  int chunk;              // rows of a chunk: a multiple of kHeadTile, or all of a shorter call, up to one of 16
  uint8_t parts[kHeadPiece / kHeadTile];  // vocabulary parts of the gradient by row tiles of the chunk, less 1
  int64_t pitch;          // elements from row to row of e
  int64_t width;          // and of the packed rows and partial planes
  // scratch, by compact row of the piece
  int *count;             // labelled tokens of the piece
  int *token, *label;
  float *label_z;
  float2 *factors;        // of the row kernel
  uint16_t *rows;         // [T, D] the labelled tokens' rows of X
  // scratch, by row of the chunk
  int sum_rows;           // a chunk's rows, up to a multiple of 4
  // [4 * column tiles, sum_rows] of each quarter tile: its sum (with a gradient, float2: and that of its rounded
  // exponentials) and its reference
  float *sums, *refs;
  int *moved;             // [chunk] a row whose references differ (refs are read only there)
  uint16_t *e;            // [chunk, pitch] bf16 exponentials (gradient)
  float *partial;         // [parts, rows, D] fp32 (gradient)
  int *err;
};
// rows and e_load: 64 x box_rows boxes, weights 64 x columns / 2, weights_grad 64 x 128 (few) or 64 x
// 64, partial 32 x 32 fp32, all with the 128-byte swizzle; e_store 32 x 32, and partial of long sums 16
// x 32, 64-byte swizzle.
struct HeadMaps {
  CUtensorMap rows, weights, weights_grad, e_store, e_load, partial;
};
cudaError_t launch_head_gather(const HeadArgs &a, cudaStream_t stream);
cudaError_t launch_head_chunk(const HeadArgs &a, const HeadMaps &m, int first, int sm_count, cudaStream_t stream);

// Rows of FP4 (sq_rows.cu, sq_fp4.cu).
struct QuantArgs {
  int64_t R;           // rows of codes
  int K, last;         // values of a row, and of the last one (quantisation)
  uint8_t *codes, *scales;
  float *row_ws2;      // each row's own scale, or null: ws2 for all
  float ws2, inv;      // inv: fl32(1 / ws2)
  // quantisation
  const uint16_t *X;
  const int32_t *slot_of;  // [R] slot of a row, its source row slot / k; null: row r is X[r]
  int k;
  int64_t slots;           // T * k
  bool wide;               // X starts on 32 bytes
};
cudaError_t launch_quantize(int fmt, const QuantArgs &a, int sm_count, cudaStream_t stream);
cudaError_t launch_spread(int fmt, const QuantArgs &a, const QuantArgs &tokens, cudaStream_t stream);
// R rows by slot of T tokens: whether to quantise each token once and copy its row. Quantising is bound by its
// arithmetic where rows come from the L2, 2.3 (NVFP4) or 3.6 values in a picosecond; a copied value costs a third (NVFP4) or
// a half of that, and the second launch about 2 us. Measured, one launch against two, in us: NVFP4, 2048 values a row, 512 tokens of 8 rows
// each 5.3 against 5.5, 2048 of 2 5.3 and 7.3, 2048 of 8 15.0 and 9.4, 8192 of 2 15.0 and 13.2; MXFP4, 2880 values, 2048
// tokens of 4 8.1 and 6.7, 8192 of 4 30.7 and 21.8, 2048 of 8 14.7 and 8.6.
inline bool quantize_tokens_first(int fmt, int64_t R, int64_t T, int K) {
  const double values = 1e-6 * K;
  return values * (static_cast<double>(R) - T) / (fmt == 0 ? 2.3 : 3.6) > 2.2 + values * R / 6.5;
}
cudaError_t launch_dequantize(int fmt, const QuantArgs &a, uint16_t *X, int sm_count, cudaStream_t stream);

// Products of FP4 rows with FP4 weights (sq_fp4.cu).
constexpr int kFp4FewTokens = 128;           // of a tile of the few-token kernel, at most
constexpr int kFp4FewBoxes = 5;              // boxes of 8 .. 128 token rows
constexpr int kFp4SmemAlone = 224 * 1024;    // of a CTA alone on its SM
constexpr int kFp4SmemShared = 112 * 1024;   // ... of two
constexpr int kFp4SmemMost = 232448 - 1536;  // ... beside its static shared memory
constexpr int kFp4PairTokens = 256, kFp4PairFeatures = 256;  // a tile of the pair kernel, at most
constexpr int kFp4PairApart = 224;  // two accumulators of up to so many tokens lie beside each other; wider ones overlap
constexpr int kFp4PairBoxes = 6;    // boxes of 8 .. 64, 112 and 128 token rows
__host__ __device__ constexpr int fp4_pair_box(int i) { return i < 4 ? 8 << i : i == 4 ? kFp4PairApart / 2 : kFp4PairTokens / 2; }
struct Fp4Maps {
  CUtensorMap w;                // codes [E][N][K / 2], boxes of 128 bytes x 128 rows
  CUtensorMap x[kFp4FewBoxes];  // codes [R][K / 2], boxes of 128 bytes x (8 << i) rows
  CUtensorMap w_scales, x_scales[kFp4FewBoxes];  // scale bytes, boxes of 16 bytes x the same rows (whole 16-byte rows only)
};
struct Fp4PairMaps {
  CUtensorMap w, x[kFp4PairBoxes];  // codes, boxes of 128 bytes x 128 features and of as many token rows
  CUtensorMap w_atoms, x_atoms;     // [atoms][512 bytes], boxes of a stage's of 128 features and 256 rows
};
struct Fp4Args {
  int64_t R;                 // rows
  int E, N, K, G;            // experts (1: dense), out features, in features, scale bytes of a row
  const uint8_t *w_scales, *x_scales;
  const float *w_ws2;        // device [E], or null: ws2
  float ws2;
  const float *row_ws2;      // device [R], or null: x_ws2
  float x_ws2;
  const int64_t *offsets;    // device [E + 1] of a grouped call, or null
  uint16_t *out;
  int *err;
  int ftiles;                // feature tiles
  bool pair;                 // the pair kernel, else the few-token one
  int tile_tokens;           // few: tokens of a tile (8 .. 128, a power of two); pair: of a whole one of a dense product
  int64_t units;             // tiles, at most
  int splits;                // few: parts of the contraction (CTAs of a cluster)
  int stages;                // of the ring
  // pair: atoms of the scales, [token tile][slice][2] and [block of 128 features][slice], and per CTA that writes them
  // whether it met a negative one
  uint4 *x_atoms, *w_atoms;
  int *negative;
  int token_blocks, atom_ctas;
  int slices;                // pair: of 256 of the contraction, in a stage: 1 or 2
  int depth;                 // pair: stages of the contraction
  int whole;                 // pair, dense: whole token tiles
};
// A few-token stage: codes of 128 features and a tile's tokens, scales of 128 rows of both. A slice
// of a pair stage: codes of 128 features and half the tokens, atoms of those features and of 256 tokens; behind the
// ring eight 1 KiB boxes of the epilogue and the experts' tiles and rows.
constexpr int fp4_few_stage(int tile_tokens) { return 128 * 128 + tile_tokens * 128 + 2 * 2048; }
__host__ __device__ constexpr int fp4_atoms(int fmt) { return fmt == 0 ? 2048 : 1024; }  // bytes of 128 rows and a slice
__host__ __device__ constexpr int fp4_atom_stages(int fmt) { return fmt == 0 ? 8 : 16; }  // slices of a CTA that writes atoms
__host__ __device__ constexpr int fp4_pair_stage(int fmt, int slices, bool wide) {
  return slices * (128 * 128 + (wide ? kFp4PairTokens : kFp4PairApart) / 2 * 128 + 3 * fp4_atoms(fmt));
}
constexpr size_t fp4_pair_smem(int fmt, int slices, bool wide, int stages, int E) {
  return 1024 + static_cast<size_t>(stages) * fp4_pair_stage(fmt, slices, wide) + 8 * 1024 + (E > 0 ? 4 * (4 * E + 1) : 0);
}
// Tokens of a whole tile of a dense product. The launch lasts as long as its waves of tiles, 400 + 1.15 h
// cycles a slice of a tile of h tokens (fitted; the MMAs alone take 2 h) and 1.23 times that where accumulators overlap (of
// 8 slices on; of fewer the wait between tiles weighs more). The factor is that wait in a tile of about 16 slices, charged
// by the slice: a deeper tile waits no longer, so it keeps some tall tiles from products that they would suit.
// The product alone in us, in tiles of 224 or fewer against 240 or 256, the taken side first. NVFP4: 1024 tokens against 8192
// x 2048 in 256 18.5, in 160 19.7; 2048 against 4096 x 2048 in 240 18.4, in 224 19.4; 1024 against 8192 x 8192 in 256 33.6, in
// 224 36.5; 2048 against 4096 x 14336 in 240 48.3, in 224 51.3; 4096 against 4096 x 4096 in 224 31.5, in 256 35.5. It
// misses 1000 against 8192 x 14336 in 144 59.0, in 256 51.7, 2048 against 14336 x 14336 in 224 174, in 256 156, and of MXFP4,
// whose shallow tiles of up to 224 have two slices a stage, 1024 against 8192 x 2048 in 256 18.0, in 160 17.2 and 2048
// against 4096 x 2048 in 240 17.9, in 224 16.7.
inline int fp4_pair_tokens(int64_t R, int64_t ftiles, int clusters, int slices) {
  auto cost = [](int64_t h) { return h > kFp4PairApart ? 1.23 * (400 + 1.15 * h) : h > 0 ? 400 + 1.15 * h : 0.0; };
  double best = 0;
  int tokens = kFp4PairApart;
  for (int h = slices >= 8 ? kFp4PairTokens : kFp4PairApart; h >= 96; h -= 16) {
    const int64_t whole = R / h * ftiles, rest = R % h ? ftiles : 0, waves = (whole + clusters - 1) / clusters;
    const int64_t left = waves * clusters - whole;
    const double cycles = waves * cost(h) + (rest > left ? (rest - left + clusters - 1) / clusters * cost(R % h) : 0.0);
    if (best == 0 || cycles < best) {
      best = cycles;
      tokens = h;
    }
  }
  return tokens;
}
// Clusters of 1 .. 8 CTAs of the few-token kernel that a device runs at once, a CTA alone on its SM or two on one. (CUDA
// 13.0 counts one CTA of this kernel to an SM, whatever its shared memory, though two do run there: both counts are 152,
// 76, 46, 36, 28, 23, 15 and 15 clusters, and a cut product is one CTA to an SM.)
struct Fp4Clusters {
  int alone[9], shared[9];  // alone[0] == 0: not asked yet
};
cudaError_t fp4_clusters(Fp4Clusters &fit);
// Kernel, tiles and parts of a product on sm_count SMs: fills the last fields of p.
//
// The kernel is chosen by estimates of both in microseconds, for each expert's rows where there are experts. Both
// sides, few-token against pair kernel with the launches ahead, measured with NVFP4, in us: 4096 x 4096 8 against 11
// with 32 rows, 21 against 22 with 1024; 4096 x 14336 13 against 20 with 32, 29 against 27 with 384; 14336 x 4096 11
// against 13 with 32, 31 against 23 with 384; 128 experts of 768 x 2048 17 against 26 with a row each, 41 against 38 with
// 16 (the estimates' worst miss), 104 against 75 with 256; of 2880 x 2880 (MXFP4) 79 against 84 with a row, 154
// against 120 with 16, 380 against 193 with 256.
inline void fp4_plan(int fmt, int sm_count, const Fp4Clusters &fit, Fp4Args &p) {
  auto up = [](double x, double n) { return static_cast<double>(static_cast<int64_t>((x + n - 1) / n)); };
  const int64_t groups = p.offsets ? std::min<int64_t>(p.E, p.R) : 1;
  const int cnt = (p.K + 255) / 256, clusters = sm_count / 2;
  const int ftiles = (p.N + 127) / 128, pair_ftiles = (p.N + kFp4PairFeatures - 1) / kFp4PairFeatures;
  int few_tokens = 8;
  while (few_tokens < kFp4FewTokens && few_tokens * groups < p.R) few_tokens *= 2;
  const int64_t few_units = (p.R + (few_tokens - 1) * groups) / few_tokens * ftiles;
  // Parts: as many as let all clusters run at once, a CTA to an SM or, where a part has few stages, two. (18 clusters of
  // 8, of which 15 fit: 187 tokens against 1048 x 2720 18.8 us, 12.5 in 6 parts; 48 of 3, of which 46 fit: a token
  // through 8 experts of 768 x 2048 12.7, 8.0 in 2.) The parts of many tokens take longer to add up than they save (256
  // against 1024 x 4096 22.6 us in 8 parts, 12.4 in 4; 64 the same in 8 and 4).
  const int stage = fp4_few_stage(few_tokens), shared_stages = std::min(8, (kFp4SmemShared - 1024) / stage);
  int splits = std::min(few_tokens <= 32 ? 8 : 4, cnt);
  auto fits = [&](int s) {
    return few_units <= fit.alone[s] || ((cnt + s - 1) / s <= shared_stages && few_units <= fit.shared[s]);
  };
  while (splits > 1 && !fits(splits)) --splits;
  const bool alone = few_units <= fit.alone[splits];
  // What the launches take: rounds of CTAs (two on an SM), or waves of pair tiles and, at least, the weight's way
  // from memory. Tiles of ragged experts are half empty on average.
  const int pair_tokens = p.offsets ? kFp4PairApart : fp4_pair_tokens(p.R, pair_ftiles, clusters, cnt);
  const double rows = static_cast<double>(p.R) / groups;
  const double few_tiles = p.offsets ? (p.R + 0.5 * few_tokens * groups) / few_tokens * ftiles : few_units;
  const double pair_tiles = (p.offsets ? (p.R + 0.5 * pair_tokens * groups) / pair_tokens : up(p.R, pair_tokens)) * pair_ftiles;
  const double height = std::min<double>(pair_tokens, rows);
  const double bytes = groups * static_cast<double>(p.N) * p.K * 0.56, atoms = (static_cast<double>(p.E) * p.N + p.R) * p.G * 2;
  const double few_us = 2 + std::max(bytes / 5.5e6, (alone ? 1.0 : up(few_tiles, 2 * sm_count)) *
                                                        (up(cnt, splits) * (alone ? 0.35 + 0.0022 * few_tokens : 0.75) + 2 + 0.02 * few_tokens));
  const double pair_us = 9 + atoms / 3.5e6 + std::max(bytes / 5.5e6, up(pair_tiles, clusters) * (cnt * (0.2 + 0.0007 * height) + 0.5));
  p.pair = pair_us < few_us || few_units > (int64_t(1) << 30);
  if (p.pair) {
    p.ftiles = pair_ftiles;
    p.tile_tokens = pair_tokens;
    const int64_t token_tiles = (p.R + (pair_tokens - 1) * groups) / pair_tokens;
    p.units = token_tiles * p.ftiles;
    p.whole = static_cast<int>(p.R / pair_tokens);
    // Two slices a stage halve the waits, commits and loads (one, two; us with the tokens' quantisation: 16384 x 14336
    // x 4096 NVFP4 352, 340, 2048 x 4096 x 14336 MXFP4 68, 63). Experts' narrow tiles wait for their loads and
    // want the finer ring (8111 tokens to four of 128 of 2880 x 2880 200, 204). An odd slice behind K is computed as
    // zeros: not where it would be more than a 17th of all. Of tall NVFP4 tiles only two such stages would fit.
    p.slices = !p.offsets && (cnt % 2 == 0 || cnt > 16) && (fmt == 1 || pair_tokens <= kFp4PairApart) ? 2 : 1;
    p.depth = (cnt + p.slices - 1) / p.slices;
    p.token_blocks = static_cast<int>(2 * token_tiles);
    p.atom_ctas = static_cast<int>((p.token_blocks + 2 * int64_t(p.E) * p.ftiles) *
                                   ((p.depth * p.slices + fp4_atom_stages(fmt) - 1) / fp4_atom_stages(fmt)));
    p.splits = 1;
    p.stages = 8;
    while (fp4_pair_smem(fmt, p.slices, pair_tokens > kFp4PairApart, p.stages, p.offsets ? p.E : 0) > static_cast<size_t>(kFp4SmemMost)) --p.stages;
    return;
  }
  p.ftiles = ftiles;
  p.tile_tokens = few_tokens;
  p.units = few_units;
  p.splits = splits;
  p.stages = alone ? std::min(8, (kFp4SmemAlone - 1024) / stage) : shared_stages;
}
cudaError_t launch_fp4_few(int fmt, const Fp4Maps &maps, const Fp4Args &p, cudaStream_t stream);
cudaError_t launch_fp4_pair(int fmt, const Fp4PairMaps &maps, const Fp4Args &p, int sm_count, cudaStream_t stream);

// Device-side error codes written to the error word.
constexpr int kErrWaitTimeout = 1;

}  // namespace sqi
