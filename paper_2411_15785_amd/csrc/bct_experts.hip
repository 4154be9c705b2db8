// The products of tokens with their experts (gfx950).  A pair p is token p / k with its slot p % k, e(p) its expert:
//
//   h[p]   = silu(x[p / k] Wg_e^T) * (x[p / k] Wu_e^T)                       bctm_expert_swiglu
//   out[r] = residual[r] + sum over s of weight[r][s] * (h[r k + s] Wd_e^T)  bctm_expert_linear
//
// Pairs come by expert (the plan of bct_route.hip), in row tiles that belong to one expert each; rows are gathered where they lie.
// Few pairs an expert: bound by reading the weights of the experts in use once, so a kernel that streams them against
// 16 rows.  Many: bound by the matrix cores, the kernel of bct_linear_rows.hip with gathered rows, the tiles of an expert side by side
// on an XCD and of the same size.  The way back leaves each pair's product in fp32, and a second kernel weights and adds up those of a token in
// the order of its slots.  (Products in 16 bits with a power of two for every eight features took half of that traffic, 4096 tokens below 498 us,
// but left a feature a thousand times smaller than its neighbour 3 % off.)
//
// us in a graph, weights from memory: 32 tokens of 8 in 64 experts, gated 4096 -> 1376 208 (1.42 GB, 6.8 TB/s), back 115 (6.2); 4096 tokens 700 (1.06
// PFLOP/s; clock 1.6 GHz, matrix cores busy 69 % of the cycles, 2.2 GB from memory; with the weights of one expert for all 607) and 586 (0.63, the sum 120 of
// them); 777 of 2 in 12, 2080 -> 2048 back 47.  Measured and not kept: lines of weights read ahead into the L2, 4 to 16 K steps (4096 tokens
// 4 to 13 % slower: each line is one more request), six stages of 64 x 128 or 128 x 256 (the same times), weights side by side by groups of 2 to 8 feature
// tiles (the same), past the caches (4 % slower), rows past the caches (a third slower), four wavefronts of 64 x 128 or 128 x 64 each (the
// same, 10 % slower), 128 x 128, 64 x 64 and 128 x 64 with K in two parts (slower but for 5 to 15 % at 24 to 64 rows an expert of small matrices), all 16-row tiles
// multiplied whether they hold rows or not (2 to 4 % slower).
#include <math.h>

#include "bct_linear_rows.h"
#include "bct_model_internal.h"

namespace bct {

namespace {

// A workgroup has one row tile (up to 16 pairs of an expert) and FT feature tiles of 16; its wavefronts share K.
template <bool SWIGLU, int WAVES, int U, int FT>
__global__ __launch_bounds__(64 * WAVES) void expert_few_kernel(const uint16_t* __restrict__ x, const u32x4* __restrict__ w,
                                                                const u32x4* __restrict__ w2, uint16_t* out, uint32_t K, uint32_t N,
                                                                ExpertTerm T) {
  constexpr int NW2 = SWIGLU ? 2 : 1, NS = FT * NW2, NTHR = 64 * WAVES;
  __shared__ float sC[WAVES][NS][16][17];
  const uint32_t NT = N / 16, features = (NT + FT - 1) / FT, nt0 = blockIdx.x % features * FT, t = blockIdx.x / features;
  if (t >= *T.n_tiles) return;
  const ExpertTile tile = expert_tile(T, t);
  if (tile.tile * 16 >= tile.pairs) return;
  const uint32_t rows = min(tile.pairs - tile.tile * 16, 16u);
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, jl = lane % 16, kg = lane / 16, KT = K / 32;
  const uint32_t kt0 = (uint32_t)((uint64_t)wave * KT / WAVES), kt1 = (uint32_t)((uint64_t)(wave + 1) * KT / WAVES);
  const int32_t* order = T.order + tile.begin + tile.tile * 16;
  const u32x4* wt[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s)   // a feature tile past the end: the last one again, not stored
    wt[s] = ((s % NW2) ? w2 : w) + tile.expert * T.stride + ((size_t)min(nt0 + s / NW2, NT - 1) * KT + kt0) * 64 + lane;
  const bool there = jl < rows;   // lanes of rows that are not there load nothing
  const uint16_t* xr = x + (size_t)(expert_pair(T, order, there ? jl : 0u) / T.per_row) * K + (size_t)kt0 * 32 + kg * 8;
  f32x4 acc[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) acc[s] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t n_t = kt1 - kt0;
  // Rounds of U tiles, all requested before the first product; the missing tiles of the last round are not loaded and count as 0.
  for (uint32_t k = 0; k < n_t; k += U) {
    u32x4 b[U][NS], a[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool is = k + u < n_t;
      a[u] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int s = 0; s < NS; ++s) b[u][s] = is ? __builtin_nontemporal_load(wt[s] + (size_t)(k + u) * 64) : u32x4{0u, 0u, 0u, 0u};
      if (is && there) a[u] = *(const u32x4*)(xr + (size_t)(k + u) * 32);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int s = 0; s < NS; ++s)
        acc[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[u]), __builtin_bit_cast(bf16x8, b[u][s]), acc[s], 0, 0, 0);
  }
  // element v of a lane: row 4 * kg + v, feature jl; the wavefronts' sums are added in their order
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int v = 0; v < 4; ++v) sC[wave][s][4 * kg + v][jl] = acc[s][v];
  __syncthreads();
  for (uint32_t o = threadIdx.x; o < FT * 256; o += NTHR) {
    const uint32_t f = o / 256, i = o % 256 / 16, j = o % 16, n = (nt0 + f) * 16 + j;
    if (i >= rows || n >= N) continue;
    float sum[NW2];
#pragma unroll
    for (int m = 0; m < NW2; ++m) {
      sum[m] = 0.f;
#pragma unroll
      for (int k = 0; k < WAVES; ++k) sum[m] += sC[k][f * NW2 + m][i][j];
    }
    const size_t at = (size_t)expert_pair(T, order, i) * N + n;
    if (SWIGLU) store_elem(out, at, sum[0] / (1.0f + __expf(-sum[0])) * sum[NW2 - 1]);
    else T.sums[at] = sum[0];
  }
}

// out[r][8 c ..] = residual + the token's products, weighted, in the order of its slots.  A thread has eight features of a token.
// S slots are requested at once, whether they have an expert or not: behind a branch they would be waited for one by one.
template <int S>
__global__ __launch_bounds__(256) void combine_kernel(const float* sums, const int32_t* expert, const float* weights, const uint16_t* residual,
                                                      uint16_t* out, uint32_t rows, uint32_t k, uint32_t N) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x, chunks = N / 8, r = i / chunks, c = i % chunks;
  if (r >= rows) return;
  float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (uint32_t s = 0; s < k; s += S) {
    f32x4 v[S][2];
    int32_t id[S];
    float w[S];
#pragma unroll
    for (int u = 0; u < S; ++u) {
      const size_t p = (size_t)r * k + min(s + u, k - 1);
      id[u] = s + u < k ? expert[p] : 0;
      w[u] = weights[p];
#pragma unroll
      for (int h = 0; h < 2; ++h) v[u][h] = ((const f32x4*)sums)[(p * chunks + c) * 2 + h];
    }
#pragma unroll
    for (int u = 0; u < S; ++u) {
      if (id[u] == 0) continue;   // its product was not computed
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = __builtin_fmaf(w[u], v[u][e / 4][e % 4], y[e]);
    }
  }
  if (residual) {
    float v[8];
    unpack16<BF16>(*(const u32x4*)(residual + (size_t)r * N + 8 * c), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] += v[e];
  }
  *(u32x4*)(out + (size_t)r * N + 8 * c) = pack16_round<BF16>(y);
}

// The form of a product's sizes: what a workgroup has, 16 rows of the streaming kernel or 64 x 128, 128 x 256 or 256 x 256 of
// rows and columns (two of a SwiGLU's feature).  The host knows how many pairs there are, not how many each expert has: as many experts
// are taken to be used as if all were as likely, and about mean / rows + 1/2 row tiles each, at least one.  Estimates in us from
//   streaming   every row tile reads the expert's weights: 6.7 TB/s
//   64 x 128    0.17 a K step alone on its compute unit, 0.21 for each of several
//   128 x 256   0.40 a K step where one round of workgroups is enough, else 0.30 for each of a compute unit, as much again for the part of its rows that
//               is used, and 3 for its ends, which a second workgroup covers in part
//   256 x 256   0.48; 0.45 and as much again, 9 for its ends, and half a round that is not full
// and for the last three the weights at 5.6, 5.6 and 5.9 TB/s.  90 drawn shapes take 0.5 % longer than in their best form, in the geometric
// mean, with weights from memory.  Measured us, streaming | 64 x 128 | 128 x 256 | 256 x 256, gated K = 4096, N = 1376, 64 experts with a mean
// of 4: 209 | 240 | 260 | 234; 8: 237 | 251 | 272 | 245; 16: 325 | 260 | 280 | 247; 48: 806 | 297 | 295 | 278; 128: - | 439 | 330 | 332; 512: - | 1232 |
// 779 | 677.  8 experts, 2048, 1024, mean 4: 12.6 | 19.3 | 32.2 | 29.7; 16: 18.1 | 19.6 | 32.5 | 30.2; 64: 43.0 | 22.2 | 36.8 | 37.4; 192: 110 | 34.1 | 38.6 |
// 51.0; 384: 208 | 55.5 | 39.0 | 50.4.  The way back (with its sum), 12 experts, 2080 -> 2048, mean 8: 23.3 | 26.8 | 40.0 | 37.6; 32: 42.7 | 30.2 | 42.8 | 42.3;
// 128: 124 | 47.9 | 52.8 | 62.1; 64 experts, 1376 -> 4096, 8: 133 | 143 | 142 | 147; 32: 295 | 170 | 161 | 165; 128: - | 274 | 231 | 236; 512: - | 839 | 630 | 586.  8
// experts, 1376 -> 4096, 750: - | 156 | 131 | 116, of which the estimate takes 131.  Beyond the sizes of the estimate, 8 experts, gated 4096 -> 14336, mean 8: 291 |
// 312 | 319 | 322; 64: 1412 | 428 | 367 | 367; 256: - | 964 | 621 | 591; back 8: 147 | 159 | 229 | 202; 64: 659 | 270 | 258 | 257; 256: - | 541 | 468 | 377, of which it
// takes 468, the most that it was off; 256 experts, gated 7168 -> 2048, mean 8: 2345 | 2364 | 2372 | 2340; 128: - | 4566 | 3366 | 3190.
// Tokens that share their experts: the streaming kernel reads an expert's weights once for 16 of them, 64 tokens of the same 8 in 64
// 4096 -> 1376 in 124 us (two forms on, 128 tokens, in 80), where 64 that choose theirs apart take 240.
enum ExpertForm { kFew, kRows64, kRows128, kRows256 };   // in the order of kPlanRows
constexpr uint32_t few_features(bool swiglu) { return swiglu ? 1 : 2; }   // feature tiles of a streaming workgroup
ExpertForm expert_form(uint32_t pairs, uint32_t E, uint32_t K, uint32_t N, bool swiglu) {
  const double used = E * -expm1(-(double)pairs / E), mean = pairs / used, bcols = swiglu ? 2.0 * N : N, KT = K / 32, expert = 2.0 * K * bcols;
  auto tiles = [&](double rows) { return used * (mean / rows > 0.5 ? mean / rows + 0.5 : 1.0); };
  ExpertForm best = kFew;
  double cost = 4 + tiles(16) * expert / 6.7e6;
  auto take = [&](ExpertForm f, double c) {
    const double stream = 4 + used * expert / (f == kRows256 ? 5.9e6 : 5.6e6);
    c = c > stream ? c : stream;
    if (c < cost) {
      cost = c;
      best = f;
    }
  };
  auto groups = [&](double rows, double cols) { return tiles(rows) * ceil(bcols / cols) / 256; };   // workgroups of a compute unit
  auto full = [&](double rows, double cols) { return pairs / rows * ceil(bcols / cols) / 256; };   // of them, were all of their rows used
  auto most = [](double a, double b) { return a > b ? a : b; };
  const double g64 = groups(64, 128), g128 = groups(128, 256), g256 = groups(256, 256);
  take(kRows64, 7 + KT * (g64 > 0.8 ? 0.21 * g64 : 0.17));
  take(kRows128, most(8 + KT * 0.40, 3 * g128 + KT * 0.30 * (g128 + full(128, 256))));
  take(kRows256, most(13.9 + KT * 0.48, 9 * g256 + KT * 0.45 * (g256 + full(256, 256) + 0.6)));
  return best;
}

// What a workgroup of a form has of the features.
uint32_t form_features(ExpertForm form, bool swiglu) {
  return form == kFew ? 16 * few_features(swiglu) : (form == kRows64 ? 128 : 256) / (swiglu ? 2 : 1);
}
uint64_t form_groups(ExpertForm form, uint32_t pairs, uint32_t E, uint32_t N, bool swiglu) {   // workgroups of the launch
  const uint32_t features = form_features(form, swiglu);
  return (uint64_t)ExpertPlan::most_tiles(pairs, E, kPlanRows[form]) * ((N + features - 1) / features);
}
constexpr uint64_t kMostThreads = 0xFFFFF000u;   // of a launch

bct_status check_products(const void* x, const void* w, const void* out, const void* plan, uint32_t rows, uint32_t k, uint32_t E,
                          uint32_t K, uint32_t N, bool swiglu) {
  if (!x || !w || !out || K == 0 || N == 0) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer or zero size");
  const bct_status st = check_expert_plan(plan, rows, k, E);
  if (st != BCT_OK) return st;
  if (K % 32 != 0 || N % 16 != 0) return mfail(BCT_ERR_UNSUPPORTED, "K must be a multiple of 32 and N of 16");
  if (K > 1u << 24 || N > 1u << 24) return mfail(BCT_ERR_UNSUPPORTED, "matrix too large");
  if ((form_groups(expert_form(rows * k, E, K, N, swiglu), rows * k, E, N, swiglu) + 8) * 512 > kMostThreads || (!swiglu && (uint64_t)rows * (N / 8) > kMostThreads))
    return mfail(BCT_ERR_UNSUPPORTED, "too many tokens");
  if (!al16(x) || !al16(w) || !al16(out)) return mfail(BCT_ERR_MISALIGNED, "pointers must be 16-byte aligned");
  if (x == out) return mfail(BCT_ERR_INVALID_ARG, "out must not be x");
  return BCT_OK;
}

template <bool SWIGLU, int MI, int NJ, int WR, int WC, int KS>
void launch_rows_of(const void* x, const void* w, const void* w2, void* out, uint32_t K, uint32_t N, const ExpertTerm& T, hipStream_t s) {
  const uint32_t bcols = SWIGLU ? 2 * N : N, NT = (bcols + 16 * NJ * WC - 1) / (16 * NJ * WC);
  const dim3 grid(8 * ((T.most_tiles * NT + 7) / 8)), block(64 * WR * WC * KS);
  const LinearOut dst = {{(uint16_t*)out, nullptr, nullptr}, {0u, N, N, N}};
  hipLaunchKernelGGL((linear_rows_kernel<SWIGLU, false, false, MI, NJ, WR, WC, KS, ExpertTerm>), grid, block, 0, s, (const uint16_t*)x,
                     (const u32x4*)w, (const u32x4*)w2, (const uint16_t*)nullptr, dst, 0u, K, NT, 0u, T);
}

template <bool SWIGLU>
void launch_products(const void* x, const void* w, const void* w2, void* out, float* sums, const int32_t* plan, uint32_t rows, uint32_t k,
                     uint32_t E, uint32_t K, uint32_t N, hipStream_t s) {
  const ExpertPlan P = ExpertPlan::of(rows, k, E);
  const ExpertForm form = expert_form(P.pairs, E, K, N, SWIGLU);
  const uint32_t list = form;
  const ExpertTerm T = {(const uint4*)(plan + P.list[list]), (const uint32_t*)(plan + P.n_tiles + list), plan + P.order,
                        ExpertPlan::most_tiles(P.pairs, E, kPlanRows[list]), P.pairs, SWIGLU ? k : 1u, E, (size_t)N * K / 8, sums};
  switch (form) {
    case kFew: {
      constexpr int FT = few_features(SWIGLU), WAVES = 4, U = 8;
      const dim3 grid((unsigned)form_groups(kFew, P.pairs, E, N, SWIGLU));
      hipLaunchKernelGGL((expert_few_kernel<SWIGLU, WAVES, U, FT>), grid, dim3(64 * WAVES), 0, s, (const uint16_t*)x, (const u32x4*)w,
                         (const u32x4*)w2, (uint16_t*)out, K, N, T);
      return;
    }
    case kRows64: return launch_rows_of<SWIGLU, 2, 4, 2, 2, 1>(x, w, w2, out, K, N, T, s);
    case kRows128: return launch_rows_of<SWIGLU, 4, 4, 2, 4, 1>(x, w, w2, out, K, N, T, s);
    case kRows256: return launch_rows_of<SWIGLU, 8, 4, 2, 4, 1>(x, w, w2, out, K, N, T, s);
  }
}

}  // namespace

}  // namespace bct

using namespace bct;

extern "C" {

bct_status bctm_expert_swiglu(const void* x, const void* w_gate, const void* w_up, void* out, const void* plan, uint32_t rows,
                              uint32_t k, uint32_t n_experts, uint32_t K, uint32_t N, void* hip_stream) {
  const bct_status st = check_products(x, w_gate, out, plan, rows, k, n_experts, K, N, true);
  if (st != BCT_OK) return st;
  if (!w_up) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer or zero size");
  if (!al16(w_up)) return mfail(BCT_ERR_MISALIGNED, "pointers must be 16-byte aligned");
  launch_products<true>(x, w_gate, w_up, out, nullptr, (const int32_t*)plan, rows, k, n_experts, K, N, (hipStream_t)hip_stream);
  return launched("expert_swiglu");
}

bct_status bctm_expert_tile(uint32_t rows, uint32_t k, uint32_t n_experts, uint32_t K, uint32_t N, uint32_t swiglu, uint32_t* tile_rows,
                            uint32_t* tile_features) {
  if (!tile_rows || !tile_features || K == 0 || N == 0) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer or zero size");
  const bct_status st = check_plan_sizes(rows, k, n_experts);
  if (st != BCT_OK) return st;
  if (K % 32 != 0 || N % 16 != 0) return mfail(BCT_ERR_UNSUPPORTED, "K must be a multiple of 32 and N of 16");
  const ExpertForm form = expert_form(rows * k, n_experts, K, N, swiglu != 0);
  *tile_rows = kPlanRows[form];
  *tile_features = form_features(form, swiglu != 0);
  return BCT_OK;
}

bct_status bctm_expert_workspace(uint32_t rows, uint32_t k, uint32_t N, size_t* bytes) {
  if (!bytes || N == 0) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer or zero size");
  const bct_status st = check_plan_sizes(rows, k, k);
  if (st != BCT_OK) return st;
  if (N % 16 != 0 || N > 1u << 24) return mfail(BCT_ERR_UNSUPPORTED, "N must be a multiple of 16, at most 16777216");
  *bytes = (size_t)rows * k * N * 4;
  return BCT_OK;
}

bct_status bctm_expert_linear(const void* h, const void* w_packed, const void* plan, const float* weights, const void* residual, void* out,
                              void* workspace, size_t workspace_bytes, uint32_t rows, uint32_t k, uint32_t n_experts, uint32_t K,
                              uint32_t N, void* hip_stream) {
  const bct_status st = check_products(h, w_packed, out, plan, rows, k, n_experts, K, N, false);
  if (st != BCT_OK) return st;
  if (!weights || !workspace) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer or zero size");
  if (!al16(residual) || !al16(workspace) || ((uintptr_t)weights & 3u)) return mfail(BCT_ERR_MISALIGNED, "pointers must be 16-byte aligned, weights to 4");
  size_t need = 0;
  bctm_expert_workspace(rows, k, N, &need);
  if (workspace_bytes < need) return mfail(BCT_ERR_BUFFER_TOO_SMALL, "the workspace is smaller than bctm_expert_workspace says");
  hipStream_t s = (hipStream_t)hip_stream;
  const ExpertPlan P = ExpertPlan::of(rows, k, n_experts);
  launch_products<false>(h, w_packed, nullptr, nullptr, (float*)workspace, (const int32_t*)plan, rows, k, n_experts, K, N, s);
  const auto combine = k <= 2 ? combine_kernel<2> : k <= 4 ? combine_kernel<4> : combine_kernel<8>;
  hipLaunchKernelGGL(combine, dim3((unsigned)(((uint64_t)rows * (N / 8) + 255) / 256)), dim3(256), 0, s, (const float*)workspace,
                     (const int32_t*)plan + P.expert, weights, (const uint16_t*)residual, (uint16_t*)out, rows, k, N);
  return launched("expert_linear");
}

}  // extern "C"
