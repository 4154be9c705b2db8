// Tokens by expert: the plan that bctm_route leaves and the expert products go by.
#ifndef BCT_EXPERTS_H
#define BCT_EXPERTS_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/bct_model.h"
#include "bct_device.h"

namespace bct {

constexpr uint32_t kMaxExperts = 512, kMaxPerToken = 16;

// Row tiles of the expert products: an expert's rows in tiles of kPlanRows[i], each expert's last one partly used.
constexpr uint32_t kTileLists = 4, kPlanRows[kTileLists] = {16, 64, 128, 256};

// A plan in memory, int32 unless said otherwise; a pair is token * k + slot.
//   offsets   [E + 1]      where each expert's pairs begin in `order`; the last one: how many pairs have an expert
//   order     [pairs]      the pairs by expert, equal ones by number; those without an expert last
//   expert    [pairs]      1 + each pair's expert, 0 for none: a plan of zeros has no tokens
//   n_tiles   [kTileLists]
//   lists     uint4        per row tile: expert, where its pairs begin in `order`, how many it has, which of its tiles this is
//   counts    [blocks][E + 1, filled up to a multiple of 4]  how many pairs of each expert a block of tokens has (while the plan is made)
struct ExpertPlan {
  uint32_t pairs, E, blocks;
  size_t order, expert, n_tiles, list[kTileLists], counts, ints;   // in ints from the plan's begin
  __host__ __device__ static uint32_t most_tiles(uint32_t pairs, uint32_t E, uint32_t rows) {
    const uint32_t some = pairs < E ? pairs : E;
    return pairs / rows + some;   // every whole tile has `rows` pairs, every expert one that is not whole
  }
  __host__ __device__ static ExpertPlan of(uint32_t rows, uint32_t k, uint32_t E) {
    ExpertPlan p;
    p.pairs = rows * k;
    p.E = E;
    // One block is one launch, several are two; but a compute unit takes long over many tokens of many experts.  us in a graph, all in one | 64 | 16
    // | 4 tokens a block, 8 of 64 experts: 32 tokens 10.8 | - | 12.7 | -, 128 15.7 | 13.9 | 12.7 | 12.7, 1024 - | 14.1 | 13.1 | 14.2; 8 of 256 with a
    // bias: 32 24.2 | - | 20.6 | 17.6, 64 32.6 | - | 20.1 | 17.7, 1024 - | 31.4 | 21.4 | 23.5.
    p.blocks = rows <= 64 && rows * E <= 4096 ? 1 : (rows + 15) / 16;
    if (p.blocks > kMostBlocks) p.blocks = kMostBlocks;
    size_t at = (E + 4) / 4 * 4;
    auto take = [&](size_t n) {
      const size_t from = at;
      at += (n + 3) / 4 * 4;
      return from;
    };
    p.order = take(p.pairs);
    p.expert = take(p.pairs);
    p.n_tiles = take(kTileLists);
    for (uint32_t i = 0; i < kTileLists; ++i) p.list[i] = take(4 * (size_t)most_tiles(p.pairs, E, kPlanRows[i]));
    p.counts = take(p.blocks > 1 ? (size_t)p.blocks * ((E + 4) / 4 * 4) : 0);
    p.ints = at;
    return p;
  }
  // tokens of a block, the last one may have fewer
  __host__ __device__ uint32_t block_rows(uint32_t rows) const { return (rows + blocks - 1) / blocks; }
  static constexpr uint32_t kMostBlocks = 256;
};

// The checks of a plan's sizes and pointer.
bct_status check_plan_sizes(uint32_t rows, uint32_t k, uint32_t E);
bct_status check_expert_plan(const void* plan, uint32_t rows, uint32_t k, uint32_t E);

// What the matrix-core kernel needs of a plan: its rows are pairs, `per_row` of them share a row of x.
struct ExpertTerm {
  const uint4* tiles;
  const uint32_t* n_tiles;
  const int32_t* order;
  uint32_t most_tiles, pairs, per_row, n_experts;
  size_t stride;   // 16-byte chunks of one expert's matrix
  void* sums;      // outputs of the plain product, [pairs][N]: blocks of eight (pack_block), from the streaming kernel fp32
};

// Eight sums in 16 bytes: whole numbers of 15 bits, multiples of a power of two that they share, each in the upper bits of a
// half word; the lowest bits of the eight are that power's exponent, word w has its bits w and w + 4.  Between the products of the way back
// and their weighted sum, halves a pass over memory and back that is a third of the call with fp32 (4096 tokens of 8 experts, 1376 ->
// 4096).  A number is off by at most 2^-14 of the largest of its eight (which is 2^13 steps at least, as long as a step is not below
// 2^-126), where the bf16 result is rounded to 2^-9 of itself.  NaN and the infinities have numbers of their own, so their
// neighbours are as exact as others.
constexpr int kBlockMost = 16382, kBlockInf = 16383, kBlockNan = -16384, kBlockLeast = 14;
__device__ __forceinline__ uint32_t block_bits(uint32_t e, int w) { return (e | e << 12) >> w & 0x00010001u; }
// The largest magnitude below 2^(e - 126) / (1 + 2^-12), so times 2^(140 - e) it is below kBlockMost, and 2^13 (1 - 2^-12) at least.
__device__ __forceinline__ uint32_t block_exponent(float top) {
  return max(__float_as_uint(top * (1.f + 1.f / 4096)) >> 23, (uint32_t)kBlockLeast);
}
// lds: the same eight, for those that are not all numbers: a loop, so that this, which stands in an epilogue many times, stays short.
__device__ __forceinline__ u32x4 pack_block(const float (&y)[8], const float* lds) {
  float top = 0.f;
  bool number = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(y[i]));
#pragma unroll
  for (int i = 0; i < 8; ++i) number = number && y[i] == y[i];   // fmaxf passes over a NaN
  u32x4 v;
  if (number && top < INFINITY) {
    const uint32_t e = block_exponent(top);
    const float scale = __uint_as_float((140 + 127 - e) << 23);   // 2^(140 - e)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      // 1.5 2^23 + q has q in its lower bits, rounded to the nearest by the addition
      const uint32_t lo = __float_as_uint(__builtin_fmaf(y[2 * w], scale, 12582912.f)), hi = __float_as_uint(__builtin_fmaf(y[2 * w + 1], scale, 12582912.f));
      v[w] = (__builtin_amdgcn_perm(hi, lo, 0x05040100u) << 1 & 0xFFFEFFFEu) | block_bits(e, w);
    }
    return v;
  }
  top = 0.f;
#pragma unroll 1
  for (int i = 0; i < 8; ++i) top = fabsf(lds[i]) < INFINITY ? fmaxf(top, fabsf(lds[i])) : top;
  const uint32_t e = block_exponent(top);
  unsigned long long low = 0, high = 0;
#pragma unroll 1
  for (int i = 7; i >= 0; --i) {
    const float f = lds[i];
    const int q = f != f ? kBlockNan : f == INFINITY ? kBlockInf : f == -INFINITY ? -kBlockInf : (int)rintf(__builtin_amdgcn_ldexpf(f, 140 - (int)e));
    high = high << 16 | low >> 48;
    low = low << 16 | ((uint32_t)q << 1 & 0xFFFEu);
  }
  v = u32x4{(uint32_t)low, (uint32_t)(low >> 32), (uint32_t)high, (uint32_t)(high >> 32)};
#pragma unroll
  for (int w = 0; w < 4; ++w) v[w] |= block_bits(e, w);
  return v;
}
// y += weight * the block's sums.
__device__ __forceinline__ void add_block(const u32x4 v, float weight, float (&y)[8]) {
  uint32_t x = 0;
  int q[8], most = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    x |= (v[w] & 0x00010001u) << w;
    q[2 * w] = (int)(v[w] << 16) >> 17;
    q[2 * w + 1] = (int)v[w] >> 17;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, max(q[i], -q[i]));
  const int e = (int)((x | x >> 12) & 0xFFu);
  const float scale = __builtin_amdgcn_ldexpf(1.f, e - 140);
  if (most <= kBlockMost) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __builtin_fmaf(weight, (float)q[i] * scale, y[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      y[i] = __builtin_fmaf(weight, q[i] == kBlockNan ? __builtin_nanf("") : q[i] == kBlockInf ? INFINITY : q[i] == -kBlockInf ? -INFINITY : (float)q[i] * scale, y[i]);
  }
}

// An expert by one of its row tiles.  One of no pairs where the plan holds something else than a tile for these sizes: no read leaves the
// buffers by it.
struct ExpertTile {
  uint32_t expert, begin, pairs, tile;
};
__device__ __forceinline__ ExpertTile expert_tile(const ExpertTerm& T, uint32_t i) {
  const uint4 t = T.tiles[i];
  const bool good = t.x < T.n_experts && t.y < T.pairs && t.z <= T.pairs - t.y && t.w <= i;
  return {good ? t.x : 0u, good ? t.y : 0u, good ? t.z : 0u, good ? t.w : 0u};
}
__device__ __forceinline__ uint32_t expert_pair(const ExpertTerm& T, const int32_t* order, uint32_t row) {
  return min((uint32_t)order[row], T.pairs - 1);
}

}  // namespace bct

#endif
