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
//   expert    [pairs]      each pair's expert, -1 for none
//   n_tiles   [kTileLists]
//   lists     uint4        per row tile: expert, first place in `order`, rows, 0
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
    p.blocks = rows <= kOneBlock ? 1 : (rows + kBlockRows - 1) / kBlockRows;
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
  static constexpr uint32_t kOneBlock = 64, kBlockRows = 64, kMostBlocks = 256;
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
// half word; the lowest bits of the eight are that power's exponent.  Between the products of the way back and their weighted
// sum, halves a pass over memory and back that is a third of the call with fp32 (4096 tokens of 8 experts, 1376 -> 4096).  A number is off by at
// most 2^-14 of the largest of its eight (which is 2^13 steps at least), where the bf16 result is rounded to 2^-9 of itself.  Sums below 2^-126 are 0; NaN
// and the infinities have numbers of their own, so their neighbours are as exact as others.
constexpr int kBlockMost = 16382, kBlockInf = 16383, kBlockNan = -16384;
__device__ __forceinline__ u32x4 pack_block(const float (&y)[8]) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(y[i]));   // of a NaN and a number, the number
  bool odd = false;
  if (!(top < INFINITY)) {
    odd = true;
    top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fabsf(y[i]) < INFINITY ? fmaxf(top, fabsf(y[i])) : top;
  }
  // the largest is below 2^(e - 126) / (1 + 2^-12), so times 2^(140 - e) below kBlockMost, and 2^13 (1 - 2^-12) at least
  const uint32_t e = __float_as_uint(top * (1.f + 1.f / 4096)) >> 23;
  const int shift = 140 - (int)e;
  u32x4 v;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t half[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = 2 * w + h;
      float f = __builtin_amdgcn_ldexpf(y[i], shift);
      int q = (int)rintf(__builtin_amdgcn_fmed3f(f, -(float)kBlockMost, (float)kBlockMost));
      if (odd || y[i] != y[i]) q = y[i] != y[i] ? kBlockNan : y[i] == INFINITY ? kBlockInf : y[i] == -INFINITY ? -kBlockInf : q;
      half[h] = ((uint32_t)q << 1 | (e >> i & 1)) & 0xFFFFu;
    }
    v[w] = half[0] | half[1] << 16;
  }
  return v;
}
__device__ __forceinline__ void unpack_block(const u32x4 v, float (&y)[8]) {
  uint32_t e = 0;
  int q[8], most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int half = i % 2 ? (int)v[i / 2] >> 16 : (int)(int16_t)v[i / 2];
    e |= (uint32_t)(half & 1) << i;
    q[i] = half >> 1;
    most = max(most, max(q[i], -q[i]));
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_ldexpf((float)q[i], (int)e - 140);
  if (most > kBlockMost) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = q[i] == kBlockNan ? __builtin_nanf("") : q[i] == kBlockInf ? INFINITY : q[i] == -kBlockInf ? -INFINITY : y[i];
  }
}

struct ExpertTile {
  uint32_t expert, first, rows;
};
// A tile of no rows where the plan holds something else than one for these sizes: no read leaves the buffers by it.
__device__ __forceinline__ ExpertTile expert_tile(const ExpertTerm& T, uint32_t i) {
  const uint4 t = T.tiles[i];
  const bool good = t.x < T.n_experts && t.y < T.pairs && t.z <= T.pairs - t.y;
  return {good ? t.x : 0u, good ? t.y : 0u, good ? t.z : 0u};
}
__device__ __forceinline__ uint32_t expert_pair(const ExpertTerm& T, const int32_t* order, uint32_t row) {
  return min((uint32_t)order[row], T.pairs - 1);
}

}  // namespace bct

#endif
