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
  float* sums;     // outputs of the plain product, [pairs][N]
};

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
