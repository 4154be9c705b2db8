// The projections of the decoder stack for MANY token rows (a prompt chunk: batch x T rows; gfx950), where the
// product is a dense contraction bound by the matrix cores and no longer by streaming the weights.
//
// Both operands are already stored in MFMA operand order (packed weights, tiled activations), so a K step of 32
// inputs is a set of 1 KB tiles that go from memory to LDS unchanged (global_load_lds: 16 bytes per lane, no
// trip through registers) and are read back by the wavefronts as v_mfma_f32_16x16x32_bf16 operands with linear
// 16-byte LDS reads (no bank conflicts).  Row-major activations take the same path with one row of 64 bytes
// per 16 lanes.
//
// What bounds it: the matrix cores, once loads and LDS reads are out of their way.  Three things do that:
//   - four LDS stages, so that a tile is requested three K steps before it is used.  A wavefront waits only for
//     its own requests of the next stage (vmcnt leaves the two later stages in flight); the barrier that
//     follows makes the stage the workgroup's.  Each stage is a __shared__ array of its own: the compiler
//     then knows that reading one stage does not depend on requests into another and adds no wait.
//   - two wavefronts per SIMD that take turns ("ping"): while one issues the K step's products, the other
//     reads its operands of the next one from LDS and requests tiles; two barriers per K step keep them
//     half a step apart, and s_setprio lets the products go first.
//   - workgroup ids mapped so that the workgroups resident on one XCD cover 4 row tiles x consecutive
//     feature tiles: each operand panel enters that XCD's L2 once per four uses.
// With one stage ahead held in registers, one barrier per K step and no turns, the same 256 x 256 tile took
// 1353 us at 16384 rows x 11008 -> 4096 (1.09 PFLOP/s); this form takes 955 us (1.55 PFLOP/s); four stages
// without turns 1131 us; bands of 8 instead of 4 row tiles 1033 us.
//
// Where 256 x 256 tiles are too few for 256 compute units, smaller tiles follow; and where even 128 x 128 tiles
// leave every compute unit at most one workgroup of four wavefronts, two groups of wavefronts share a
// tile, each with half of the inputs, and are the two that take turns on a SIMD (see rows_shape for the choice
// and the measurements).  128 x 512 fills rounds where 256 wastes rows.
#include "bct_linear_rows.h"

namespace bct {

// The tile of a shape.  It decides in how many parts K is summed as well, so a result's last bits depend on the
// row and feature counts (bctm_linear_tile tells).  The time of a launch is the number of rounds its workgroups take on 256 compute units
// times the K steps times what a step of a resident workgroup takes; measured us per K step at 640 and 16384
// rows, K = 11008 / 4096, one set of weights again and again, so out of the caches:
//   256 x 256             one workgroup per compute unit  0.46 (few) - 0.69 (chip full)
//   128 x 512             one                             0.80
//   128 x 256             one                             0.34 - 0.44
//   128 x 128             two of four wavefronts          0.26 alone on its compute unit, 0.46 for a pair
//   128 x 128, K in two   one                             0.19 - 0.25
//   128 x 64, K in two    one                             0.16
//   64 x 64, K in two     two                             0.11 alone, 0.19 for a pair
// so 256 x 256 wins where the chip is full (4 rounds of it against 16 of 128 x 128), the others where its
// workgroups are few: 640 rows x 11008 -> 4096 takes 157 us in 256 x 256, 117, 88, 67, 94 in the last four (with weights from
// memory, as a stack of layers has them, the 67 are 96).
// A compute unit gets 50 to 60 GB/s of operands then, however many stages are in flight (5 or 8 stages instead of 4:
// the same times), so the fewest bytes per compute unit win among the shapes that have one round of workgroups, and 128 x 64 is
// for where 64 x 64 would be pairs and 128 x 128 would leave compute units idle.  us, weights from memory, without | with it: 320
// rows, 11008 -> 4096 82.9 | 62.4, 4096 -> 4096 30.9 | 25.9, 5120 -> 5120 41.7 | 37.9; 384 85.2 | 70.4, 31.8 | 28.3, 42.4 | 36.3; 512
// 86.9 | 73.6, 33.5 | 29.8; 192, 2048 -> 6144 18.6 | 16.4; 1024, 2048 -> 2048 17.6 | 16.5; 700, 2048 -> 2048 15.3 | 15.6.
// 128 x 512 has the work of 256 x 256 and 5 / 4 of its loads; it is there for row counts that 256 wastes, where it saves
// a round of workgroups.  With weights from memory, us without | with it, tiled x: against 128 x 256 838 rows, 4096 -> 53248
// 367 | 326, 384, 8192 -> 37376 242 | 212; against 128 x 128 526, 4096 -> 66560 366 | 314, 319, 4096 -> 69632 239 | 216 (a predicted 2 %:
// the price of many pairs is low).  Against 256 x 256 it depends on K: up to 4096 885, 4096 -> 66560 426 | 414, 3690, 2048 ->
// 22528 280 | 269, 1057, 512 -> 68608 111 | 102 (44 shapes, 0.986 to 1.12 times as fast); from 5120 on a step of 256 x 256 takes 0.62 to
// 0.68, of 128 x 512 0.78 to 0.83, and where it saves one round of six or seven it loses: 1658, 8192 -> 24576 SwiGLU 1019 | 1070,
// 4654, 11008 -> 20992 1626 | 1676 (15 shapes, 0.95 to 1.015; on another card 0.96 to 1.0), hence 83 there, which leaves it one of
// five: 2135, 11008 -> 14592 SwiGLU 1103 | 1071 (7 shapes, 0.98 to 1.045).  A row-major x waits longer for its rows, and the wider
// tile wins in all 37 shapes: 4654, 11008 -> 20992 2105 | 1841, 1911, 1024 -> 50176 218 | 212.
// A count of columns that 128 does not divide leaves the last tile of every row of tiles partly used, in any shape: all of them
// are open to it, at what their whole tiles cost.
RowsShape rows_shape(uint32_t rows, uint32_t bcols, uint32_t K, bool x_tiled) {
  auto tiles = [&](uint32_t bm, uint32_t bn) { return (uint64_t)((rows + bm - 1) / bm) * ((bcols + bn - 1) / bn); };
  // hundredths of a us per K step: one workgroup per compute unit at a time; two, a last one may have it alone
  auto one = [](uint64_t t, uint64_t cost) { return (t + 255) / 256 * cost; };
  auto two = [](uint64_t t, uint64_t alone, uint64_t pair) {
    const uint64_t rem = t % 512;
    return t / 512 * pair + (rem > 256 ? pair : rem ? alone : 0);
  };
  RowsShape best = kTile128;
  uint64_t cost = two(tiles(128, 128), 26, 46);
  auto take = [&](RowsShape s, uint64_t c) {
    if (c < cost) {
      cost = c;
      best = s;
    }
  };
  take(kTile128K2, one(tiles(128, 128), 25));
  take(kTile128x64K2, one(tiles(128, 64), 16));
  take(kTile64K2, two(tiles(64, 64), 11, 19));
  const bool ragged = bcols % 128 != 0;
  if (bcols % 256 == 0 || ragged) {
    take(kTile128x256, one(tiles(128, 256), 44));
    take(kTile256, one(tiles(256, 256), 69));
  }
  // (dear only against 256 x 256, which sums K in one part as well: the parts do not depend on x's order)
  if (bcols % 512 == 0 || ragged) take(kTile128x512, one(tiles(128, 512), best == kTile256 && x_tiled && K > 4096 ? 83 : 80));
  return best;
}

LinearTile linear_rows_tile(uint32_t rows, uint32_t K, uint32_t N, bool swiglu, bool x_tiled) {
  const uint32_t per = swiglu ? 2 : 1;   // B columns of a feature
  switch (rows_shape(rows, per * N, K, x_tiled)) {
    case kTile256: return {256, 256 / per, 1};
    case kTile128x512: return {128, 512 / per, 1};
    case kTile128x256: return {128, 256 / per, 1};
    case kTile128: return {128, 128 / per, 1};
    case kTile128K2: return {128, 128 / per, 2};
    case kTile128x64K2: return {128, 64 / per, 2};
    case kTile64K2: return {64, 64 / per, 2};
  }
  return {0, 0, 0};
}

hipError_t launch_linear_rows(const void* x, const void* w, const void* w2, const void* residual, const LinearOut& dst,
                              uint32_t rows, uint32_t K, uint32_t N, bool x_tiled, bool out_tiled, hipStream_t s,
                              const LoraTerm* lora) {
  auto launch = [&](auto... term) {
    if (w2) {
      if (x_tiled) launch_rows<true, true>(x, w, w2, residual, dst, rows, K, N, out_tiled, s, term...);
      else launch_rows<true, false>(x, w, w2, residual, dst, rows, K, N, out_tiled, s, term...);
    } else {
      if (x_tiled) launch_rows<false, true>(x, w, w2, residual, dst, rows, K, N, out_tiled, s, term...);
      else launch_rows<false, false>(x, w, w2, residual, dst, rows, K, N, out_tiled, s, term...);
    }
  };
  if (lora) launch(*lora);
  else launch();
  return hipGetLastError();
}

}  // namespace bct
