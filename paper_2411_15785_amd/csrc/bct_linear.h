// What the projection kernels' files share: the outputs of a projection and the tiled activation layout.
#ifndef BCT_LINEAR_H
#define BCT_LINEAR_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bct_device.h"

namespace bct {

// Up to three row-major outputs side by side along N: output i takes the features [start[i], start[i + 1]).
struct LinearOut {
  uint16_t* ptr[3];
  uint32_t start[4];
};

// Tiled activations: rows in groups of 32, inputs in groups of 32; group (r / 32, k / 32) is 2 KB, two A
// operands of v_mfma_f32_16x16x32_bf16 (rows 0-15 and 16-31 of the group), each 64 lanes x 16 bytes with
// lane 16 * ((k % 32) / 8) + r % 16 holding the inputs k % 8 = 0..7.  Returns the 16-byte chunk index.
__device__ __forceinline__ size_t tiled_chunk(uint32_t r, uint32_t k, uint32_t K) {
  return ((((size_t)(r / 32) * (K / 32) + k / 32) * 2 + (r % 32) / 16) * 64) + 16 * ((k % 32) / 8) + r % 16;
}

// The low-rank term of a projection's rows (bct_lora.hip): out[r] += t[r] B_a^T, a = adapter[r].  t is fp32 [parts][rows][width],
// the parts to be added up, column segment * rank + j: the rank-j input of output `segment` (of the gate and up matrices in a
// SwiGLU).  b: per adapter 16-byte chunks of 8 ranks of one feature, chunk (feature / 16 * rank / 8 + j / 8) * 16 + feature % 16.
struct LoraTerm {
  const float* t;
  const u32x4 *b, *b2;
  const int32_t* adapter;
  uint32_t n, rank, width, parts, segments;
};

// The rows of an adapter a row tile has, one adapter after the other in ascending order: ids of the tiles' rows, one a lane of
// 16 (n from a row without one); the least id from `from` on, n if there is none.
template <int RT>
__device__ __forceinline__ uint32_t next_adapter(const uint32_t* id, uint32_t from, uint32_t n) {
  uint32_t m = n;
#pragma unroll
  for (int i = 0; i < RT; ++i) m = min(m, id[i] >= from ? id[i] : n);
#pragma unroll
  for (int o = 1; o < 16; o *= 2) m = min(m, (uint32_t)__shfl_xor(m, o, 64));
  return __builtin_amdgcn_readfirstlane(m);
}
__device__ __forceinline__ uint32_t adapter_of(const int32_t* adapter, uint32_t row, uint32_t rows, uint32_t n) {
  const uint32_t id = (uint32_t)adapter[min(row, rows - 1)];   // a negative one is beyond n
  return row < rows ? min(id, n) : n;
}

// Adds the term to RT row tiles (of 16, from row0) x CT tiles of 16 features whose accumulators are acc(i, j), lane layout of
// v_mfma_f32_16x16x32_bf16.  MATS = 2: the tiles of two matrices in turn (j % 2), each a column segment of t; else segment(j).
// tile(j): the feature tile.  A product takes 16 ranks: t goes in as two bf16 addends side by side in the contraction, its
// rounding in entries 0-15 and what that left in 16-31, both against the same B, so 16 bits of t count.  The wavefronts share
// the work by adapter and rank.  The products of a row tile are selected by row, not multiplied by zero, for rows of other
// adapters or of none: an infinity or a NaN in one adapter's weights stays in its rows.
template <int RT, int CT, int MATS, typename SEG, typename TILE, typename ACC>
__device__ __forceinline__ void lora_add(const LoraTerm& L, uint32_t row0, uint32_t rows, uint32_t N, uint32_t share, uint32_t shares,
                                         SEG segment, TILE tile, ACC acc) {
  const uint32_t lane = threadIdx.x % 64, jl = lane % 16, kg = lane / 16, half = kg % 2;
  uint32_t id[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) id[i] = adapter_of(L.adapter, row0 + 16 * i + jl, rows, L.n);
  uint32_t turn = 0;
  for (uint32_t cur = next_adapter<RT>(id, 0, L.n); cur < L.n; cur = next_adapter<RT>(id, cur + 1, L.n)) {
    const size_t mat0 = (size_t)cur * (N / 16) * (L.rank / 8) * 16;
    for (uint32_t ks = 0; ks < L.rank / 16; ++ks) {
      if (turn++ % shares != share) continue;
      u32x4 b[CT];
#pragma unroll
      for (int j = 0; j < CT; ++j)
        b[j] = (MATS == 2 && j % 2 ? L.b2 : L.b)[mat0 + ((size_t)tile(j) * (L.rank / 8) + 2 * ks + half) * 16 + jl];
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        __builtin_amdgcn_sched_barrier(0);   // one row tile after the other: their operands need not be there at once
        const uint64_t match = __ballot(id[i] == cur);
        if (match == 0) continue;
        const uint32_t mine = (uint32_t)(match >> (4 * kg));   // bit v: row 4 kg + v of the tile
        const float* row = L.t + (size_t)min(row0 + 16 * i + jl, rows - 1) * L.width + 16 * ks + 8 * half;
        auto operand = [&](uint32_t seg) -> bf16x8 {
          const float* t = row + seg * L.rank;
          f32x4 lo = *(const f32x4*)t, hi = *(const f32x4*)(t + 4);
          for (uint32_t p = 1; p < L.parts; ++p) {
            t += (size_t)rows * L.width;
            lo += *(const f32x4*)t;
            hi += *(const f32x4*)(t + 4);
          }
          u32x4 a;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = e < 2 ? lo[2 * e] : hi[2 * e - 4], y = e < 2 ? lo[2 * e + 1] : hi[2 * e - 3];
            const uint32_t r = pack_bf16x2(x, y);
            a[e] = kg < 2 ? r : pack_bf16x2(x - __uint_as_float(r << 16), y - __uint_as_float(r & 0xFFFF0000u));
          }
          return __builtin_bit_cast(bf16x8, a);
        };
        auto product = [&](bf16x8 a, int j, uint32_t take) {
          const f32x4 d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, b[j]), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
          for (int v = 0; v < 4; ++v) acc(i, j)[v] = (take >> v & 1) ? acc(i, j)[v] + d[v] : acc(i, j)[v];
        };
        if constexpr (MATS == 2) {
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const bf16x8 a = operand(m);
#pragma unroll
            for (int j = m; j < CT; j += 2) product(a, j, mine);
          }
        } else {
          // one segment for all tiles, but where the border between two outputs lies within them
          for (uint32_t seg = segment(0); seg <= segment(CT - 1); ++seg) {
            const bf16x8 a = operand(seg);
#pragma unroll
            for (int j = 0; j < CT; ++j) product(a, j, segment(j) == seg ? mine : 0u);
          }
        }
      }
    }
  }
}

// What a projection launch gives each workgroup: rows x features (SwiGLU: of the product), and in how many parts K is
// summed (each a chain of its own, the parts added in order).
struct LinearTile {
  uint32_t rows, features, k_parts;
};

// The tile of launch_linear_rows for a shape: host logic, what that launch itself goes by.
LinearTile linear_rows_tile(uint32_t rows, uint32_t K, uint32_t N, bool swiglu, bool x_tiled);

// The matrix-core projection of many rows (bct_linear_rows.hip).  w2 non-null: SwiGLU of w and w2.  x_tiled /
// out_tiled: activations in the tiled order.  N is a multiple of 16 (out_tiled: 32), K of 32.
hipError_t launch_linear_rows(const void* x, const void* w, const void* w2, const void* residual, const LinearOut& dst,
                              uint32_t rows, uint32_t K, uint32_t N, bool x_tiled, bool out_tiled, hipStream_t s,
                              const LoraTerm* lora = nullptr);

}  // namespace bct

#endif
