// What the projection kernels' files share: the outputs of a projection and the tiled activation layout.
#ifndef BCT_LINEAR_H
#define BCT_LINEAR_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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

// Whether a kernel's terms have one of a type, and that one.
template <typename T, typename... TERM>
constexpr bool kHas = (std::is_same<T, TERM>::value || ... || false);
template <typename T>
__device__ __forceinline__ const T& only(const T& term) {
  return term;
}

// The activations of bctm_linear_act, in fp32; act is a value of BCTM_ACT_, the same in every lane.  One branch for all values of a
// call, and few instructions in each: they stand in an epilogue once for every row tile of a wavefront, and with a switch for each value and
// erfc in it that epilogue did not fit the instruction cache.  4096 x 4096 x 11008 without activation 256 us, in this form with silu or gelu_tanh 277, gelu 272, relu
// 260; in that one 327 to 349.
template <int N>
__device__ __forceinline__ void activate(uint32_t act, float (&y)[N]) {
  if (act == 0) return;
  if (act == 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = y[i] < 0.f ? 0.f : y[i];   // a NaN stays one
  } else if (act == 3) {
    // y Phi(y).  Phi's tail by the rational approximation 7.1.26 of Abramowitz and Stegun's Handbook, within 0.75e-7: with t =
    // 1 / (1 + p |y| / sqrt 2), t (a1 + t (a2 + ..)) exp(-y^2 / 2) / 2.  Of itself the tail is off by 2e-4 at most down to y = -3.5, 9e-4 to -4.5
    // and 4e-3, half a step of bf16, to -6, where the result is -6e-9.
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float v = y[i], t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f * 0.70710678f, fabsf(v), 1.f));
      float p = __builtin_fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
      p = __builtin_fmaf(t, p, 0.5f * 1.421413741f);
      p = __builtin_fmaf(t, p, 0.5f * -0.284496736f);
      p = __builtin_fmaf(t, p, 0.5f * 0.254829592f);
      const float below = fminf(fabsf(v), 1e4f) * (t * p * __expf(-0.5f * v * v));   // 0 from |v| = 16 on, infinities too
      y[i] = v < 0.f ? -below : v - below;
    }
  } else {
    // silu, gelu_tanh and sigmoid: y or 1, over 1 + exp(-z), z = y, sqrt(8 / pi) (y + 0.044715 y^3) (as (1 + tanh u) / 2 = 1 / (1 + exp(-2 u)))
    // or y
    const float c1 = act == 4 ? -1.5957691f : -1.f, c3 = act == 4 ? -1.5957691f * 0.044715f : 0.f;
    const bool one = act == 5;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float v = y[i], z = act == 4 ? v * __builtin_fmaf(c3, v * v, c1) : v * c1;
      y[i] = (one ? 1.f : v) * __builtin_amdgcn_rcpf(1.f + __expf(z));
    }
  }
}
// Bias and activation of a projection's outputs (before its residual), bf16 or fp32 outputs.
struct EpilogueTerm {
  const uint16_t* bias;   // bf16 [N] or null
  uint32_t act, out32;
  __device__ __forceinline__ float bias_of(uint32_t n) const { return bias ? __uint_as_float((uint32_t)bias[n] << 16) : 0.f; }
  // eight features from n on, a multiple of 8
  __device__ __forceinline__ void apply(float (&y)[8], uint32_t n) const {
    if (bias) {
      float b[8];
      unpack16<BF16>(*(const u32x4*)(bias + n), b);
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] += b[k];
    }
    activate(act, y);
  }
};

// The low-rank term of a projection's rows (bct_lora.hip): out[r] += t[r] B_a^T, a = adapter[r].
// t, for the streaming kernel: fp32 [parts][rows][width], the parts to be added up, column segment * rank + j: the rank-j input
// of output `segment` (of the gate and up matrices in a SwiGLU).
// op, for the matrix-core kernel: pairs of A operands of v_mfma_f32_16x16x32_bf16, 16 rows x 16 ranks as four bf16 addends side by
// side in two contractions (entries 0-15 and 16-31 of each), whose sum is t to its last bit; pair number
// (row / 16 * segments + segment) * (rank / 16) + j / 16.
// b: per adapter 16-byte chunks of 8 ranks of one feature, chunk (feature / 16 * rank / 8 + j / 8) * 16 + feature % 16.
struct LoraTerm {
  const float* t;
  const u32x4 *op, *b, *b2;
  const int32_t* adapter;
  uint32_t n, rank, width, parts, segments;
};

// The adapter of a row: n for none, which is also that of rows past the end.
__device__ __forceinline__ uint32_t adapter_of(const int32_t* adapter, uint32_t row, uint32_t rows, uint32_t n) {
  uint32_t id = (uint32_t)adapter[min(row, rows - 1)];   // a negative one is beyond n
  asm("" : "+v"(id));   // requested in any case: behind a branch, several of them would be waited for one by one
  return row < rows ? min(id, n) : n;
}
// The adapters that RT tiles of 16 rows have, one after the other: id is that of row 16 i + lane % 16, todo[i] the lanes whose
// adapter has not come yet.  next: the adapter of the first of them and all rows that have it.
template <int RT>
struct AdapterWalk {
  uint32_t id[RT];
  uint64_t todo[RT], match[RT];
  uint32_t cur;
  __device__ __forceinline__ AdapterWalk(const int32_t* adapter, uint32_t row0, uint32_t rows, uint32_t n) {
#pragma unroll
    for (int i = 0; i < RT; ++i) id[i] = adapter_of(adapter, row0 + 16 * i + threadIdx.x % 16, rows, n);
#pragma unroll
    for (int i = 0; i < RT; ++i) todo[i] = __ballot(id[i] < n);
  }
  __device__ __forceinline__ bool next() {
    bool any = false;
#pragma unroll
    for (int i = RT - 1; i >= 0; --i)
      if (todo[i]) {
        cur = __builtin_amdgcn_readlane(id[i], (int)__builtin_ctzll(todo[i]));
        any = true;
      }
    if (!any) return false;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      match[i] = __ballot(id[i] == cur);
      todo[i] &= ~match[i];
    }
    return true;
  }
};

// The wavefront's part of a term, operands and accumulators in the lane layout of v_mfma_f32_16x16x32_bf16: CT tiles of 16
// features; MATS = 2: those of two matrices in turn (j % 2), each a column segment of t, else segment(j); tile(j): the feature
// tile; N: all features.
template <int CT, int MATS, typename SEG, typename TILE>
struct LoraTiles {
  const LoraTerm& L;
  uint32_t N;
  SEG segment;
  TILE tile;
  static constexpr int kSets = MATS;   // operands of t for a row tile and 16 ranks
  // a product takes 16 ranks: all addends of t meet the same weights
  __device__ __forceinline__ void weights(uint32_t adapter, uint32_t ks, bf16x8 (&b)[CT]) const {
    const size_t at = ((size_t)adapter * (N / 16) * (L.rank / 8) + 2 * ks) * 16 + threadIdx.x / 16 % 2 * 16 + threadIdx.x % 16;
#pragma unroll
    for (int j = 0; j < CT; ++j)
      b[j] = __builtin_bit_cast(bf16x8, (MATS == 2 && j % 2 ? L.b2 : L.b)[at + (size_t)tile(j) * (L.rank / 8) * 16]);
  }
  __device__ __forceinline__ void operand(uint32_t row_tile, uint32_t seg, uint32_t ks, bf16x8 (&a)[2]) const {
    const u32x4* op = L.op + (((size_t)row_tile * L.segments + seg) * (L.rank / 16) + ks) * 128 + threadIdx.x % 64;
    a[0] = __builtin_bit_cast(bf16x8, op[0]);
    a[1] = __builtin_bit_cast(bf16x8, op[64]);
  }
  static __device__ __forceinline__ f32x4 product(const bf16x8 (&a)[2], bf16x8 b, f32x4 sum) {
    sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[0], b, sum, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[1], b, sum, 0, 0, 0);
  }
};

// Adds the term of RT tiles of 16 rows (from row0) to the accumulators acc(i, j), which are those of the K loop and hold nothing
// else yet.  Each row's sum is one chain over its own adapter's ranks in their order, whether its tile has one adapter or several,
// so its bits do not depend on its neighbours: a matrix instruction sums every row apart, and where a tile's rows have
// several adapters, its result is selected for the rows of the one that was multiplied.  Selected, not multiplied by zero, so
// an infinity or a NaN in one adapter's weights stays in its rows.
template <int RT, int CT, int MATS, typename SEG, typename TILE, typename ACC>
__device__ __forceinline__ void lora_add(const LoraTiles<CT, MATS, SEG, TILE>& T, uint32_t row0, uint32_t rows, ACC acc) {
  const uint32_t last = (rows - 1) / 16, n = T.L.n, steps = T.L.rank / 16;
  uint32_t id[RT], cur[RT], mixed = 0;
#pragma unroll
  for (int i = 0; i < RT; ++i) id[i] = adapter_of(T.L.adapter, row0 + 16 * i + threadIdx.x % 16, rows, n);
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    cur[i] = __builtin_amdgcn_readfirstlane(id[i]);
    if (__ballot(id[i] == cur[i]) != ~0ull) {
      cur[i] = n;
      mixed |= 1u << i;
    }
  }
  // the row tiles whose rows all have one adapter
  for (uint32_t ks = 0; ks < steps; ++ks) {
    // row tiles whose operands are requested at once: as many as there are registers for beside 32 accumulators
    constexpr int AT_ONCE = RT * CT > 16 ? 16 / CT : 8, WANT = AT_ONCE / (2 * MATS), G = WANT < 1 ? 1 : WANT < RT ? WANT : RT;
    bf16x8 a[G][MATS][2], b[CT];
#pragma unroll
    for (int i0 = 0; i0 < RT; i0 += G) {
      // a row tile past the end or without an adapter takes an operand that is there, and no product
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int m = 0; m < MATS; ++m) T.operand(min(row0 / 16 + i0 + g, last), MATS == 2 ? m : T.segment(0), ks, a[g][m]);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int i = i0 + g;
        if (cur[i] >= n) continue;
        if (i == 0 || cur[i] != cur[i - (i > 0)]) T.weights(cur[i], ks, b);
#pragma unroll
        for (int j = 0; j < CT; ++j) {
          // where the border between two outputs lies within the tiles
          if (MATS == 1 && j > 0 && T.segment(j) != T.segment(j - 1)) T.operand(row0 / 16 + i, T.segment(j), ks, a[g][0]);
          acc(i, j) = T.product(a[g][j % MATS], b[j], acc(i, j));
        }
      }
    }
  }
  // Those with several, or with rows without one: adapter after adapter, the next product's operands requested before this one
  // (with eight feature tiles there are no registers for them).
  constexpr bool AHEAD = CT <= 4;
  const uint32_t kg = threadIdx.x % 64 / 16;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    if (!(mixed >> i & 1)) continue;
    const uint32_t row_tile = row0 / 16 + i;
    AdapterWalk<1> walk(T.L.adapter, 16 * row_tile, rows, n);
    uint32_t ks = 0;
    bf16x8 a[MATS][2], b[CT];
    auto request = [&](bf16x8 (&to_a)[MATS][2], bf16x8 (&to_b)[CT]) {
      T.weights(walk.cur, ks, to_b);
#pragma unroll
      for (int m = 0; m < MATS; ++m) T.operand(row_tile, MATS == 2 ? m : T.segment(0), ks, to_a[m]);
    };
    bool more = walk.next();   // one at least has an adapter
    if (AHEAD) request(a, b);
    while (more) {
      if (!AHEAD) request(a, b);
      const uint32_t mine = (uint32_t)(walk.match[0] >> (4 * kg)), now = ks;   // bit v: row 4 kg + v
      if (++ks == steps) {
        ks = 0;
        more = walk.next();   // no more: the last one's first operands once again
      }
      bf16x8 next_a[MATS][2], next_b[CT];
      if (AHEAD) {
        request(next_a, next_b);
        // Before the products, which the compiler sees to by itself in a SwiGLU only.  us, without | with: 256 x 4096 x 12288, 256 adapters of
        // rank 16 68.5 | 62.2, 512 rows of 64 106 | 93.7, SwiGLU of 256 x 4096 x 11008 of 64 87.2 | 94.3.
        if (MATS == 1) __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        if (MATS == 1 && j > 0 && T.segment(j) != T.segment(j - 1)) T.operand(row_tile, T.segment(j), now, a[0]);
        const f32x4 d = T.product(a[j % MATS], b[j], acc(i, j));
#pragma unroll
        for (int v = 0; v < 4; ++v) acc(i, j)[v] = (mine >> v & 1) ? d[v] : acc(i, j)[v];
      }
      if (AHEAD) {
#pragma unroll
        for (int m = 0; m < 2 * MATS; ++m) a[m / 2][m % 2] = next_a[m / 2][m % 2];
#pragma unroll
        for (int j = 0; j < CT; ++j) b[j] = next_b[j];
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

// The same with bias and activation (bct_linear_act.hip).
hipError_t launch_linear_rows_act(const void* x, const void* w, const void* residual, const LinearOut& dst, uint32_t rows,
                                  uint32_t K, uint32_t N, bool x_tiled, bool out_tiled, hipStream_t s, const EpilogueTerm& term);
// Few features: workgroups of 16 * row_tiles rows (1 or 2) and 64 features, K in eight parts; N a multiple of 64.
hipError_t launch_linear_narrow(const void* x, const void* w, const void* residual, void* out, uint32_t rows, uint32_t K, uint32_t N,
                                bool x_tiled, bool out_tiled, hipStream_t s, const EpilogueTerm& term, uint32_t row_tiles);

}  // namespace bct

#endif
