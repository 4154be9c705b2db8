// Low-rank adapters of many requests at once beside a shared projection (gfx950): row r of a batch belongs to a request with
// the adapter a = adapter[r], and
//
//   out[r] = x[r] W^T + scale_a (x[r] A_a^T) B_a^T
//
// The first half, t = scale_a x A_a^T, is this file's kernel; the second is added to the accumulators of the projection
// itself (lora_add) or to the outputs before their rounding (lora_outputs), so they are rounded once and not read again.
//
// The first half reads every adapter in use once, A_a [rank][K], and is bound by that in a decode batch, where every row
// may have another one, and by reading x for many rows.  A workgroup takes 16 rows and the adapters they have, one after the
// other, on v_mfma_f32_16x16x32_bf16 (rows = token rows, columns = ranks); rows of other adapters go through the product as
// well and are not stored.  What fills the chip when rows are few: the adapters of a row tile are dealt out to several
// workgroups, and so is K, in parts that the second half (a decode batch) or a small kernel (many rows) adds up.
// 32 rows of 32 adapters, K = 4096, three segments of rank 16 (12.6 MB of A): 5.8 us; 3587 rows, K = 11008, rank 64 (79 MB of x): 27 us, and
// 5 for the parts' sums.  Whole calls, without | with: three outputs of 4096 each 19.2 | 27.7, SwiGLU 2048 x 4096 x 11008 of rank 32 267 |
// 296, 3587 x 11008 x 4096 247 | 287.
#include "bct_lora.h"

#include <algorithm>

#include "bct_device.h"
#include "bct_model_internal.h"

namespace bct {

namespace {

constexpr uint32_t kMaxRank = 256;

struct LoraPlan {
  uint32_t row_tiles;     // of 16 rows, of a workgroup
  uint32_t parts;         // of K
  uint32_t chunks, each;  // the columns of t: so many workgroups, each so many tiles of 16
};
constexpr uint32_t kGroupsFew = 256, kGroupsMany = 512, kMostParts = 8, kMostRowTiles = 4;

uint32_t tiles_of(uint32_t rows, uint32_t each) { return rows / each + (rows % each != 0); }

LoraPlan lora_plan(uint32_t rows, uint32_t K, uint32_t width) {
  LoraPlan p;
  const uint32_t tiles = width / 16;
  p.chunks = (tiles + 3) / 4;
  p.each = (tiles + p.chunks - 1) / p.chunks;
  // Row tiles of a workgroup: more of them read A fewer times where rows share an adapter, and multiply each adapter with more rows
  // of others where they do not, which the host cannot see: two from 12 million activations on, four from 36 million where they
  // also share what is loaded of x between three column tiles or more.  us of a call with 128 features, 1 | 2 | 4 row tiles, rows of 8 adapters
  // in runs of 512; of 60; of 64 adapters in turn:
  //   2048 x 4096 rank 64      29.4 | 30.6 | 30.4     34.0 | 35.8 | 34.9     108 | 148 | 188
  //   4096 x 1024 rank 64      17.3 | 21.8 | 20.5     20.5 | 26.1 | 25.5     85 | 143 | 184
  //   1500 x 11008 rank 16     48.6 | 48.7 | 49.3     52.7 | 50.6 | 51.1     104 | 113 | 143
  //   3000 x 11008 rank 64     64.7 | 60.7 | 61.0     87.3 | 72.6 | 69.5     314 | 357 | 502
  //   8192 x 4096 rank 32      35.9 | 36.3 | 37.7     39.1 | 39.6 | 40.7     179 | 190 | 261
  //   8192 x 4096 rank 128     55.5 | 53.3 | 53.8     85.2 | 71.9 | 65.3     518 | 542 | 690
  //   4096 x 11008 rank 64     73.4 | 67.4 | 66.7     92.4 | 83.8 | 78.4     379 | 434 | 563
  //   16384 x 4096 rank 16     61.6 | 55.6 | 60.8     62.7 | 60.3 | 64.7     326 | 319 | 361
  //   16384 x 4096 rank 128    109 | 93.6 | 86.0      145 | 133 | 114        983 | 1040 | 1315
  const uint64_t x = (uint64_t)rows * K;
  p.row_tiles = x < 12u << 20 ? 1 : x < 36u << 20 || p.each < 3 ? 2 : 4;
  // As many parts as give the chip one or two workgroups a compute unit, each wavefront at least two steps of 32 inputs.  us, one
  // | two: 1024 rows, 1 row tile, runs of 512 5.0 | 5.4, rank 64 9.0 | 10.0, an adapter for each row 14.5 | 15.9, 37 | 50; the call
  // of 3587 rows, 4 row tiles, 298 | 290.
  const uint64_t groups = (uint64_t)tiles_of(rows, 16 * p.row_tiles) * p.chunks, most = p.row_tiles == 1 ? kGroupsFew : kGroupsMany;
  p.parts = 1;
  while (p.parts < kMostParts && groups * p.parts * 2 <= most && K / 32 >= 16 * p.parts) p.parts *= 2;
  // Two parts of a short K do not make up for the kernel that adds them (many rows only): us of a call with two | one, K = 512 19.2 |
  // 17.1, 736 12.3 | 10.9, 960 61.4 | 59.0, 1184 19.6 | 18.5, 2016 116 | 116, 5184 41.6 | 43.3.
  if (p.parts == 2 && K < 2048 && rows >= 128) p.parts = 1;
  return p;
}

// The addends of a float in bf16: its upper bits, those below and those below these, cut off and not rounded, so that 24 bits of it
// are in three and all have its sign.  An addend that would be zero takes a part of the one before it, which is exact, so that an
// infinite weight times t is one, not as 0 * inf; an infinity or a NaN is in each.
__device__ __forceinline__ void addends_of(float t, float (&part)[3]) {
  const bool finite = fabsf(t) < INFINITY;
  part[0] = __uint_as_float(__float_as_uint(t) & 0xFFFF0000u);
  const float rest = t - part[0];
  part[1] = __uint_as_float(__float_as_uint(rest) & 0xFFFF0000u);
  part[2] = rest - part[1];
  if (rest == 0.f) part[0] *= 0.5f, part[1] = part[0];
  if (part[2] == 0.f) part[1] *= 0.5f, part[2] = part[1];
  if (!finite) part[0] = part[1] = part[2] = t;
}
// Where the operands of 16 rows x 16 ranks are written: 8 ranks of a row, the third addend in two halves.
__device__ __forceinline__ void store_operand(u32x4* op, size_t number, uint32_t row, uint32_t half, const float* t) {
  u32x4 w[3];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float p0[3], p1[3];
    addends_of(t[2 * e], p0);
    addends_of(t[2 * e + 1], p1);
    p0[2] *= 0.5f;
    p1[2] *= 0.5f;
#pragma unroll
    for (int i = 0; i < 3; ++i) w[i][e] = pack_bf16x2(p0[i], p1[i]);
  }
  op += number * 128 + 16 * half + row;
  op[0] = w[0];
  op[32] = w[1];
  op[64] = op[96] = w[2];
}

// OP: t goes out as operands (one part of K), else as fp32.  Workgroup ids go round the eight XCDs: the parts of K are dealt to
// them, so that an XCD's L2 sees one part of every adapter.
template <bool XT, int CT, int RT, bool OP>
__global__ __launch_bounds__(256) void lora_inputs_kernel(const uint16_t* __restrict__ x, const u32x4* __restrict__ a,
                                                          const float* __restrict__ scale,
                                                          const int32_t* __restrict__ adapter, float* __restrict__ t,
                                                          uint32_t rows, uint32_t K, uint32_t width, uint32_t n, uint32_t chunks,
                                                          uint32_t slots, uint32_t parts, uint32_t rank, uint32_t used) {
  constexpr int WAVES = 4, U = 4;
  __shared__ __attribute__((aligned(16))) float sC[WAVES][RT][16][20];
  const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64, jl = lane % 16, kg = lane / 16;
  const uint32_t part = blockIdx.x % 8 % parts, work = blockIdx.x / 8 * (8 / parts) + blockIdx.x % 8 / parts;
  const uint32_t groups = rows / (16 * RT) + (rows % (16 * RT) != 0), slot = work / (groups * chunks);
  if (slot >= slots) return;   // the last round of ids
  const uint32_t r0 = work / chunks % groups * (16 * RT), ct0 = work % chunks * CT, tiles = width / 16, KT = K / 32;
  const uint32_t p0 = (uint32_t)((uint64_t)part * KT / parts), p1 = (uint32_t)((uint64_t)(part + 1) * KT / parts);
  const uint32_t kt0 = p0 + wave * (p1 - p0) / WAVES, n_t = p0 + (wave + 1) * (p1 - p0) / WAVES - kt0;
  const uint16_t* xr[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) {   // row tiles past the end: the last one again, not stored
    const uint32_t row = min(r0 + 16 * i, (rows - 1) / 16 * 16);
    xr[i] = XT ? x + (((size_t)(row / 32) * KT + kt0) * 128 + row % 32 / 16 * 64 + lane) * 8
               : x + (size_t)min(row + jl, rows - 1) * K + (size_t)kt0 * 32 + kg * 8;
  }
  constexpr size_t xstep = XT ? 128 * 8 : 32;
  AdapterWalk<RT> walk(adapter, r0, rows, n);
  uint32_t turn = 0;
  while (walk.next()) {
    if (turn++ % slots != slot) continue;
    // a row tile without this adapter is read as one that has it, from cache
    const uint16_t* xs[RT];
#pragma unroll
    for (int i = RT - 1; i >= 0; --i)
      if (walk.match[i]) xs[0] = xr[i];
#pragma unroll
    for (int i = RT - 1; i >= 0; --i) xs[i] = walk.match[i] ? xr[i] : xs[0];
    const u32x4* at[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)   // tiles past the end: the last one again, not stored
      at[c] = a + (((size_t)walk.cur * tiles + min(ct0 + c, tiles - 1)) * KT + kt0) * 64 + lane;
    f32x4 acc[CT][RT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int i = 0; i < RT; ++i) acc[c][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    // U steps' loads are issued before the first product; those past the end are the last step's again, against zeros
    for (uint32_t s = 0; s < n_t; s += U) {
      const bool whole = s + U <= n_t;
      u32x4 av[U][CT], xv[U][RT];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const size_t i = whole ? s + u : min(s + u, n_t - 1);
#pragma unroll
        for (int c = 0; c < CT; ++c) av[u][c] = at[c][i * 64];
#pragma unroll
        for (int r = 0; r < RT; ++r) xv[u][r] = *(const u32x4*)(xs[r] + i * xstep);
      }
      if (!whole) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (s + u >= n_t) {
#pragma unroll
            for (int c = 0; c < CT; ++c) av[u][c] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int r = 0; r < RT; ++r) xv[u][r] = u32x4{0u, 0u, 0u, 0u};
          }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int r = 0; r < RT; ++r)
            acc[c][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, xv[u][r]),
                                                                __builtin_bit_cast(bf16x8, av[u][c]), acc[c][r], 0, 0, 0);
    }
    // the wavefronts' sums, one tile of ranks after the other; eight ranks of a row at a time go out
    const float f = scale ? scale[walk.cur] : 1.0f;
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      __syncthreads();   // what was there has been read
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int v = 0; v < 4; ++v) sC[wave][r][4 * kg + v][jl] = acc[c][r][v];
      __syncthreads();
      const uint32_t e = threadIdx.x, half = e % 2, i = e / 2 % 16, r = e / 32, row = r0 + 16 * r + i;
      if (e < RT * 32 && ct0 + c < tiles && adapter_of(adapter, row, rows, n) == walk.cur) {
        float sum[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t j = 8 * half + k;
          sum[k] = f * ((sC[0][r][i][j] + sC[1][r][i][j]) + (sC[2][r][i][j] + sC[3][r][i][j]));
        }
        const uint32_t col = (ct0 + c) * 16, rank0 = col - (col >= 2 * rank ? 2 * rank : col >= rank ? rank : 0u);   // of up to three segments
        if (rank0 + 16 > used) {
#pragma unroll
          for (uint32_t k = 0; k < 8; ++k) sum[k] = rank0 + 8 * half + k < used ? sum[k] : 0.f;
        }
        if (OP) {
          store_operand((u32x4*)t, (size_t)(row / 16) * tiles + ct0 + c, i, half, sum);
        } else {
          float* o = t + ((size_t)part * rows + row) * width + (ct0 + c) * 16 + 8 * half;
          *(f32x4*)o = f32x4{sum[0], sum[1], sum[2], sum[3]};
          *(f32x4*)(o + 4) = f32x4{sum[4], sum[5], sum[6], sum[7]};
        }
      }
    }
  }
}

// The parts of t, fp32, added up into operands: a thread takes eight ranks of a row.
template <int PARTS>
__global__ __launch_bounds__(256) void lora_operands_kernel(const float* __restrict__ t, u32x4* __restrict__ op,
                                                            uint32_t rows, uint32_t width) {
  const uint32_t eights = width / 8;
  const size_t e = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= (size_t)rows * eights) return;
  const uint32_t row = (uint32_t)(e / eights), c = (uint32_t)(e % eights);
  f32x4 v[PARTS][2];
#pragma unroll
  for (int p = 0; p < PARTS; ++p)
#pragma unroll
    for (int h = 0; h < 2; ++h) v[p][h] = ((const f32x4*)(t + ((size_t)p * rows + row) * width + 8 * c))[h];
  float sum[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    sum[k] = v[0][k / 4][k % 4];
#pragma unroll
    for (int p = 1; p < PARTS; ++p) sum[k] += v[p][k / 4][k % 4];
  }
  store_operand(op, (size_t)(row / 16) * (width / 16) + c / 2, row % 16, c % 2, sum);
}

// Row-major b [N][rank] -> 16-byte chunks of 8 ranks of one feature, (n / 16 * rank / 8 + k / 8) * 16 + n % 16.
__global__ __launch_bounds__(256) void lora_pack_kernel(const uint16_t* __restrict__ b, u32x4* __restrict__ packed, uint32_t N,
                                                        uint32_t rank) {
  const size_t c = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= (size_t)N * rank / 8) return;
  const size_t n = c / 16 / (rank / 8) * 16 + c % 16;
  packed[c] = *(const u32x4*)(b + n * rank + c / 16 % (rank / 8) * 8);
}

// Room for the parts in fp32 and for the operands, which are whole tiles of 16 rows with four bf16 for each t: for any number of
// rows up to this one.  Where K is in several parts, they and the workgroups are at most kGroupsMany.
size_t lora_bytes(uint32_t rows, uint32_t width) {
  const uint32_t tiles = tiles_of(rows, 16), split = kMostRowTiles * (kGroupsMany / ((width / 16 + 3) / 4));
  const size_t parts = std::max<size_t>(tiles, std::min<size_t>((size_t)kMostParts * tiles, split));
  return (2 * tiles + parts) * 16 * width * sizeof(float);
}

}  // namespace

bct_status check_lora(const bctm_lora* l, uint32_t rows, uint32_t K, uint32_t N, uint32_t segments, bool swiglu) {
  if (!l->a || !l->b || !l->adapter || l->n_adapters == 0 || l->rank == 0) return mfail(BCT_ERR_INVALID_ARG, "adapters: NULL pointer or zero size");
  if (swiglu != (l->b_up != nullptr)) return mfail(BCT_ERR_INVALID_ARG, "adapters: b_up goes with a SwiGLU");
  if (l->rank % 16 != 0 || l->rank > kMaxRank) return mfail(BCT_ERR_UNSUPPORTED, "adapters: rank must be a multiple of 16, at most 256");
  if (l->used > l->rank) return mfail(BCT_ERR_INVALID_ARG, "adapters: more ranks used than there are");
  if (l->n_adapters > 0x7FFFFFFFu) return mfail(BCT_ERR_UNSUPPORTED, "too many adapters");
  if ((uint64_t)tiles_of(rows, 16) * lora_plan(rows, K, segments * l->rank).chunks > 0x0FFFFFFFu) return mfail(BCT_ERR_UNSUPPORTED, "too many rows");
  if ((uint64_t)l->n_adapters * l->rank > (1ull << 56) / ((uint64_t)N + (uint64_t)segments * K)) return mfail(BCT_ERR_UNSUPPORTED, "too many adapters");
  if (!al16(l->a) || !al16(l->b) || !al16(l->b_up) || !al16(l->workspace)) return mfail(BCT_ERR_MISALIGNED, "pointers must be 16-byte aligned");
  if (!l->workspace || l->workspace_bytes < lora_bytes(rows, segments * l->rank))
    return mfail(BCT_ERR_BUFFER_TOO_SMALL, "adapters: the workspace is smaller than bctm_lora_workspace says");
  return BCT_OK;
}

template <bool XT, int RT, bool OP>
static void launch_inputs(const bctm_lora& l, const void* x, void* t, uint32_t rows, uint32_t K, uint32_t width, const LoraPlan& p,
                          hipStream_t s) {
  const uint32_t groups = tiles_of(rows, 16 * RT), most = l.n_adapters < 16 * RT ? l.n_adapters : 16 * RT;
  // how many workgroups share the adapters of a row tile: us, all in one | up to 256 | 1024 | 4096 workgroups in all: 32 rows of 32
  // adapters, K = 4096, rank 16 13.1 | 5.0 | 5.0 | 5.0, rank 64 43.6 | 13.0 | 13.0 | 13.0; 100 rows 13.9 | 7.0 | 7.1 | 7.0, 44 | 20 | 18.6 | 18.7; one
  // adapter a tile, 4096 rows 10.0 | 10.0 | 9.9 | 14.9
  uint32_t slots = 1;
  while (slots < most && rows > 1 && (uint64_t)groups * p.chunks * p.parts * slots * 2 <= 1024) slots *= 2;
  const uint64_t work = (uint64_t)groups * p.chunks * slots, per = 8 / p.parts;   // of one part
  const dim3 grid((unsigned)(8 * ((work + per - 1) / per))), block(256);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, s, (const uint16_t*)x, (const u32x4*)l.a, l.scale, l.adapter, (float*)t, rows, K,
                       width, l.n_adapters, p.chunks, slots, p.parts, l.rank, l.used ? l.used : l.rank);
  };
  if (p.each == 4) return launch(lora_inputs_kernel<XT, 4, RT, OP>);
  if (p.each == 3) return launch(lora_inputs_kernel<XT, 3, RT, OP>);
  if constexpr (RT < 4) {   // lora_plan: four row tiles with three column tiles or more
    if (p.each == 2) return launch(lora_inputs_kernel<XT, 2, RT, OP>);
    return launch(lora_inputs_kernel<XT, 1, RT, OP>);
  }
}
template <bool XT>
static void launch_inputs_of(const bctm_lora& l, const void* x, void* t, uint32_t rows, uint32_t K, uint32_t width,
                             const LoraPlan& p, bool operands, hipStream_t s) {
  if (p.row_tiles == 4) {
    if (operands) launch_inputs<XT, 4, true>(l, x, t, rows, K, width, p, s);
    else launch_inputs<XT, 4, false>(l, x, t, rows, K, width, p, s);
  } else if (p.row_tiles == 2) {
    if (operands) launch_inputs<XT, 2, true>(l, x, t, rows, K, width, p, s);
    else launch_inputs<XT, 2, false>(l, x, t, rows, K, width, p, s);
  } else {
    if (operands) launch_inputs<XT, 1, true>(l, x, t, rows, K, width, p, s);
    else launch_inputs<XT, 1, false>(l, x, t, rows, K, width, p, s);
  }
}

bct_status launch_lora_inputs(const bctm_lora& l, const void* x, uint32_t rows, uint32_t K, bool x_tiled, uint32_t segments,
                              bool operands, hipStream_t s, LoraTerm* term) {
  const uint32_t width = segments * l.rank;
  const LoraPlan p = lora_plan(rows, K, width);
  // the operands first, then the parts
  u32x4* op = (u32x4*)l.workspace;
  float* t = (float*)l.workspace + (size_t)tiles_of(rows, 16) * 32 * width;
  const bool at_once = operands && p.parts == 1;
  if (x_tiled) launch_inputs_of<true>(l, x, at_once ? (void*)op : t, rows, K, width, p, at_once, s);
  else launch_inputs_of<false>(l, x, at_once ? (void*)op : t, rows, K, width, p, at_once, s);
  if (operands && !at_once) {
    const size_t blocks = ((size_t)rows * (width / 8) + 255) / 256;
    if (blocks > 0x7FFFFFFFu) return mfail(BCT_ERR_UNSUPPORTED, "too many rows");
    const auto kernel = p.parts == 2 ? lora_operands_kernel<2> : p.parts == 4 ? lora_operands_kernel<4> : lora_operands_kernel<8>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, s, t, op, rows, width);
  }
  *term = {t, op, (const u32x4*)l.b, (const u32x4*)l.b_up, l.adapter, l.n_adapters, l.rank, width, p.parts, segments};
  return launched("lora");
}

}  // namespace bct

using namespace bct;

extern "C" {

bct_status bctm_lora_workspace(uint32_t rows, uint32_t K, uint32_t rank, uint32_t segments, size_t* bytes) {
  if (!bytes || rows == 0 || K == 0 || rank == 0 || segments == 0) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer or zero size");
  if (K % 32 != 0 || rank % 16 != 0 || rank > kMaxRank || segments > 3)
    return mfail(BCT_ERR_UNSUPPORTED, "K must be a multiple of 32, rank of 16 and at most 256, segments at most 3");
  *bytes = lora_bytes(rows, segments * rank);
  return BCT_OK;
}

bct_status bctm_lora_pack(const void* b, void* packed, uint32_t N, uint32_t rank, void* hip_stream) {
  if (!b || !packed || N == 0 || rank == 0) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer or zero size");
  if (b == packed) return mfail(BCT_ERR_INVALID_ARG, "packing in place is not possible");
  if (N % 16 != 0 || rank % 16 != 0 || rank > kMaxRank)
    return mfail(BCT_ERR_UNSUPPORTED, "N and rank must be multiples of 16, rank at most 256");
  if (!al16(b) || !al16(packed)) return mfail(BCT_ERR_MISALIGNED, "pointers must be 16-byte aligned");
  const size_t chunks = (size_t)N * rank / 8;
  if ((chunks + 255) / 256 > 0x7FFFFFFFu) return mfail(BCT_ERR_UNSUPPORTED, "matrix too large");
  hipLaunchKernelGGL(lora_pack_kernel, dim3((unsigned)((chunks + 255) / 256)), dim3(256), 0, (hipStream_t)hip_stream,
                     (const uint16_t*)b, (u32x4*)packed, N, rank);
  return launched("lora_pack");
}

}  // extern "C"
