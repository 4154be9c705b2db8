// The matrix-core projections of many token rows with bias, activation, residual and fp32 outputs in their epilogue: the kernel of
// bct_linear_rows.hip with an EpilogueTerm.  It is applied to the fp32 sums where they are written out, so it costs no pass
// over memory of its own.  4096 x 4096 x 11008, tiled x: 249 us without bias and activation (bctm_linear), 256 with a bias, 266 into fp32, 277 with bias
// and gelu_tanh.
//
// Few features of many rows (a router's logits) are neither: no tile of it is wide enough for the matrix cores to be busy, and the streaming
// kernel, a workgroup per 16 features, reads every row once for each of them.  linear_narrow_kernel has all 64 features in a
// workgroup of 16 or 32 rows, so it reads the rows once.
#include "bct_linear_rows.h"

namespace bct {

namespace {

// 16 * RT rows and 64 features of a workgroup; its wavefronts share K, each with row tiles of its own in LDS.  Bound by the address
// unit of a compute unit: a kilobyte of weights or rows takes 16 cycles of it, but rows read as operands lie, 16 side by side, take
// 64; so a row's 256 bytes of four K tiles come to LDS whole (chunk c of row r at place c ^ r of its 16, so that an operand read
// finds its rows in different banks), a round of four ahead of the products.  Every second round only: on the path from the loop's break its second
// half's registers count as unfinished, so at its head the compiler waits for all loads in flight before the next are requested.  4096 rows, 4096 -> 64: 12.9 us (33.5 MB of rows are 5.5 at the rate of a
// copy); rows as operands lie, the weights straight to registers all the same: 18.
template <bool XT, int RT>
__global__ __launch_bounds__(512) void linear_narrow_kernel(const uint16_t* __restrict__ x, const u32x4* __restrict__ w,
                                                            const uint16_t* residual, void* out, uint32_t rows, uint32_t K, uint32_t N,
                                                            uint32_t out_tiled, EpilogueTerm term) {
  constexpr int WAVES = 8, FT = 4, U = 4;
  __shared__ union {
    u32x4 x[2][WAVES][RT][256];       // two rounds: 16 rows of 16 chunks
    float sum[WAVES][FT][16][17];
  } s;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, jl = lane % 16, kg = lane / 16, KT = K / 32;
  const uint32_t kt0 = wave * KT / WAVES, n_t = (wave + 1) * KT / WAVES - kt0, r0 = blockIdx.x * (16 * RT), n0 = blockIdx.y * 64;
  const u32x4* wt[FT];
#pragma unroll
  for (int f = 0; f < FT; ++f) wt[f] = w + ((size_t)(n0 / 16 + f) * KT + kt0) * 64 + lane;
  // Lane l of load i: row 4 i + l / 16 (rows past the end: the last one again); of tiled activations K tile i as it lies, an operand.
  const uint16_t* xr[RT][4];
#pragma unroll
  for (int j = 0; j < RT; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      xr[j][i] = XT ? x + (((size_t)min(r0 / 32 + (r0 % 32 / 16 + j) / 2, (rows + 31) / 32 - 1) * KT + kt0) * 128 + (r0 / 16 + j) % 2 * 64 + lane) * 8
                    : x + (size_t)min(r0 + 16 * j + 4 * i + kg, rows - 1) * K + (size_t)kt0 * 32;
  f32x4 acc[FT][RT];
#pragma unroll
  for (int f = 0; f < FT; ++f)
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[f][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto request = [&](uint32_t t, uint32_t stage, u32x4 (&b)[U][FT]) {   // tiles past the end: the last one again, not multiplied
    const uint32_t last = n_t - 1;
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t c = jl ^ (4 * i + kg);
        load_to_lds(xr[j][i] + (XT ? (size_t)min(t + i, last) * 1024 : (size_t)min(t + c / 4, last) * 32 + c % 4 * 8), &s.x[stage][wave][j][64 * i]);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int f = 0; f < FT; ++f) b[u][f] = wt[f][(size_t)min(t + u, last) * 64];
  };
  auto products = [&](uint32_t t, uint32_t stage, const u32x4 (&b)[U][FT]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t + u >= n_t) break;
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        const bf16x8 a = __builtin_bit_cast(bf16x8, s.x[stage][wave][j][XT ? 64 * u + lane : 16 * jl + ((4 * u + kg) ^ jl)]);
#pragma unroll
        for (int f = 0; f < FT; ++f) acc[f][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, b[u][f]), acc[f][j], 0, 0, 0);
      }
    }
  };
  if (n_t > 0) {
    u32x4 b0[U][FT], b1[U][FT];
    request(0, 0, b0);
    for (uint32_t t = 0; t < n_t; t += 2 * U) {
      // a stage is asked for again once its reads have returned; what arrives is the wavefront's alone, so no barriers
      request(t + U, 1, b1);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(wait_vm(4 * RT + U * FT));
      products(t, 0, b0);
      __builtin_amdgcn_s_waitcnt(kWaitLds);
      __builtin_amdgcn_sched_barrier(0);
      if (t + U >= n_t) break;
      request(t + 2 * U, 0, b0);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(wait_vm(4 * RT + U * FT));
      products(t + U, 1, b1);
      __builtin_amdgcn_s_waitcnt(kWaitLds);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __builtin_amdgcn_s_waitcnt(wait_vm(0));   // the last requests, before LDS is used otherwise
  // Element v of a lane: row 4 * kg + v, feature jl.  A thread adds up eight features of a row, the wavefronts' sums in their order.
#pragma unroll
  for (int j = 0; j < RT; ++j) {
    __syncthreads();
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
      for (int v = 0; v < 4; ++v) s.sum[wave][f][4 * kg + v][jl] = acc[f][j][v];
    __syncthreads();
    const uint32_t i = threadIdx.x / 8, c = threadIdx.x % 8, row = r0 + 16 * j + i, n = n0 + 8 * c;
    if (i < 16 && row < rows) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[e] = 0.f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) y[e] += s.sum[k][c / 2][i][c % 2 * 8 + e];
      }
      term.apply(y, n);
      const size_t at = (size_t)row * N + n;
      if (residual) {
        float v[8];
        unpack16<BF16>(*(const u32x4*)(residual + at), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] += v[e];
      }
      if (term.out32) {
        *(f32x4*)((float*)out + at) = *(const f32x4*)&y[0];
        *(f32x4*)((float*)out + at + 4) = *(const f32x4*)&y[4];
      } else {
        const u32x4 o = pack16_round<BF16>(y);
        if (out_tiled) ((u32x4*)out)[tiled_chunk(row, n, N)] = o;
        else *(u32x4*)((uint16_t*)out + at) = o;
      }
    }
  }
}

}  // namespace

hipError_t launch_linear_narrow(const void* x, const void* w, const void* residual, void* out, uint32_t rows, uint32_t K, uint32_t N,
                                bool x_tiled, bool out_tiled, hipStream_t s, const EpilogueTerm& term, uint32_t row_tiles) {
  const dim3 grid((rows + 16 * row_tiles - 1) / (16 * row_tiles), N / 64);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(512), 0, s, (const uint16_t*)x, (const u32x4*)w, (const uint16_t*)residual, out, rows, K, N,
                       out_tiled ? 1u : 0u, term);
  };
  if (x_tiled) row_tiles == 1 ? launch(linear_narrow_kernel<true, 1>) : launch(linear_narrow_kernel<true, 2>);
  else row_tiles == 1 ? launch(linear_narrow_kernel<false, 1>) : launch(linear_narrow_kernel<false, 2>);
  return hipGetLastError();
}

hipError_t launch_linear_rows_act(const void* x, const void* w, const void* residual, const LinearOut& dst, uint32_t rows,
                                  uint32_t K, uint32_t N, bool x_tiled, bool out_tiled, hipStream_t s, const EpilogueTerm& term) {
  if (x_tiled) launch_rows<false, true>(x, w, nullptr, residual, dst, rows, K, N, out_tiled, s, term);
  else launch_rows<false, false>(x, w, nullptr, residual, dst, rows, K, N, out_tiled, s, term);
  return hipGetLastError();
}

}  // namespace bct
