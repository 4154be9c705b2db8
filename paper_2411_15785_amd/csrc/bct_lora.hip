// Low-rank adapters of many requests at once beside a shared projection (gfx950): row r of a batch belongs to a request with
// the adapter a = adapter[r], and
//
//   out[r] = x[r] W^T + scale_a (x[r] A_a^T) B_a^T
//
// The first half, t = scale_a x A_a^T, is this file's kernel; the second is added to the accumulators of the projection
// itself (lora_add), so the rows' outputs are rounded once and not read again.
//
// The first half reads every adapter in use once, A_a [rank][K], and is bound by that in a decode batch, where every row
// may have another one, and by reading x for many rows.  A workgroup takes 16 rows and the adapters they have, one after the
// other, on v_mfma_f32_16x16x32_bf16 (rows = token rows, columns = ranks); rows of other adapters go through the product as
// well and are not stored.  What fills the chip when rows are few: the adapters of a row tile are dealt out to several
// workgroups, and so is K, in parts that the second half adds up.
#include "bct_lora.h"

#include "bct_device.h"
#include "bct_model_internal.h"

namespace bct {

namespace {

constexpr uint32_t kMaxRank = 256;

struct LoraPlan {
  uint32_t parts;         // of K
  uint32_t chunks, each;  // the columns of t: so many workgroups, each so many tiles of 16
};

LoraPlan lora_plan(uint32_t rows, uint32_t K, uint32_t width) {
  LoraPlan p;
  const uint32_t tiles = width / 16;
  p.chunks = (tiles + 3) / 4;
  p.each = (tiles + p.chunks - 1) / p.chunks;
  // as many parts as give the chip two workgroups a compute unit, each wavefront at least two steps of 32 inputs
  const uint64_t groups = (uint64_t)((rows / 16 + (rows % 16 != 0))) * p.chunks;
  p.parts = 1;
  while (p.parts < 8 && groups * p.parts * 2 <= 512 && K / 32 >= 16 * p.parts) p.parts *= 2;
  return p;
}

template <bool XT, int CT>
__global__ __launch_bounds__(256) void lora_inputs_kernel(const uint16_t* __restrict__ x, const u32x4* __restrict__ a,
                                                          const float* __restrict__ scale,
                                                          const int32_t* __restrict__ adapter, float* __restrict__ t,
                                                          uint32_t rows, uint32_t K, uint32_t width, uint32_t n, uint32_t chunks) {
  constexpr int WAVES = 4, U = 4;
  __shared__ float sC[WAVES][CT][16][17];
  const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64, jl = lane % 16, kg = lane / 16;
  const uint32_t r0 = blockIdx.x / chunks * 16, ct0 = blockIdx.x % chunks * CT, tiles = width / 16, KT = K / 32;
  const uint32_t part = blockIdx.z, parts = gridDim.z;
  const uint32_t p0 = (uint32_t)((uint64_t)part * KT / parts), p1 = (uint32_t)((uint64_t)(part + 1) * KT / parts);
  const uint32_t kt0 = p0 + wave * (p1 - p0) / WAVES, n_t = p0 + (wave + 1) * (p1 - p0) / WAVES - kt0;
  const uint16_t* xr = XT ? x + (((size_t)(r0 / 32) * KT + kt0) * 128 + r0 % 32 / 16 * 64 + lane) * 8
                          : x + (size_t)min(r0 + jl, rows - 1) * K + (size_t)kt0 * 32 + kg * 8;
  constexpr size_t xstep = XT ? 128 * 8 : 32;
  const uint32_t id[1] = {adapter_of(adapter, r0 + jl, rows, n)};
  uint32_t turn = 0;
  for (uint32_t cur = next_adapter<1>(id, 0, n); cur < n; cur = next_adapter<1>(id, cur + 1, n)) {
    if (turn++ % gridDim.y != blockIdx.y) continue;
    const u32x4* at[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)   // tiles past the end: the last one again, not stored
      at[c] = a + (((size_t)cur * tiles + min(ct0 + c, tiles - 1)) * KT + kt0) * 64 + lane;
    f32x4 acc[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (uint32_t s = 0; s < n_t; s += U) {
      u32x4 av[U][CT], xv[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t i = min(s + u, n_t - 1);
#pragma unroll
        for (int c = 0; c < CT; ++c) av[u][c] = at[c][(size_t)i * 64];
        xv[u] = *(const u32x4*)(xr + i * xstep);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (s + u < n_t) {
#pragma unroll
          for (int c = 0; c < CT; ++c)
            acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, xv[u]),
                                                             __builtin_bit_cast(bf16x8, av[u][c]), acc[c], 0, 0, 0);
        }
    }
    __syncthreads();   // the sums of the adapter before have been read
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int v = 0; v < 4; ++v) sC[wave][c][4 * kg + v][jl] = acc[c][v];
    __syncthreads();
    const uint32_t row = r0 + threadIdx.x / 16, col = threadIdx.x % 16;
    if (adapter_of(adapter, row, rows, n) == cur) {
      const float f = scale ? scale[cur] : 1.0f;
#pragma unroll
      for (int c = 0; c < CT; ++c)
        if (ct0 + c < tiles) {
          const uint32_t i = threadIdx.x / 16;
          t[((size_t)part * rows + row) * width + (ct0 + c) * 16 + col] =
              f * ((sC[0][c][i][col] + sC[1][c][i][col]) + (sC[2][c][i][col] + sC[3][c][i][col]));
        }
    }
  }
}

// Row-major b [N][rank] -> 16-byte chunks of 8 ranks of one feature, (n / 16 * rank / 8 + k / 8) * 16 + n % 16.
__global__ __launch_bounds__(256) void lora_pack_kernel(const uint16_t* __restrict__ b, u32x4* __restrict__ packed, uint32_t N,
                                                        uint32_t rank) {
  const size_t c = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= (size_t)N * rank / 8) return;
  const size_t n = c / 16 / (rank / 8) * 16 + c % 16;
  packed[c] = *(const u32x4*)(b + n * rank + c / 16 % (rank / 8) * 8);
}

size_t lora_bytes(uint32_t rows, uint32_t K, uint32_t width) {
  return (size_t)lora_plan(rows, K, width).parts * rows * width * sizeof(float);
}

}  // namespace

bct_status check_lora(const bctm_lora* l, uint32_t rows, uint32_t K, uint32_t N, uint32_t segments, bool swiglu) {
  if (!l->a || !l->b || !l->adapter || l->n_adapters == 0 || l->rank == 0) return mfail(BCT_ERR_INVALID_ARG, "adapters: NULL pointer or zero size");
  if (swiglu != (l->b_up != nullptr)) return mfail(BCT_ERR_INVALID_ARG, "adapters: b_up goes with a SwiGLU");
  if (l->rank % 16 != 0 || l->rank > kMaxRank) return mfail(BCT_ERR_UNSUPPORTED, "adapters: rank must be a multiple of 16, at most 256");
  if (l->n_adapters > 0x7FFFFFFFu) return mfail(BCT_ERR_UNSUPPORTED, "too many adapters");
  if ((uint64_t)((rows / 16 + (rows % 16 != 0))) * lora_plan(rows, K, segments * l->rank).chunks > 0x7FFFFFFFu) return mfail(BCT_ERR_UNSUPPORTED, "too many rows");
  if ((uint64_t)l->n_adapters * l->rank > (1ull << 56) / ((uint64_t)N + (uint64_t)segments * K)) return mfail(BCT_ERR_UNSUPPORTED, "too many adapters");
  if (!al16(l->a) || !al16(l->b) || !al16(l->b_up) || !al16(l->workspace)) return mfail(BCT_ERR_MISALIGNED, "pointers must be 16-byte aligned");
  if (!l->workspace || l->workspace_bytes < lora_bytes(rows, K, segments * l->rank))
    return mfail(BCT_ERR_BUFFER_TOO_SMALL, "adapters: the workspace is smaller than bctm_lora_workspace says");
  return BCT_OK;
}

template <bool XT>
static void launch_inputs(const bctm_lora& l, const void* x, uint32_t rows, uint32_t K, uint32_t width, const LoraPlan& p,
                          hipStream_t s) {
  const uint32_t tiles = (rows / 16 + (rows % 16 != 0)), most = l.n_adapters < 16 ? l.n_adapters : 16;
  uint32_t slots = 1;
  while (slots < most && rows > 1 && (uint64_t)tiles * p.chunks * p.parts * slots * 2 <= 1024) slots *= 2;
  const dim3 grid(tiles * p.chunks, slots, p.parts), block(256);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, s, (const uint16_t*)x, (const u32x4*)l.a, l.scale, l.adapter, (float*)l.workspace,
                       rows, K, width, l.n_adapters, p.chunks);
  };
  switch (p.each) {
    case 1: return launch(lora_inputs_kernel<XT, 1>);
    case 2: return launch(lora_inputs_kernel<XT, 2>);
    case 3: return launch(lora_inputs_kernel<XT, 3>);
    default: return launch(lora_inputs_kernel<XT, 4>);
  }
}

bct_status launch_lora_inputs(const bctm_lora& l, const void* x, uint32_t rows, uint32_t K, bool x_tiled, uint32_t segments,
                              hipStream_t s, LoraTerm* term) {
  const uint32_t width = segments * l.rank;
  const LoraPlan p = lora_plan(rows, K, width);
  if (x_tiled) launch_inputs<true>(l, x, rows, K, width, p, s);
  else launch_inputs<false>(l, x, rows, K, width, p, s);
  *term = {(const float*)l.workspace, (const u32x4*)l.b, (const u32x4*)l.b_up, l.adapter, l.n_adapters, l.rank, width, p.parts, segments};
  return launched("lora");
}

}  // namespace bct

using namespace bct;

extern "C" {

bct_status bctm_lora_workspace(uint32_t rows, uint32_t K, uint32_t rank, uint32_t segments, size_t* bytes) {
  if (!bytes || rows == 0 || K == 0 || rank == 0 || segments == 0) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer or zero size");
  if (K % 32 != 0 || rank % 16 != 0 || rank > kMaxRank || segments > 3)
    return mfail(BCT_ERR_UNSUPPORTED, "K must be a multiple of 32, rank of 16 and at most 256, segments at most 3");
  *bytes = lora_bytes(rows, K, segments * rank);
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
