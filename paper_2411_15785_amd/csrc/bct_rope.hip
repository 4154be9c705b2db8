// Norms of the queries and write queries of each head with the position rotation in the same pass (gfx950): what stands
// between the projections W_q, W_wq (section 3.2 step 1) and the bounded cache that the two address.
//
//   y = x * rsqrt(mean(x^2) + eps) * gain                                    over the head's d elements
//   (y_a, y_b) = (y_a cos t - y_b sin t, y_a sin t + y_b cos t),  t = position * inv_freq[j], pair j of the rotated part
//
// Bound by memory: every element is read once and written once, 16 bytes a lane.  A lane keeps the two chunks of a head
// that rotate into each other (16 bytes each: elements E l .. E l + E - 1 of both halves, or two chunks of neighbours), so a
// pair never leaves its lane, and the d / 2E lanes of a head share one sum of squares.  The angles of a row are those of
// all its heads: a lane works out its E pairs once, while the heads it will turn are on their way from memory.
// 16384 rows x 64 heads of 128 bf16 (537 MB): 94 us, 5.7 TB/s (a copy of 1 GB reaches 6.1); 1 row 3.2 us, the launch.
#include <math.h>

#include <type_traits>

#include "bct_device.h"
#include "bct_model_internal.h"

namespace bct {

namespace {

struct HeadBlock {   // the heads of one input: rows of n heads side by side, ld elements from row to row
  const void* in;
  void* out;
  const void* gain;   // [d], or NULL for ones
  size_t ld, out_ld;
  uint32_t n;
};

enum RopePairs { kNoRotation, kHalves, kNeighbours };

// cos and sin of position * inv_freq.  The angle is a product in 64 bits and loses its whole turns there: in 32 bits a
// position of 2^20 would leave 0.06 of a radian unknown.  What remains, less its nearest quarter turn, is at most pi / 4; R is
// the type that it goes on in.  float, for bf16 heads: the Taylor series of degree 9 and 10 are within 2e-9, and roundings leave less than
// 2^-23, of which the output's rounding leaves nothing.  double, for fp32 heads: degree 11 and 12, within 7e-12, and one rounding to fp32.
template <typename R>
__device__ __forceinline__ void turn_of(int32_t position, double inv_freq, float* c, float* s) {
  const double turns = (double)position * inv_freq * 0.15915494309189533577;
  const double quarters = rint(4.0 * turns);
  const R x = (R)((turns - 0.25 * quarters) * 6.28318530717958647692);
  const float q = (float)(quarters - 4.0 * floor(0.25 * quarters));   // 0 to 3: which quarter turn
  const R z = x * x;
  auto fma = [](R a, R b, R c) -> R {
    if constexpr (sizeof(R) == 4) return __builtin_fmaf(a, b, c);
    else return __builtin_fma(a, b, c);
  };
  R sn = (R)(1.0 / 362880), cs = (R)(-1.0 / 3628800);
  if constexpr (sizeof(R) == 8) {
    sn = fma(z, -1.0 / 39916800, sn);
    cs = fma(z, 1.0 / 479001600, cs);
  }
  sn = fma(z, sn, (R)(-1.0 / 5040));
  sn = fma(z, sn, (R)(1.0 / 120));
  sn = fma(z, sn, (R)(-1.0 / 6));
  sn = fma(z * x, sn, x);
  cs = fma(z, cs, (R)(1.0 / 40320));
  cs = fma(z, cs, (R)(-1.0 / 720));
  cs = fma(z, cs, (R)(1.0 / 24));
  cs = fma(z, cs, (R)-0.5);
  cs = fma(z, cs, (R)1.0);
  const bool odd = q == 1.f || q == 3.f;
  const float a = (float)(odd ? sn : cs), b = (float)(odd ? cs : sn);
  *c = q == 1.f || q == 2.f ? -a : a;
  *s = q >= 2.f ? -b : b;
}

// G lanes to a head (the power of two from d / 2E on), HPG heads to a group of them: slot s of the `slots` groups of a row
// has the heads s, s + slots, ...  q's heads come first, then k's.  PAST: loads and stores leave the caches as they are.
template <typename DT, bool NORM, RopePairs PAIRS, int G, int HPG, bool PAST>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(HeadBlock q, HeadBlock k, const int32_t* __restrict__ positions,
                                                           const double* __restrict__ inv_freq, uint32_t rot, uint32_t rows,
                                                           uint32_t d, uint32_t slots, float eps) {
  typedef typename DT::elem elem;
  constexpr uint32_t E = DT::kElemsPerVec;
  const uint64_t group = ((uint64_t)blockIdx.x * 256 + threadIdx.x) / G;
  const uint32_t l = threadIdx.x % G, slot = (uint32_t)(group % slots);
  const uint64_t row = group / slots;
  const bool mine = row < rows && l < d / (2 * E);
  // the lane's two chunks of a head, in elements; lanes behind the rotated part hold neighbours that pass
  const bool turned = PAIRS != kNoRotation && l < rot / (2 * E);
  const uint32_t e0 = PAIRS == kHalves && turned ? E * l : 2 * E * l, e1 = PAIRS == kHalves && turned ? E * l + rot / 2 : e0 + E;

  u32x4 v[HPG][2];
#pragma unroll
  for (int i = 0; i < HPG; ++i) {
    const uint32_t h = slot + i * slots;
    if (mine && h < q.n + k.n) {
      const elem* p = h < q.n ? (const elem*)q.in + row * q.ld + (size_t)h * d : (const elem*)k.in + row * k.ld + (size_t)(h - q.n) * d;
      v[i][0] = PAST ? __builtin_nontemporal_load((const u32x4*)(p + e0)) : *(const u32x4*)(p + e0);
      v[i][1] = PAST ? __builtin_nontemporal_load((const u32x4*)(p + e1)) : *(const u32x4*)(p + e1);
    } else {
      v[i][0] = v[i][1] = u32x4{0u, 0u, 0u, 0u};
    }
  }
  float cs[E], sn[E];
  if constexpr (PAIRS != kNoRotation) {
    if (mine && turned) {
      const int32_t at = positions[row];
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) turn_of<std::conditional_t<E == 4, double, float>>(at, inv_freq[E * l + e], &cs[e], &sn[e]);
    } else {
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) {
        cs[e] = 1.f;
        sn[e] = 0.f;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < HPG; ++i) {
    const uint32_t h = slot + i * slots;
    float f[2 * E];
    unpack16<DT>(v[i][0], f);
    unpack16<DT>(v[i][1], f + E);
    if constexpr (NORM) {
      float ss = 0.f;
#pragma unroll
      for (uint32_t e = 0; e < 2 * E; ++e) ss = __builtin_fmaf(f[e], f[e], ss);
      ss = xor_sum<1, G / 2>(ss);
      const float r = 1.0f / sqrtf(ss / (float)d + eps);
      const elem* gain = (const elem*)(h < q.n ? q.gain : k.gain);
      if (gain && mine) {
        float g[2 * E];
        unpack16<DT>(*(const u32x4*)(gain + e0), g);
        unpack16<DT>(*(const u32x4*)(gain + e1), g + E);
#pragma unroll
        for (uint32_t e = 0; e < 2 * E; ++e) f[e] = f[e] * r * g[e];
      } else {
#pragma unroll
        for (uint32_t e = 0; e < 2 * E; ++e) f[e] *= r;
      }
    }
    if constexpr (PAIRS != kNoRotation) {
      if (turned) {   // not by a turn of nothing: an infinity beside it would make a NaN of what passes
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) {
          const uint32_t a = PAIRS == kHalves ? e : 2 * e, b = PAIRS == kHalves ? E + e : 2 * e + 1;
          const float fa = f[a], fb = f[b];
          f[a] = fa * cs[e] - fb * sn[e];
          f[b] = fa * sn[e] + fb * cs[e];
        }
      }
    }
    if (mine && h < q.n + k.n) {
      elem* o = h < q.n ? (elem*)q.out + row * q.out_ld + (size_t)h * d : (elem*)k.out + row * k.out_ld + (size_t)(h - q.n) * d;
      const u32x4 o0 = pack16_round<DT>(f), o1 = pack16_round<DT>(f + E);
      if (PAST) {
        __builtin_nontemporal_store(o0, (u32x4*)(o + e0));
        __builtin_nontemporal_store(o1, (u32x4*)(o + e1));
      } else {
        *(u32x4*)(o + e0) = o0;
        *(u32x4*)(o + e1) = o1;
      }
    }
  }
}

struct RopeCall {
  HeadBlock q, k;
  const int32_t* positions;
  const double* inv_freq;
  uint32_t rot, rows, d;
  float eps;
  hipStream_t s;
};

template <typename DT, bool NORM, RopePairs PAIRS, int G, int HPG, bool PAST>
bct_status launch_rope(const RopeCall& c) {
  const uint32_t heads = c.q.n + c.k.n, slots = (heads + HPG - 1) / HPG;
  const uint64_t blocks = ((uint64_t)c.rows * slots * G + 255) / 256;
  if (blocks > 0x7FFFFFFFull) return mfail(BCT_ERR_UNSUPPORTED, "too many rows and heads for one launch");
  hipLaunchKernelGGL((qk_norm_rope_kernel<DT, NORM, PAIRS, G, HPG, PAST>), dim3((unsigned)blocks), dim3(256), 0, c.s, c.q, c.k,
                     c.positions, c.inv_freq, c.rot, c.rows, c.d, slots, c.eps);
  return launched("qk_norm_rope");
}

// Two heads a group, once one leaves eight wavefronts for each of 256 compute units: its loads are in flight at once and
// the angles are worked out for two.  us, 1 | 2 | 4 | 8 heads, bf16: 1 row of 64 heads of 128 3.27 | 3.58 | 4.69 | 6.74; 256 rows x 64
// x 64 (2048 wavefronts) 3.69 | 4.09 | 5.11 | 7.36; x 128 (4096) 4.83 | 4.40 | 5.46 | 7.66; 2048 x 64 x 128 16.2 | 15.0 | 14.5 | 15.7; 16384 x
// 64 x 128 122 | 97.5 | 97.3 | 102; fp32 256 x 64 x 64 4.22 | 3.89 | 5.38 | 6.29, 16384 x 64 x 128 371 | 378 | 375 | 402 for heads of 256, 187
// | 186 | 192 | 198.
// Past the caches where what is read and written is more than the last-level cache's 256 MB, so that nothing of it would be found
// there: 16384 x 64 x 128 bf16 (537 MB) 104 | 94.4 us (5.7 TB/s).  Smaller outputs are in that cache for the step that follows.
template <typename DT, bool NORM, RopePairs PAIRS, int G>
bct_status rope_heads(const RopeCall& c) {
  const bool two = (uint64_t)c.rows * (c.q.n + c.k.n) * G >= 8ull * 64 * 256;
  const uint64_t elements = (uint64_t)c.rows * (c.q.n + c.k.n) * c.d;
  if (2 * elements * (16 / DT::kElemsPerVec) > 256ull << 20) return launch_rope<DT, NORM, PAIRS, G, 2, true>(c);
  return two ? launch_rope<DT, NORM, PAIRS, G, 2, false>(c) : launch_rope<DT, NORM, PAIRS, G, 1, false>(c);
}
template <typename DT, bool NORM, RopePairs PAIRS>
bct_status rope_group(const RopeCall& c) {
  const uint32_t lanes = c.d / (2 * DT::kElemsPerVec);
  if (lanes <= 4) return rope_heads<DT, NORM, PAIRS, 4>(c);
  if (lanes <= 8) return rope_heads<DT, NORM, PAIRS, 8>(c);
  if constexpr (DT::kElemsPerVec == 4) {   // a bf16 head has at most 16 lanes
    if (lanes > 16) return rope_heads<DT, NORM, PAIRS, 32>(c);
  }
  return rope_heads<DT, NORM, PAIRS, 16>(c);
}
template <typename DT>
bct_status rope_form(const RopeCall& c, bool norm, RopePairs pairs) {
  if (!norm) return pairs == kHalves ? rope_group<DT, false, kHalves>(c) : rope_group<DT, false, kNeighbours>(c);
  if (pairs == kHalves) return rope_group<DT, true, kHalves>(c);
  if (pairs == kNeighbours) return rope_group<DT, true, kNeighbours>(c);
  return rope_group<DT, true, kNoRotation>(c);
}

// Whether the n * d wide rows of two blocks (a with rows at a distance of lda elements, b of ldb) share a byte.
bool rows_overlap(const void* a, uint64_t wide_a, uint64_t lda, const void* b, uint64_t wide_b, uint64_t ldb, uint32_t rows,
                  uint64_t size) {
  const uint64_t pa = (uintptr_t)a, pb = (uintptr_t)b;
  if (pa + ((rows - 1) * lda + wide_a) * size <= pb || pb + ((rows - 1) * ldb + wide_b) * size <= pa) return false;
  if (lda != ldb) return true;   // not looked at row by row
  // rows of one distance: side by side in it, or not
  const uint64_t step = lda * size, at = pb >= pa ? (pb - pa) % step : (step - (pa - pb) % step) % step;
  return at < wide_a * size || at + wide_b * size > step;
}

}  // namespace
}  // namespace bct

using namespace bct;

extern "C" bct_status bctm_qk_norm_rope(const void* q, void* q_out, const void* q_gain, uint32_t n_q_heads, size_t q_ld,
                                        size_t q_out_ld, const void* k, void* k_out, const void* k_gain,
                                        uint32_t n_kv_heads, size_t k_ld, size_t k_out_ld, const int32_t* positions,
                                        const double* inv_freq, uint32_t rotary_dim, uint32_t rows, uint32_t head_dim,
                                        float eps, int32_t dtype, uint32_t flags, void* hip_stream) {
  if (rows == 0 || head_dim == 0 || n_q_heads == 0 || !q || !q_out) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer or zero size");
  if ((n_kv_heads != 0) != (k != nullptr) || (n_kv_heads != 0) != (k_out != nullptr))
    return mfail(BCT_ERR_INVALID_ARG, "k, k_out and n_kv_heads: all or none");
  if (dtype != BCT_F32 && dtype != BCT_BF16) return mfail(BCT_ERR_UNSUPPORTED, "dtype must be BCT_F32 or BCT_BF16");
  if (flags & ~(BCTM_HEAD_NORM | BCTM_ROPE_INTERLEAVED)) return mfail(BCT_ERR_INVALID_ARG, "unknown flag");
  const bool norm = (flags & BCTM_HEAD_NORM) != 0;
  if (!norm && rotary_dim == 0) return mfail(BCT_ERR_INVALID_ARG, "neither a norm nor a rotation");
  if (!norm && (q_gain || k_gain)) return mfail(BCT_ERR_INVALID_ARG, "a gain needs BCTM_HEAD_NORM");
  if (norm && !(eps >= 0.f)) return mfail(BCT_ERR_INVALID_ARG, "eps must not be negative");
  if (head_dim % 16 != 0 || head_dim > 256) return mfail(BCT_ERR_UNSUPPORTED, "head_dim must be a multiple of 16, at most 256");
  if (rotary_dim % 16 != 0 || rotary_dim > head_dim)
    return mfail(BCT_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 16, at most head_dim");
  if ((rotary_dim != 0) != (positions != nullptr) || (rotary_dim != 0) != (inv_freq != nullptr))
    return mfail(BCT_ERR_INVALID_ARG, "positions, inv_freq and rotary_dim: all or none");
  const uint64_t size = dtype == BCT_F32 ? 4 : 2, wq = (uint64_t)n_q_heads * head_dim, wk = (uint64_t)n_kv_heads * head_dim;
  if ((uint64_t)n_q_heads + n_kv_heads > 0xFFFFFFu) return mfail(BCT_ERR_UNSUPPORTED, "too many heads");
  const size_t widest_q = q_ld > q_out_ld ? q_ld : q_out_ld, widest_k = k_ld > k_out_ld ? k_ld : k_out_ld;
  if ((widest_q > widest_k ? widest_q : widest_k) > (1ull << 48) / rows) return mfail(BCT_ERR_UNSUPPORTED, "matrix too large");
  if (q_ld < wq || q_out_ld < wq || (k && (k_ld < wk || k_out_ld < wk)))
    return mfail(BCT_ERR_INVALID_ARG, "a row distance below the width of the heads");
  if (!al16(q) || !al16(q_out) || !al16(q_gain) || !al16(k) || !al16(k_out) || !al16(k_gain) || !al16(inv_freq) ||
      q_ld * size % 16 || q_out_ld * size % 16 || (k && (k_ld * size % 16 || k_out_ld * size % 16)))
    return mfail(BCT_ERR_MISALIGNED, "pointers and row distances must be 16-byte aligned");
  auto clash = [&](const void* out, uint64_t wo, uint32_t ldo, const void* in, uint64_t wi, uint32_t ldi, bool own) {
    if (own && out == in && ldo == ldi) return false;   // in place
    return rows_overlap(out, wo, ldo, in, wi, ldi, rows, size);
  };
  if (clash(q_out, wq, q_out_ld, q, wq, q_ld, true) ||
      (k && (clash(k_out, wk, k_out_ld, k, wk, k_ld, true) || clash(q_out, wq, q_out_ld, k, wk, k_ld, false) ||
             clash(k_out, wk, k_out_ld, q, wq, q_ld, false) || clash(q_out, wq, q_out_ld, k_out, wk, k_out_ld, false))))
    return mfail(BCT_ERR_INVALID_ARG, "an output overlaps an input other than its own, or the other output");
  const RopeCall c = {{q, q_out, q_gain, q_ld, q_out_ld, n_q_heads}, {k, k_out, k_gain, k_ld, k_out_ld, n_kv_heads},
                      positions, inv_freq, rotary_dim, rows, head_dim, eps, (hipStream_t)hip_stream};
  const RopePairs pairs = rotary_dim == 0 ? kNoRotation : flags & BCTM_ROPE_INTERLEAVED ? kNeighbours : kHalves;
  return dtype == BCT_F32 ? rope_form<F32>(c, norm, pairs) : rope_form<BF16>(c, norm, pairs);
}
