// The next token of each sequence drawn from its logits (gfx950): temperature, top-k, top-p and min-p of each row's own, and
// one uniform number a row.
//
//   tokens in descending order of their logit l, equal ones by index; those that are NaN or -inf never
//   w = exp((l - max) / T),  cum(j) = w_1 + .. + w_j
//   n = the least of  top_k,  the fewest with cum(n) >= top_p * cum(top_k),  how many have w >= min_p;  at least 1
//   drawn: the first j with cum(j) > u * cum(n)
//
// No sort: what is asked of the order is only where cumulated weights or counts pass a threshold.  A histogram of the row
// over 1/64 octaves of w, with the count and the weight of each bin, says in which bin that is; a histogram of the keys of
// that bin alone, once more where they are many, at which logit; and equal logits have equal weights, so the rest is a
// division.  A token is a whole number, so the sums must not depend on an order of additions, nor on fp32 roundings: weights
// are whole multiples of 2^-S, S at least 40 (a bit over half the digits of an fp64), added as 64-bit integers.
#include <math.h>

#include "bct_device.h"
#include "bct_model_internal.h"

namespace bct {

namespace {

constexpr uint32_t kThreads = 1024;
constexpr uint32_t kPerOctave = 64, kOctaves = 47, kBins = kPerOctave * kOctaves, kBinsEach = (kBins + kThreads - 1) / kThreads;
constexpr uint32_t kSub = 1024;    // bins of keys, and blocks of indexes: one a thread
constexpr uint32_t kMaxVocab = 1u << 22;

typedef unsigned long long u64;

struct SampleArgs {
  const void* logits;
  size_t ld;
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* ids;
  float* prob;
  uint32_t N, S;   // S: weights are multiples of 2^-S
};

// Keys order like the logits, as integers: 32 bits of an fp32, 16 of a bf16.
template <typename DT>
struct Key;
template <>
struct Key<F32> {
  static constexpr uint32_t kMinusInf = 0x007FFFFFu, kInf = 0xFF800000u;
  static __device__ __forceinline__ uint32_t of(float l) {
    const uint32_t b = __float_as_uint(l + 0.0f);   // -0 is 0
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
  }
  static __device__ __forceinline__ float value(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }
};
template <>
struct Key<BF16> {
  static constexpr uint32_t kMinusInf = 0x007Fu, kInf = 0xFF80u;
  static __device__ __forceinline__ uint32_t of(float l) { return Key<F32>::of(l) >> 16; }
  static __device__ __forceinline__ float value(uint32_t k) {
    const uint32_t b = k ^ ((k >> 15) ? 0x8000u : 0xFFFFu);
    return __uint_as_float(b << 16);
  }
};
template <typename DT>
__device__ __forceinline__ bool allowed(uint32_t key) { return key > Key<DT>::kMinusInf && key <= Key<DT>::kInf; }

// A row's weights: 2^y with y = (l - max) * log2(e) / T.
struct Weigher {
  float top;   // the largest logit
  double c;    // log2(e) / T
  uint32_t S;
  // at least -1000, which is as good as no weight; the largest logit (an infinity too) has 0
  __device__ __forceinline__ double octaves(float l) const { return l == top ? 0.0 : fmax(((double)l - (double)top) * c, -1000.0); }
  static __device__ __forceinline__ uint32_t bin(double y) { return min((uint32_t)(-y * kPerOctave), kBins); }   // kBins: none
  // 2^(y + S): the fraction of y by its Taylor series up to degree 10, within 2e-13
  __device__ __forceinline__ double scaled(double y) const {
    const double n = rint(y), f = y - n;
    double p = 7.054911620801121e-09;
    p = __builtin_fma(p, f, 1.0178086009239696e-07);
    p = __builtin_fma(p, f, 1.3215486790144305e-06);
    p = __builtin_fma(p, f, 1.5252733804059838e-05);
    p = __builtin_fma(p, f, 0.00015403530393381606);
    p = __builtin_fma(p, f, 0.0013333558146428441);
    p = __builtin_fma(p, f, 0.009618129107628477);
    p = __builtin_fma(p, f, 0.055504108664821576);
    p = __builtin_fma(p, f, 0.2402265069591007);
    p = __builtin_fma(p, f, 0.6931471805599453);
    p = __builtin_fma(p, f, 1.0);
    return ldexp(p, (int)n + (int)S);
  }
  // rounded to a whole number by adding 2^52, whose last place is 1 (S is at most 46)
  __device__ __forceinline__ u64 weight(double y) const {
    return (u64)__double_as_longlong(scaled(y) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
  }
};

// f(index, logit) for every logit of the row, 16 bytes a lane where the row is aligned.
template <typename DT, bool VEC, typename F>
__device__ __forceinline__ void each_logit(const typename DT::elem* row, uint32_t N, F f) {
  constexpr uint32_t E = DT::kElemsPerVec;
  const uint32_t nvec = VEC ? N / E : 0u;
  for (uint32_t v0 = threadIdx.x; v0 < nvec; v0 += 4 * kThreads) {
    u32x4 raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (v0 + i * kThreads < nvec) raw[i] = *(const u32x4*)(row + (size_t)(v0 + i * kThreads) * E);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (v0 + i * kThreads < nvec) {
        float l[E];
        unpack16<DT>(raw[i], l);
#pragma unroll
        for (uint32_t e = 0; e < E; ++e) f((v0 + i * kThreads) * E + e, l[e]);
      }
  }
  for (uint32_t j = nvec * E + threadIdx.x; j < N; j += kThreads) f(j, load_elem(row, j));
}

struct Sums {
  uint32_t count;
  u64 mass;
};

struct SampleShared {
  u64 mass[kBins + 1];        // of the bins before each; the last entry: of all
  uint32_t count[kBins + 1];
  u64 sub_mass[kSub];
  uint32_t sub_count[kSub];
  u64 wave_mass[kThreads / 64];
  uint32_t wave_count[kThreads / 64];
  uint32_t found[2];
  uint32_t range[2];
};

// What the threads before this one hold, and what all hold.
__device__ __forceinline__ Sums before_thread(SampleShared& s, Sums mine, Sums* all) {
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  Sums run = mine;
#pragma unroll
  for (uint32_t o = 1; o < 64; o *= 2) {
    const uint32_t c = __shfl_up(run.count, o, 64);
    const u64 m = __shfl_up(run.mass, o, 64);
    if (lane >= o) {
      run.count += c;
      run.mass += m;
    }
  }
  __syncthreads();   // the last call's sums have been read
  if (lane == 63) {
    s.wave_count[wave] = run.count;
    s.wave_mass[wave] = run.mass;
  }
  __syncthreads();
  Sums before = {run.count - mine.count, run.mass - mine.mass}, total = {0u, 0ull};
#pragma unroll
  for (uint32_t w = 0; w < kThreads / 64; ++w) {
    if (w < wave) {
      before.count += s.wave_count[w];
      before.mass += s.wave_mass[w];
    }
    total.count += s.wave_count[w];
    total.mass += s.wave_mass[w];
  }
  *all = total;
  return before;
}

// The least key in (none, top] for which `is` holds, which holds for top and from some key on: 64 tries a round, by the
// lanes of one wavefront.
template <typename P>
__device__ __forceinline__ uint32_t least_key(uint32_t none, uint32_t top, P is) {
  uint32_t lo = none, hi = top;   // does not hold at lo (or lo is no key), holds at hi
  while (hi - lo > 1) {
    const uint32_t step = (hi - lo - 1) / 64 + 1;
    const u64 at = (u64)lo + (u64)step * (threadIdx.x % 64 + 1);
    const u64 yes = __ballot(at >= hi || is((uint32_t)at));
    const uint32_t first = __builtin_ctzll(yes);   // lane 63 always says yes: lo + 64 * step >= hi
    const u64 from = (u64)lo + (u64)step * first, to = from + step;
    hi = to < hi ? (uint32_t)to : hi;
    lo = (uint32_t)from;
  }
  return hi;
}

struct Place {   // a logit in the order of the row
  uint32_t key;
  Sums before;   // of the larger ones
  uint32_t equal;   // how many have this key
};

// The logit at which the counts (by_count) or weights cumulated in the row's order reach `threshold`, at least 1 and at
// most what all of them have.
template <typename DT, bool VEC>
__device__ Place place_of(SampleShared& s, const typename DT::elem* row, uint32_t N, const Weigher& w, uint32_t top_key,
                          bool by_count, u64 threshold) {
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < kBins; b += kThreads) {
    const u64 from = by_count ? s.count[b] : s.mass[b], to = by_count ? s.count[b + 1] : s.mass[b + 1];
    if (from < threshold && threshold <= to) s.found[0] = b;
  }
  __syncthreads();
  const uint32_t bin = s.found[0];
  Place at;
  at.before = {s.count[bin], s.mass[bin]};
  // the bin's keys, smallest and largest
  if (threadIdx.x < 64) {
    const uint32_t k = least_key(Key<DT>::kMinusInf, top_key, [&](uint32_t key) { return w.bin(w.octaves(Key<DT>::value(key))) <= bin; });
    if (threadIdx.x == 0) s.range[0] = k;
  } else if (threadIdx.x < 128) {
    uint32_t k = top_key + 1;
    if (bin > 0) k = least_key(Key<DT>::kMinusInf, top_key, [&](uint32_t key) { return w.bin(w.octaves(Key<DT>::value(key))) < bin; });
    if (threadIdx.x == 64) s.range[1] = k - 1;
  }
  __syncthreads();
  uint32_t lo = s.range[0], hi = s.range[1];
  for (;;) {
    uint32_t shift = 0;
    while (((hi - lo) >> shift) >= kSub) ++shift;
    s.sub_count[threadIdx.x] = 0;
    s.sub_mass[threadIdx.x] = 0;
    __syncthreads();
    each_logit<DT, VEC>(row, N, [&](uint32_t, float l) {
      const uint32_t key = Key<DT>::of(l);
      if (key >= lo && key <= hi) {
        atomicAdd(&s.sub_count[(hi - key) >> shift], 1u);
        atomicAdd(&s.sub_mass[(hi - key) >> shift], w.weight(w.octaves(l)));
      }
    });
    __syncthreads();
    Sums mine = {s.sub_count[threadIdx.x], s.sub_mass[threadIdx.x]}, all;
    const Sums ahead = before_thread(s, mine, &all);
    const u64 from = by_count ? at.before.count + ahead.count : at.before.mass + ahead.mass, to = from + (by_count ? mine.count : mine.mass);
    if (from < threshold && threshold <= to) {
      s.found[1] = threadIdx.x;
      s.sub_count[0] = ahead.count;   // both have been read by their threads before the barriers in before_thread
      s.sub_mass[0] = ahead.mass;
      s.sub_count[1] = mine.count;
    }
    __syncthreads();
    at.before.count += s.sub_count[0];
    at.before.mass += s.sub_mass[0];
    at.equal = s.sub_count[1];
    const uint32_t f = s.found[1], top = hi - (f << shift), span = (1u << shift) - 1;
    __syncthreads();
    hi = top;
    lo = top - lo > span ? top - span : lo;
    if (shift == 0) break;
  }
  at.key = hi;
  return at;
}

template <typename DT, bool VEC>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  typedef typename DT::elem elem;
  __shared__ SampleShared s;
  const uint32_t r = blockIdx.x, N = a.N;
  const elem* row = (const elem*)a.logits + (size_t)r * a.ld;

  // the largest logit
  uint32_t top_key = 0;
  each_logit<DT, VEC>(row, N, [&](uint32_t, float l) {
    const uint32_t key = Key<DT>::of(l);
    if (allowed<DT>(key)) top_key = max(top_key, key);
  });
#pragma unroll
  for (uint32_t o = 1; o < 64; o *= 2) top_key = max(top_key, (uint32_t)__shfl_xor(top_key, o, 64));
  if (threadIdx.x % 64 == 0) s.wave_count[threadIdx.x / 64] = top_key;
  __syncthreads();
#pragma unroll
  for (uint32_t i = 0; i < kThreads / 64; ++i) top_key = max(top_key, s.wave_count[i]);
  if (top_key == 0) {   // no token is left
    if (threadIdx.x == 0) {
      a.ids[r] = -1;
      if (a.prob) a.prob[r] = 0.f;
    }
    return;
  }

  const float T = a.temperature ? a.temperature[r] : 1.0f;
  uint32_t key = top_key, nth = 1;   // the token drawn: the nth with this key
  float prob = 1.0f;
  if (T > 0.f) {
    const Weigher w = {Key<DT>::value(top_key), 1.4426950408889634074 / (double)T, a.S};
    for (uint32_t b = threadIdx.x; b <= kBins; b += kThreads) {
      s.count[b] = 0;
      s.mass[b] = 0;
    }
    __syncthreads();
    each_logit<DT, VEC>(row, N, [&](uint32_t, float l) {
      const uint32_t k = Key<DT>::of(l);
      if (!allowed<DT>(k)) return;
      const double y = w.octaves(l);
      const uint32_t b = w.bin(y);
      if (b >= kBins) return;   // below 2^-47: no weight
      const u64 m = w.weight(y);
      // where a wavefront's logits are all equal, one lane adds them
      const uint32_t first = __builtin_amdgcn_readfirstlane(k);
      const u64 here = __ballot(1), same = __ballot(k == first);
      if (here == same) {
        const uint32_t n = __popcll(here);
        if (threadIdx.x % 64 == __builtin_ctzll(here)) {
          atomicAdd(&s.count[b], n);
          atomicAdd(&s.mass[b], m * n);
        }
      } else {
        atomicAdd(&s.count[b], 1u);
        atomicAdd(&s.mass[b], m);
      }
    });
    __syncthreads();
    // sums of the bins before each
    Sums bins[kBinsEach], mine = {0u, 0ull}, all;
#pragma unroll
    for (uint32_t i = 0; i < kBinsEach; ++i) {
      const uint32_t b = threadIdx.x * kBinsEach + i;
      bins[i] = {b < kBins ? s.count[b] : 0u, b < kBins ? s.mass[b] : 0ull};
      mine.count += bins[i].count;
      mine.mass += bins[i].mass;
    }
    Sums before = before_thread(s, mine, &all);
#pragma unroll
    for (uint32_t i = 0; i < kBinsEach; ++i) {
      const uint32_t b = threadIdx.x * kBinsEach + i;
      if (b <= kBins) {
        s.count[b] = before.count;
        s.mass[b] = before.mass;
      }
      before.count += bins[i].count;
      before.mass += bins[i].mass;
    }
    if (threadIdx.x == 0) {
      s.count[kBins] = all.count;
      s.mass[kBins] = all.mass;
    }
    __syncthreads();

    // the weight that is kept, of the first so many
    u64 kept = all.mass;
    const int32_t k = a.top_k ? a.top_k[r] : 0;
    if (k > 0 && (uint32_t)k < all.count) {
      const Place at = place_of<DT, VEC>(s, row, N, w, top_key, true, (u64)k);
      kept = at.before.mass + (k - at.before.count) * w.weight(w.octaves(Key<DT>::value(at.key)));
    }
    const float p = a.top_p ? a.top_p[r] : 1.0f;
    const u64 of_k = kept;
    if (p < 1.f) {
      // cum >= p * cum(k): p as a multiple of 2^-64, the product's whole part and whether there is more
      const u64 p64 = p > 0.f ? (u64)((double)p * 18446744073709551616.0) : 0ull;
      const u64 need = __umul64hi(of_k, p64) + (of_k * p64 != 0 ? 1 : 0);
      const u64 threshold = need > 0 ? need : 1;
      const Place at = place_of<DT, VEC>(s, row, N, w, top_key, false, threshold);
      const u64 m = w.weight(w.octaves(Key<DT>::value(at.key)));
      kept = at.before.mass + (threshold - at.before.mass + m - 1) / m * m;
    }
    const float mp = a.min_p ? a.min_p[r] : 0.0f;
    if (mp > 0.f) {
      const u64 one = 1ull << a.S;
      u64 of_m = one;   // beyond 1 nothing has as much: the first
      if (mp <= 1.f) {
        const u64 least = (u64)ceil((double)mp * (double)one);
        __syncthreads();
        if (threadIdx.x < 64) {
          const uint32_t from = least_key(Key<DT>::kMinusInf, top_key, [&](uint32_t key) { return w.weight(w.octaves(Key<DT>::value(key))) >= least; });
          if (threadIdx.x == 0) s.range[0] = from;
        }
        __syncthreads();
        const uint32_t from = s.range[0], b = min(w.bin(w.octaves(Key<DT>::value(from))), kBins - 1);
        Sums inside = {0u, 0ull}, sum;
        each_logit<DT, VEC>(row, N, [&](uint32_t, float l) {
          const uint32_t key = Key<DT>::of(l);
          if (key < from || key > top_key) return;
          const double y = w.octaves(l);
          if (w.bin(y) == b) inside.mass += w.weight(y);
        });
        before_thread(s, inside, &sum);
        of_m = s.mass[b] + sum.mass;
      }
      kept = min(kept, of_m);
    }

    const float u = a.u[r];
    const u64 u64ths = u > 0.f ? u < 1.f ? (u64)((double)u * 18446744073709551616.0) : ~0ull : 0ull;
    const u64 threshold = __umul64hi(kept, u64ths) + 1;
    const Place at = place_of<DT, VEC>(s, row, N, w, top_key, false, threshold);
    const double y = w.octaves(Key<DT>::value(at.key));
    const u64 m = w.weight(y);
    key = at.key;
    nth = (uint32_t)((threshold - at.before.mass + m - 1) / m);
    prob = (float)(w.scaled(y) / (double)kept);
  }

  // the nth logit with this key in the order of the indexes: how many each block of indexes has, then inside one block
  uint32_t bits = 6;
  while ((N - 1) >> bits >= kSub) ++bits;
  s.sub_count[threadIdx.x] = 0;
  __syncthreads();
  each_logit<DT, VEC>(row, N, [&](uint32_t j, float l) {
    if (Key<DT>::of(l) == key) atomicAdd(&s.sub_count[j >> bits], 1u);
  });
  __syncthreads();
  Sums mine = {s.sub_count[threadIdx.x], 0ull}, all;
  const Sums before = before_thread(s, mine, &all);
  if (before.count < nth && nth <= before.count + mine.count) {
    s.found[0] = threadIdx.x;
    s.found[1] = nth - before.count;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    uint32_t left = s.found[1];
    const uint32_t from = s.found[0] << bits;
    for (uint32_t at = from; at < from + (1u << bits); at += 64) {
      const uint32_t j = at + threadIdx.x;
      const u64 yes = __ballot(j < N && Key<DT>::of(load_elem(row, j < N ? j : N - 1)) == key);
      const uint32_t n = __popcll(yes);
      if (left <= n) {
        // the lane that is the left-th of them
        if ((yes >> threadIdx.x & 1) && __popcll(yes & ((2ull << threadIdx.x) - 1)) == left) a.ids[r] = (int32_t)j;
        break;
      }
      left -= n;
    }
    if (threadIdx.x == 0 && a.prob) a.prob[r] = prob;
  }
}

}  // namespace
}  // namespace bct

using namespace bct;

extern "C" bct_status bctm_sample(const void* logits, size_t ld, const float* temperature, const int32_t* top_k,
                                  const float* top_p, const float* min_p, const float* u, int32_t* ids, float* prob,
                                  uint32_t rows, uint32_t N, int32_t dtype, void* hip_stream) {
  if (!logits || !u || !ids || rows == 0 || N == 0) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer or zero size");
  if (dtype != BCT_F32 && dtype != BCT_BF16) return mfail(BCT_ERR_UNSUPPORTED, "dtype must be BCT_F32 or BCT_BF16");
  if (ld < N) return mfail(BCT_ERR_INVALID_ARG, "ld below N");
  if (N > kMaxVocab) return mfail(BCT_ERR_UNSUPPORTED, "more than 4194304 tokens");
  if (rows > 0x7FFFFFFFu || ld > (SIZE_MAX / 8) / rows) return mfail(BCT_ERR_UNSUPPORTED, "matrix too large");
  const size_t size = dtype == BCT_F32 ? 4 : 2;
  if ((uintptr_t)logits % size) return mfail(BCT_ERR_MISALIGNED, "logits: aligned to their type");
  uint32_t log2n = 0;
  while ((1u << log2n) < N) ++log2n;
  const SampleArgs a = {logits, ld, temperature, top_p, min_p, u, top_k, ids, prob, N, log2n <= 16 ? 46u : 62u - log2n};
  const bool vec = al16(logits) && ld * size % 16 == 0;
  const auto kernel = dtype == BCT_F32 ? (vec ? sample_kernel<F32, true> : sample_kernel<F32, false>)
                                       : (vec ? sample_kernel<BF16, true> : sample_kernel<BF16, false>);
  hipLaunchKernelGGL(kernel, dim3(rows), dim3(kThreads), 0, (hipStream_t)hip_stream, a);
  return launched("sample");
}
