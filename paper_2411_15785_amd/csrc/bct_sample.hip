// The next token of each sequence drawn from its logits (gfx950): temperature, top-k, top-p and min-p of each row's own, and
// one uniform number a row.
//
//   tokens in descending order of their logit l, equal ones by index; those that are NaN or -inf never
//   w = exp((l - max) / T),  cum(j) = w_1 + .. + w_j
//   n = the least of  top_k,  the fewest with cum(n) >= top_p * cum(top_k),  how many have w >= min_p;  at least 1
//   drawn: the first j with cum(j) > u * cum(n)
//
// No sort: what is asked of the order is only where cumulated weights or counts pass a threshold, and histograms tell that.
// A token is a whole number, so the sums must not depend on an order of additions, nor on fp32 roundings: weights are whole
// multiples of 2^-S, S at least 40, added as 64-bit integers.
//   bf16   a value is one of 65536, and those with a weight seldom span more than 36864 of them (not where logits are beyond
//          2^17), so the row is counted by value, exactly, in 144 KB of LDS, and a weight is worked out for each value that
//          occurs instead of for each token.  Sums over groups of 128 values say in which group the threshold is passed, the
//          counts of that group at which value.
//   fp32   a histogram of weights over 1/64 octaves of w; the bin where the threshold is passed is gathered and divided
//          further by value.
// Equal values have equal weights, so the rest is a division, and the token the nth with its value in the order of the indexes.
// One workgroup a row, which it keeps in registers (bf16 up to 131072 tokens, fp32 65536; beyond, it is read again).
// Bound by the latency of a workgroup's steps, with long rows by its compute unit: loading a row, counting it in LDS, the 64-bit
// weights of fp32 tokens.  us in a graph, temperature and top-p: bf16 1 x 32000 15.5, 32 x 32000 16, 24 x 65536 19, 128 x 131072 29.6,
// 32 x 131072 26.5, 152064 38, 262144 53; fp32 24 x 4096 15.5, 32000 24, 50001 34 (this size spills 21 registers), 131072 87; with temperature
// alone fp32 32000 20, 50001 30, 131072 78.
#include <math.h>

#include "bct_device.h"
#include "bct_model_internal.h"

namespace bct {

namespace {

constexpr uint32_t kThreads = 1024;
constexpr uint32_t kSub = 1024;      // bins of keys, and blocks of indexes: one a thread
constexpr uint32_t kGroup = 128, kGroups = 65536 / kGroup, kWindow = 288;   // bf16 values of a group; groups counted at a time
constexpr uint32_t kList = 4096, kFew = kThreads / 8;
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

// Keys order like the logits, as integers: 32 bits of an fp32, 16 of a bf16; 2^31 or 2^15 is zero of either sign.  A NaN lies
// beyond the infinities.
template <typename DT>
struct Key;
template <>
struct Key<F32> {
  static constexpr uint32_t kMinusInf = 0x00800000u, kInf = 0xFF800000u;
  static __device__ __forceinline__ uint32_t of(uint32_t bits) {
    const uint32_t sign = (uint32_t)((int32_t)bits >> 31);
    return (((bits & 0x7FFFFFFFu) ^ sign) - sign) ^ 0x80000000u;
  }
  static __device__ __forceinline__ float value(uint32_t k) {
    const int32_t v = (int32_t)(k ^ 0x80000000u);
    return __uint_as_float(v < 0 ? 0x80000000u | (uint32_t)-v : (uint32_t)v);
  }
};
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
template <>
struct Key<BF16> {
  static constexpr uint32_t kMinusInf = 0x0080u, kInf = 0xFF80u;
  static __device__ __forceinline__ uint32_t of(uint32_t bits) {   // two values of a word
    const i16x2 sign = __builtin_bit_cast(i16x2, bits) >> (int16_t)15;
    const i16x2 v = __builtin_bit_cast(i16x2, (bits & 0x7FFF7FFFu) ^ __builtin_bit_cast(uint32_t, sign)) - sign;
    return __builtin_bit_cast(uint32_t, v) ^ 0x80008000u;
  }
  static __device__ __forceinline__ float value(uint32_t k) {
    const int32_t v = (int32_t)k - 0x8000;
    return __uint_as_float((v < 0 ? 0x8000u | (uint32_t)-v : (uint32_t)v) << 16);
  }
};

// A row's weights: 2^(-s / 64) with s = 64 log2(e) (max - l) / T.
constexpr uint32_t kPerOctave = 64, kBins = kPerOctave * 47;   // 2^-47 and less is no weight
// ALL: the table has 2^S times the weight of every whole s, else 2^(-i / 64) for i < 64.
template <bool ALL>
struct Weigher {
  double top;  // the largest logit; where that is infinite, far above every other
  double c;    // 64 log2(e) / T
  uint32_t S;
  const double* table;
  __device__ __forceinline__ Weigher(float largest, float T, uint32_t S_, const double* table_)
      : top(largest < INFINITY ? (double)largest : 1e300), c(fmax(92.332482616893656877 / (double)T, 1e-290)), S(S_), table(table_) {}
  // the whole number next to s, and what it is beyond s; an infinite logit, which is the largest, has 0
  struct Parts {
    uint32_t b;
    double f;
  };
  __device__ __forceinline__ Parts parts(float l) const {
    const double s = fmin(fmax((top - (double)l) * c, 0.0), (double)kBins), n = rint(s);
    return {(uint32_t)n, n - s};
  }
  // 2^(S - s / 64): the whole part from the table, the rest by its Taylor series up to degree 4, within 4e-14
  __device__ __forceinline__ double scaled(Parts t) const {
    const double f = t.f;
    double p = 5.732851688640402e-10;
    p = __builtin_fma(p, f, 2.1173137155464774e-07);
    p = __builtin_fma(p, f, 5.864904955056169e-05);
    p = __builtin_fma(p, f, 0.010830424696249145);
    p = __builtin_fma(p, f, 1.0);
    return ALL ? p * table[t.b] : ldexp(p * table[t.b % kPerOctave], (int)S - (int)(t.b / kPerOctave));
  }
  // rounded to a whole number by adding 2^52, whose last place is 1 (S is at most 46)
  __device__ __forceinline__ u64 weight(Parts t) const {
    return (u64)__double_as_longlong(scaled(t) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
  }
  __device__ __forceinline__ u64 weight_of(float l) const { return weight(parts(l)); }
};
__device__ __forceinline__ void fill_octave(double* table) {   // a barrier follows
  if (threadIdx.x < kPerOctave) table[threadIdx.x] = exp2(-(double)threadIdx.x / kPerOctave);
}

struct Sums {
  uint32_t count;
  u64 mass;
};

struct WaveSums {
  u64 mass[kThreads / 64];
  uint32_t count[kThreads / 64];
};

// The value of the lane that the data-parallel-primitive control names, 0 where there is none or the row is not in ROWS: no
// trip through the LDS crossbar.
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ uint32_t other_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ u64 other_lane(u64 v) {
  return (u64)other_lane<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | other_lane<CTRL, ROWS>((uint32_t)v);
}
// What the lanes up to this one hold, of its row of 16 or of all: lanes 1, 2, 4 and 8 before (row_shr), then the last lane of the
// row before (row_bcast15 into rows 1 and 3) and of the second row (row_bcast31 into rows 2 and 3).
template <int LANES = 64, typename V>
__device__ __forceinline__ V up_to_lane(V run) {
  run += other_lane<0x111>(run);
  run += other_lane<0x112>(run);
  run += other_lane<0x114>(run);
  run += other_lane<0x118>(run);
  if (LANES == 64) {
    run += other_lane<0x142, 0xA>(run);
    run += other_lane<0x143, 0xC>(run);
  }
  return run;
}
template <int LANES = 64>
__device__ __forceinline__ Sums up_to_lane(Sums run) {
  return {up_to_lane<LANES>(run.count), up_to_lane<LANES>(run.mass)};
}
// The sum over eight lanes side by side: with lane ^ 1 and lane ^ 2 of its quad, then with the lane mirrored in the eight.
template <typename V>
__device__ __forceinline__ V of_eight(V v) {
  v += other_lane<0xB1>(v);
  v += other_lane<0x4E>(v);
  v += other_lane<0x141>(v);
  return v;
}
__device__ __forceinline__ u64 lane_of(u64 v, int lane) {
  return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
// What the threads before this one hold, and what all hold.
__device__ __forceinline__ Sums before_thread(WaveSums& s, Sums mine, Sums* all) {
  constexpr int W = kThreads / 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const Sums run = up_to_lane(mine);
  __syncthreads();   // the last call's sums have been read
  if (threadIdx.x % 64 == 63) {
    s.count[wave] = run.count;
    s.mass[wave] = run.mass;
  }
  __syncthreads();
  const Sums waves = up_to_lane<W>({s.count[threadIdx.x % W], s.mass[threadIdx.x % W]});
  Sums before = {run.count - mine.count, run.mass - mine.mass};
  if (wave > 0) {
    before.count += (uint32_t)__builtin_amdgcn_readlane((int)waves.count, wave - 1);
    before.mass += lane_of(waves.mass, wave - 1);
  }
  *all = {(uint32_t)__builtin_amdgcn_readlane((int)waves.count, W - 1), lane_of(waves.mass, W - 1)};
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

// What is asked of the order, one after the other: where top-k ends, where min-p, where top-p, and which token u draws.
enum Stage { kTopK, kMinP, kTopP, kDraw, kStages };

// The row's keys, NV 16-byte vectors a thread (two bf16 keys to a word); a token that is never drawn has one of at most
// kMinusInf.  ONE: that is the whole row, it is loaded once and stays; else it is loaded piece by piece for each pass.  Vector v
// has the tokens v * E and on; behind the last whole one, the first threads have one token each.
template <typename DT, int NV, bool ONE>
struct RowKeys {
  static constexpr uint32_t E = DT::kElemsPerVec, kLoad = kThreads * NV;   // vectors of a load
  static constexpr uint32_t kNone = E == 8 ? 0x00010001u : 1u;             // keys of no token
  typedef typename DT::elem elem;
  const elem* row;
  uint32_t N, loads, at;
  u32x4 k[NV];
  uint32_t last;

  __device__ __forceinline__ RowKeys(const elem* row_, uint32_t N_) : row(row_), N(N_) {
    loads = ONE ? 1 : (N / E + kLoad - 1) / kLoad;
    if (ONE) fetch(0);
  }
  __device__ __forceinline__ void load(uint32_t n) {   // the nth piece of the row
    if (!ONE) fetch(n);
  }
  static __device__ __forceinline__ uint32_t without_nan(uint32_t keys) {
    if constexpr (E == 8) return ((keys & 0xFFFFu) > Key<DT>::kInf ? 0u : keys & 0xFFFFu) | (keys >> 16 > Key<DT>::kInf ? 0u : keys & 0xFFFF0000u);
    else return keys > Key<DT>::kInf ? 0u : keys;
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    if constexpr (E == 8) return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
    else return max(a, b);
  }
  static __device__ __forceinline__ uint32_t largest_of(uint32_t keys) { return E == 8 ? max(keys & 0xFFFFu, keys >> 16) : keys; }
  uint32_t most;   // the largest keys of what is loaded
  __device__ __forceinline__ void fetch(uint32_t n) {
    at = n;
    const uint32_t nvec = N / E, v0 = n * kLoad + threadIdx.x;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t v = v0 + i * kThreads;
      k[i] = u32x4{~0u, ~0u, ~0u, ~0u};   // NaNs of the sign whose keys are the least
      if (v < nvec) {   // element by element as the row may begin anywhere; the compiler makes one load of 16 bytes of it
        const elem* p = row + (size_t)v * E;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (E == 8) k[i][e] = (uint32_t)p[2 * e] | (uint32_t)p[2 * e + 1] << 16;
          else k[i][e] = __float_as_uint(p[e]);
        }
      }
    }
    const uint32_t j = nvec * E + threadIdx.x;
    last = kNone;
    if (n == loads - 1 && threadIdx.x < E && j < N) {
      if constexpr (E == 8) last = Key<DT>::of(row[j] | 0xFFFF0000u);
      else last = Key<DT>::of(__float_as_uint(row[j]));
    }
    most = last;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        k[i][e] = Key<DT>::of(k[i][e]);
        most = larger(most, k[i][e]);
      }
    if (largest_of(most) > Key<DT>::kInf) {   // a NaN is among them
      last = without_nan(last);
      most = last;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          k[i][e] = without_nan(k[i][e]);
          most = larger(most, k[i][e]);
        }
    }
  }
  // whether any thread has an ith vector
  __device__ __forceinline__ bool there(uint32_t i) const { return at * kLoad + i * kThreads < N / E; }
  // f(vector, index of its first token) for the vectors of a thread, and for the token left over, in a vector of its own
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (E == 4 || i == 0 || there(i)) f(k[i], (at * kLoad + i * kThreads + threadIdx.x) * E);
    if (N % E != 0 && threadIdx.x < 64) f(u32x4{last, kNone, kNone, kNone}, N / E * E + threadIdx.x);
  }
  // The same for a long f: it stands there for four vectors, which are copied one four after the other.  What f makes of a key is
  // not kept from one stage for the next, the registers are full without.
  template <typename F>
  __device__ __forceinline__ void each_four(F f) const {
#pragma unroll 1
    for (uint32_t n = 0; n < NV && (n == 0 || there(n)); n += 4) {
      uint32_t now[4][4];
#pragma unroll
      for (int m = 0; m < NV; m += 4)
        if (NV <= 4 || n == m) {
#pragma unroll
          for (int i = 0; i < 16 && i < 4 * NV; ++i) {
            now[i / 4][i % 4] = k[m + i / 4][i % 4];
            asm volatile("" : "+v"(now[i / 4][i % 4]));
          }
        }
#pragma unroll
      for (int i = 0; i < 4 && i < NV; ++i) f(u32x4{now[i][0], now[i][1], now[i][2], now[i][3]});
    }
    if (N % E != 0 && threadIdx.x < 64) f(u32x4{last, kNone, kNone, kNone});
  }
  // g(key) for every token of a vector
  template <typename G>
  static __device__ __forceinline__ void tokens(u32x4 v, G g) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (E == 8) {
        g(v[e] & 0xFFFFu);
        g(v[e] >> 16);
      } else {
        g(v[e]);
      }
    }
  }
  // The key of one token, read from the row; at most kMinusInf for none.
  __device__ __forceinline__ uint32_t key_at(uint32_t j) const {
    uint32_t key;
    if constexpr (E == 8) key = Key<DT>::of(row[j]) & 0xFFFFu;
    else key = Key<DT>::of(__float_as_uint(row[j]));
    return key > Key<DT>::kInf ? 0u : key;
  }
  // How many tokens of a vector have this key.
  static __device__ __forceinline__ uint32_t how_many(u32x4 v, uint32_t key) {
    uint32_t others = 0;
    if constexpr (E == 8) {
      const uint32_t both = key | key << 16;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        others += __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, v[e] ^ both), (u16x2){1, 1}));
      return 8 - (others & 0xFFFFu) - (others >> 16);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) others += v[e] == key ? 1u : 0u;
      return others;
    }
  }
  __device__ __forceinline__ uint32_t largest(uint32_t* waves) {   // over the row, for all threads
    uint32_t top = 0;
    for (uint32_t n = 0; n < loads; ++n) {
      load(n);
      top = max(top, largest_of(most));
    }
#pragma unroll
    for (uint32_t o = 1; o < 64; o *= 2) top = max(top, (uint32_t)__shfl_xor(top, o, 64));
    if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = top;
    __syncthreads();
    top = waves[threadIdx.x % (kThreads / 64)];
#pragma unroll
    for (uint32_t o = 1; o < kThreads / 64; o *= 2) top = max(top, (uint32_t)__shfl_xor(top, o, 64));
    return __builtin_amdgcn_readfirstlane(top);
  }
};

// The settings of a row, as the integers that sums are compared with.
struct Settings {
  float T;
  int32_t k;
  float p, min_p;
  u64 p64, u64ths;   // top_p and u as multiples of 2^-64
};
__device__ __forceinline__ u64 of_two_to_64(float x) { return (u64)((double)x * 18446744073709551616.0); }   // 0 < x < 1
__device__ __forceinline__ Settings settings_of(const SampleArgs& a, uint32_t r) {
  Settings s;
  s.T = a.temperature ? a.temperature[r] : 1.0f;
  s.k = a.top_k ? a.top_k[r] : 0;
  s.p = a.top_p ? a.top_p[r] : 1.0f;
  s.min_p = a.min_p ? a.min_p[r] : 0.0f;
  const float u = a.u[r];
  s.p64 = s.p > 0.f && s.p < 1.f ? of_two_to_64(s.p) : 0ull;
  s.u64ths = u > 0.f ? u < 1.f ? of_two_to_64(u) : ~0ull : 0ull;
  return s;
}
// The least cumulated weight that is top_p of `mass`: the product's whole part and one more if there is a rest; at least 1.
__device__ __forceinline__ u64 top_p_threshold(const Settings& s, u64 mass) {
  const u64 need = __umul64hi(mass, s.p64) + (mass * s.p64 != 0 ? 1 : 0);
  return need > 0 ? need : 1;
}
// How many tokens of weight m reach `threshold` above `before`, rounded up.
__device__ __forceinline__ u64 tokens_to(u64 threshold, u64 before, u64 m) { return (threshold - before + m - 1) / m; }

// The nth token with this key in the order of the indexes: how many each block of indexes has, then inside one block.
template <typename DT, int NV, bool ONE>
__device__ __forceinline__ void write_token(RowKeys<DT, NV, ONE>& keys, WaveSums& waves, uint32_t* blocks, uint32_t* found,
                                            uint32_t key, uint32_t nth, int32_t* id) {
  uint32_t bits = 6;
  while ((keys.N - 1) >> bits >= kSub) ++bits;
  blocks[threadIdx.x] = 0;
  __syncthreads();
  for (uint32_t n = 0; n < keys.loads; ++n) {
    keys.load(n);
    keys.each([&](u32x4 v, uint32_t index) {   // a vector's tokens lie in one block
      const uint32_t here = keys.how_many(v, key);
      if (here) atomicAdd(&blocks[index >> bits], here);
    });
  }
  __syncthreads();
  const uint32_t mine = blocks[threadIdx.x], run = up_to_lane(mine), lane = threadIdx.x % 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  if (lane == 63) waves.count[wave] = run;
  __syncthreads();
  const uint32_t sums = up_to_lane<kThreads / 64>(waves.count[threadIdx.x % (kThreads / 64)]);
  const uint32_t before = run - mine + (wave > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)sums, wave - 1) : 0u);
  if (before < nth && nth <= before + mine) {
    found[0] = threadIdx.x;
    found[1] = nth - before;
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    uint32_t left = found[1];
    const uint32_t from = found[0] << bits;
    for (uint32_t at = from; at < from + (1u << bits); at += 64) {
      const uint32_t j = at + lane;
      const u64 yes = __ballot(j < keys.N && keys.key_at(min(j, keys.N - 1)) == key);
      const uint32_t n = __popcll(yes);
      if (left <= n) {
        // the lane that is the left-th of them
        if ((yes >> lane & 1) && __popcll(yes & ((2ull << lane) - 1)) == left) *id = (int32_t)j;
        break;
      }
      left -= n;
    }
  }
}

__device__ __forceinline__ void write_none(const SampleArgs& a, uint32_t r) {
  if (threadIdx.x == 0) {
    a.ids[r] = -1;
    if (a.prob) a.prob[r] = 0.f;
  }
}

// ---------------------------------------------------------------- bf16: counted by value

struct CountShared {
  uint32_t count[kWindow * kGroup];   // of each value
  u64 mass[kGroups];                  // of each group of values; then of the groups above each
  uint32_t tokens[kGroups];
  uint32_t one[kSub];                 // counts of one group's values; blocks of indexes
  double octave[kPerOctave];
  WaveSums waves;
  uint32_t found[2], from_p, nth, key;
  Sums above;                         // the groups above the one that is looked at
  u64 kept, of_k;
  float prob;
};

// The values of a vector counted, those from `base` on, `span` of them; one of a wavefront's lanes adds for all where they
// have the same words.
__device__ __forceinline__ void count_values(uint32_t* count, u32x4 v, uint32_t base, uint32_t span) {
  const uint32_t first = __builtin_amdgcn_readfirstlane(v[0]);
  if (__ballot(v[0] == first) == ~0ull) {
#pragma unroll 1
    for (int e = 0; e < 8; ++e) {
      const uint32_t k = v[0] & 0xFFFFu;
      const bool same = __ballot(k == __builtin_amdgcn_readfirstlane(k)) == ~0ull;
      if (k - base < span && (!same || threadIdx.x % 64 == 0)) atomicAdd(&count[k - base], same ? 64u : 1u);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = v[i] >> 16 | (i < 3 ? v[(i + 1) % 4] << 16 : 0u);
    }
  } else {
    auto add = [&](uint32_t at) {   // in bytes
      if (at < 4 * span) atomicAdd((uint32_t*)((char*)count + at), 1u);
    };
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      add((v[e] << 2 & 0x3FFFCu) - 4 * base);
      add((v[e] >> 14 & 0x3FFFCu) - 4 * base);
    }
  }
}

template <int NV, bool ONE>
__global__ __launch_bounds__(kThreads) void sample_bf16_kernel(SampleArgs a) {
  __shared__ CountShared s;
  const uint32_t r = blockIdx.x, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  RowKeys<BF16, NV, ONE> keys((const uint16_t*)a.logits + (size_t)r * a.ld, a.N);
  auto clear = [&] {
    for (uint32_t i = threadIdx.x; i < kWindow * kGroup / 4; i += kThreads) ((u32x4*)s.count)[i] = u32x4{0u, 0u, 0u, 0u};
  };
  clear();
  if (threadIdx.x < kGroups) {
    s.mass[threadIdx.x] = 0;
    s.tokens[threadIdx.x] = 0;
  }
  fill_octave(s.octave);
  const Settings set = settings_of(a, r);
  const uint32_t top_key = keys.largest(s.waves.count);
  if (top_key <= Key<BF16>::kMinusInf) return write_none(a, r);

  if (!(set.T > 0.f)) {
    if (threadIdx.x == 0) {
      s.key = top_key;
      s.nth = 1;
      s.prob = 1.0f;
    }
  } else {
    const Weigher<false> w(Key<BF16>::value(top_key), set.T, a.S, s.octave);
    auto weight_of = [&](uint32_t k) -> u64 { return w.weight_of(Key<BF16>::value(k)); };
    const u64 one = 1ull << a.S;
    // values that are counted: those 47 octaves below the largest and less have no weight (the value there may be a step off)
    uint32_t cut = Key<BF16>::kMinusInf + 1;
    const double end = w.top - kBins / w.c;
    if (end > -3e38) cut = max(cut, (Key<BF16>::of(__float_as_uint((float)end) >> 16) & 0xFFFFu) - 2);

    if (threadIdx.x < 64 && set.min_p > 0.f && set.min_p <= 1.f) {   // the least value that has min_p
      const u64 need = (u64)ceil((double)set.min_p * (double)one);
      const uint32_t k = least_key(Key<BF16>::kMinusInf, top_key, [&](uint32_t k) { return weight_of(k) >= need; });
      if (lane == 0) s.from_p = k;
    }

    // Counted, and the counts added up into the groups' sums, a window of groups at a time from the largest value down
    const uint32_t g_cut = cut / kGroup;
    uint32_t g1 = top_key / kGroup, g0;
    bool one_window = true;
    for (;;) {
      g0 = g1 >= g_cut + kWindow ? g1 - kWindow + 1 : g_cut;
      for (uint32_t n = 0; n < keys.loads; ++n) {
        keys.load(n);
        keys.each_four([&](u32x4 v) { count_values(s.count, v, g0 * kGroup, (g1 - g0 + 1) * kGroup); });
      }
      __syncthreads();
      // a wavefront takes 128 values at a time, the next one the next
#pragma unroll 1
      for (uint32_t g = g0 + wave; g <= g1; g += 4 * (kThreads / 64)) {
        uint2 c[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
          c[i] = g + i * (kThreads / 64) <= g1 ? ((const uint2*)s.count)[(g + i * (kThreads / 64) - g0) * 64 + lane] : uint2{0u, 0u};
#pragma unroll 1
        for (uint32_t i = 0; i < 4; ++i) {
          const uint2 now = c[0];
          c[0] = c[1];
          c[1] = c[2];
          c[2] = c[3];
          if (__ballot((now.x | now.y) != 0) == 0) continue;
          const uint32_t of = g + i * (kThreads / 64), k = of * kGroup + 2 * lane;
          Sums t = {now.x + now.y, 0ull};
          if (t.count) t.mass = now.x * weight_of(k) + now.y * weight_of(k + 1);
          t = up_to_lane(t);
          if (lane == 63) {
            s.tokens[of] = t.count;
            s.mass[of] = t.mass;
          }
        }
      }
      __syncthreads();
      if (g0 == g_cut) break;
      one_window = false;
      g1 = g0 - 1;
      clear();
      __syncthreads();
    }
    // sums of the groups above each; thread t has group kGroups - 1 - t
    Sums mine = {0u, 0ull}, all;
    if (threadIdx.x < kGroups) mine = {s.tokens[kGroups - 1 - threadIdx.x], s.mass[kGroups - 1 - threadIdx.x]};
    const Sums above = before_thread(s.waves, mine, &all);
    if (threadIdx.x < kGroups) s.mass[kGroups - 1 - threadIdx.x] = above.mass;
    if (threadIdx.x == 0) s.kept = s.of_k = all.mass;   // the weight that is kept, of the first so many; what top-k leaves

    uint32_t from_p = 0;
#pragma unroll 1
    for (int stage = kTopK; stage < kStages; ++stage) {
      // the value where the counts (top-k) or weights cumulated in the row's order reach `threshold`, or the key of min-p
      u64 threshold = 0;
      const bool by_count = stage == kTopK;
      __syncthreads();
      const u64 kept = s.kept;
      if (stage == kTopK) {
        if (set.k <= 0 || (uint32_t)set.k >= all.count) continue;
        threshold = (u64)set.k;
      } else if (stage == kMinP) {
        if (!(set.min_p > 0.f)) continue;
        if (set.min_p > 1.f) {   // nothing has as much: the first
          if (threadIdx.x == 0) s.kept = min(kept, one);
          continue;
        }
        from_p = s.from_p;
        if (s.mass[from_p / kGroup] >= kept) continue;   // it cuts nothing off
      } else if (stage == kTopP) {
        threshold = top_p_threshold(set, s.of_k);
        if (!(set.p < 1.f) || threshold > kept) continue;
      } else {
        threshold = __umul64hi(kept, set.u64ths) + 1;
      }
      if (stage == kMinP) {
        if (threadIdx.x == 0) {
          s.found[0] = from_p / kGroup;
          s.above = {0u, s.mass[from_p / kGroup]};
        }
      } else {
        const u64 from = by_count ? above.count : above.mass, to = from + (by_count ? mine.count : mine.mass);
        if (from < threshold && threshold <= to) {
          s.found[0] = kGroups - 1 - threadIdx.x;
          s.above = above;
        }
      }
      if (!one_window && threadIdx.x < kGroup) s.one[threadIdx.x] = 0;
      __syncthreads();
      const uint32_t g = s.found[0];
      if (!one_window) {   // the group's counts once more
        for (uint32_t j0 = 0; j0 < keys.N; j0 += kThreads) {
          const uint32_t j = j0 + threadIdx.x, k = j < keys.N ? keys.key_at(j) : 0u;
          if (k / kGroup != g) continue;
          const u64 here = __ballot(1);
          const bool same = __ballot(k == __builtin_amdgcn_readfirstlane(k)) == here;
          if (!same || lane == __builtin_ctzll(here)) atomicAdd(&s.one[k % kGroup], same ? (uint32_t)__popcll(here) : 1u);
        }
        __syncthreads();
      }
      if (threadIdx.x < 64) {   // from the largest value down, two a lane
        const uint32_t i = kGroup - 1 - 2 * lane, k = g * kGroup + i;
        const uint32_t* counts = one_window ? s.count + (g - g0) * kGroup : s.one;
        const uint32_t n1 = counts[i], n0 = counts[i - 1];
        const u64 m1 = n1 ? weight_of(k) : 0ull, m0 = n0 ? weight_of(k - 1) : 0ull;
        const Sums hi = {n1, n1 * m1}, both = {n1 + n0, n1 * m1 + n0 * m0}, run = up_to_lane(both);
        Sums b = {s.above.count + run.count - both.count, s.above.mass + run.mass - both.mass};
        const u64 f = by_count ? b.count : b.mass, h = f + (by_count ? hi.count : hi.mass), t = f + (by_count ? both.count : both.mass);
        const bool here = stage == kMinP ? k == from_p || k - 1 == from_p : f < threshold && threshold <= t;
        if (here) {
          const bool second = stage == kMinP ? k != from_p : threshold > h;
          if (second) b = {b.count + hi.count, b.mass + hi.mass};
          const u64 m = second ? m0 : m1;
          if (stage == kTopK) {
            s.of_k = s.kept = b.mass + ((uint32_t)set.k - b.count) * m;
          } else if (stage == kMinP) {
            s.kept = min(kept, b.mass + (second ? n0 : n1) * m);
          } else if (stage == kTopP) {
            s.kept = min(kept, b.mass + tokens_to(threshold, b.mass, m) * m);
          } else {
            s.key = second ? k - 1 : k;
            s.nth = (uint32_t)tokens_to(threshold, b.mass, m);
            s.prob = (float)(w.scaled(w.parts(Key<BF16>::value(s.key))) / (double)kept);
          }
        }
      }
    }
  }
  __syncthreads();
  write_token(keys, s.waves, s.one, s.found, s.key, s.nth, a.ids + r);
  if (threadIdx.x == 0 && a.prob) a.prob[r] = s.prob;
}

// ---------------------------------------------------------------- fp32: weights over octaves

constexpr uint32_t kBinsEach = (kBins + kThreads - 1) / kThreads;
struct OctaveShared {
  u64 mass[kBins + 1];        // of the bins before each; the last entry: of all
  uint32_t count[kBins + 1];
  u64 sub_mass[kSub];
  uint32_t sub_count[kSub];
  uint32_t list[kList];       // the keys of one bin
  uint32_t row[kList];        // all keys that are weighed, where they are so few
  double octave[kPerOctave], table[kBins + 1];
  WaveSums waves;
  uint32_t found[2], range[2], listed, in_row, nth, key;
  u64 kept, above;
  float prob;
};

template <int NV, bool ONE>
__global__ __launch_bounds__(kThreads) void sample_f32_kernel(SampleArgs a) {
  __shared__ OctaveShared s;
  const uint32_t r = blockIdx.x, lane = threadIdx.x % 64;
  RowKeys<F32, NV, ONE> keys((const float*)a.logits + (size_t)r * a.ld, a.N);
  fill_octave(s.octave);
  const Settings set = settings_of(a, r);
  const uint32_t top_key = keys.largest(s.waves.count);
  if (top_key <= Key<F32>::kMinusInf) return write_none(a, r);

  if (!(set.T > 0.f)) {
    if (threadIdx.x == 0) {
      s.key = top_key;
      s.nth = 1;
      s.prob = 1.0f;
    }
  } else {
    const Weigher<true> w(Key<F32>::value(top_key), set.T, a.S, s.table);
    auto weight_of = [&](uint32_t k) -> u64 { return w.weight_of(Key<F32>::value(k)); };
    auto bin_of = [&](uint32_t k) -> uint32_t { return w.parts(Key<F32>::value(k)).b; };
    // The least key for which `is` holds, from some key on.  It lies next to the logit `near`, but for roundings: looked for
    // there, and among all keys where it is not.
    auto least_near = [&](double near, auto is) -> uint32_t {
      const uint32_t at = Key<F32>::of(__float_as_uint((float)near));
      const uint32_t none = Key<F32>::kMinusInf, lo = at > none + 1000 ? at - 1000 : none, hi = at < top_key - 1000 ? at + 1000 : top_key;
      const bool there = lo < hi && hi <= top_key && (lo == none || !is(lo)) && is(hi);
      return least_key(there ? lo : none, there ? hi : top_key, is);
    };
    auto least_of_bin = [&](uint32_t bin) -> uint32_t {   // of the bins up to this one
      return least_near(w.top - (bin + 0.5) / w.c, [&](uint32_t k) { return bin_of(k) <= bin; });
    };
    for (uint32_t b = threadIdx.x; b <= kBins; b += kThreads)
      s.table[b] = b < kBins ? ldexp(s.octave[b % kPerOctave], (int)a.S - (int)(b / kPerOctave)) : 0.0;
    __syncthreads();
    const u64 one = 1ull << a.S;
    if (threadIdx.x < 64 && set.min_p > 0.f && set.min_p <= 1.f) {   // the least key that has min_p
      const u64 need = (u64)ceil((double)set.min_p * (double)one);
      const uint32_t k = least_near(w.top + log2((double)set.min_p) * kPerOctave / w.c, [&](uint32_t k) { return weight_of(k) >= need; });
      if (lane == 0) s.range[0] = k;
    }
    __syncthreads();
    const uint32_t from_p = s.range[0];

    // f(key) for the keys of a gathered bin: from the list, or from the row where that is too short
    auto members = [&](auto f) {
      const bool listed = s.listed <= kList;
      const uint32_t n = listed ? s.listed : keys.N, lo = s.range[0], hi = s.range[1];
#pragma unroll 1
      for (uint32_t j = threadIdx.x; j < n; j += kThreads) {
        const uint32_t k = listed ? s.list[j] : keys.key_at(j);
        if (k >= lo && k <= hi) f(k);
      }
    };

    u64 kept = 0, of_k = 0;   // the weight that is kept, of the first so many; what top-k leaves
    uint32_t least = Key<F32>::kMinusInf + 1;   // the keys that are weighed: top-k's and all that equal its last
    u64 too_many = 0;                           // of those, how many it leaves out
    // Where few tokens are left, by a mask that comes with the logits or by top-k, they are listed and the row is not looked
    // at again.
    uint32_t drawable = 0;
    for (uint32_t n = 0; n < keys.loads; ++n) {
      keys.load(n);
      keys.each([&](u32x4 v, uint32_t) { keys.tokens(v, [&](uint32_t k) { drawable += k >= least ? 1u : 0u; }); });
    }
    Sums drawables;
    before_thread(s.waves, {drawable, 0ull}, &drawables);
    bool to_list = drawables.count <= kList, row_listed = false;
#pragma unroll 1
    for (int stage = kTopK; stage < kStages; ++stage) {
      const bool by_count = stage == kTopK;
      __syncthreads();
      if (to_list) {
        if (threadIdx.x == 0) s.in_row = 0;
        __syncthreads();
        for (uint32_t n = 0; n < keys.loads; ++n) {
          keys.load(n);
          keys.each([&](u32x4 v, uint32_t) {
            keys.tokens(v, [&](uint32_t k) {
              if (k >= least) {
                const uint32_t i = atomicAdd(&s.in_row, 1u);
                if (i < kList) s.row[i] = k;
              }
            });
          });
        }
        __syncthreads();
        row_listed = s.in_row <= kList;
        to_list = false;
      }
      if (by_count && (set.k <= 0 || (uint32_t)set.k >= keys.N)) continue;
      if (stage == kTopP && !(set.p < 1.f)) continue;
      Sums all = {0u, 0ull};
      if (stage <= kMinP) {
        // the histogram over octaves of the tokens from key `least` on, by count or by weight; each bin's sum, then that of
        // the bins before it
        for (uint32_t b = threadIdx.x; b <= kBins; b += kThreads) {
          s.count[b] = 0;
          s.mass[b] = 0;
        }
        __syncthreads();
        auto token = [&](uint32_t k) {
          const auto t = w.parts(Key<F32>::value(k));
          if (k < least || t.b >= kBins) return;
          if (by_count) atomicAdd(&s.count[t.b], 1u);
          else atomicAdd(&s.mass[t.b], w.weight(t));
        };
        for (uint32_t j = threadIdx.x; row_listed && j < s.in_row; j += kThreads) token(s.row[j]);
        for (uint32_t n = 0; !row_listed && n < keys.loads; ++n) {
          keys.load(n);
          keys.each_four([&](u32x4 v) {
            // where a wavefront's logits are all equal, one lane adds them
            bool same = true;
#pragma unroll
            for (int e = 0; e < 4; ++e) same = same && __ballot(v[e] == __builtin_amdgcn_readfirstlane(v[0])) == ~0ull;
            if (same) {
              const auto t = w.parts(Key<F32>::value(v[0]));
              if (v[0] >= least && t.b < kBins && lane == 0) {
                if (by_count) atomicAdd(&s.count[t.b], 256u);
                else atomicAdd(&s.mass[t.b], w.weight(t) * 256);
              }
            } else {
              keys.tokens(v, token);
            }
          });
        }
        __syncthreads();
        Sums bins[kBinsEach], mine = {0u, 0ull};
#pragma unroll
        for (uint32_t i = 0; i < kBinsEach; ++i) {
          const uint32_t b = threadIdx.x * kBinsEach + i;
          bins[i] = {b < kBins ? s.count[b] : 0u, b < kBins ? s.mass[b] : 0ull};
          mine.count += bins[i].count;
          mine.mass += bins[i].mass;
        }
        Sums before = before_thread(s.waves, mine, &all);
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
      }
      if (stage == kMinP) of_k = kept = all.mass - too_many * weight_of(least);
      // the value where the counts (top-k) or weights cumulated in the row's order reach `threshold`, or the key of min-p
      u64 threshold = 0;
      uint32_t bin = 0;
      if (by_count) {
        if ((uint32_t)set.k >= all.count) continue;
        threshold = (u64)set.k;
      } else if (stage == kMinP) {
        if (!(set.min_p > 0.f)) continue;
        if (set.min_p > 1.f) kept = min(kept, one);   // nothing has as much: the first
        bin = min(bin_of(max(from_p, least)), kBins - 1);
        if (set.min_p > 1.f || s.mass[bin] >= kept) continue;   // or it cuts nothing off
      } else if (stage == kTopP) {
        threshold = top_p_threshold(set, of_k);
        if (threshold > kept) continue;
      } else {
        threshold = __umul64hi(kept, set.u64ths) + 1;
      }
      if (stage != kMinP) {
        for (uint32_t b = threadIdx.x; b < kBins; b += kThreads) {
          const u64 from = by_count ? s.count[b] : s.mass[b], to = by_count ? s.count[b + 1] : s.mass[b + 1];
          if (from < threshold && threshold <= to) s.found[0] = b;
        }
        __syncthreads();
        bin = s.found[0];
      }
      // the bin's keys, smallest and largest, and their list
      if (threadIdx.x < 64) {
        const uint32_t k = least_of_bin(bin);
        if (threadIdx.x == 0) s.range[0] = max(k, least);
      } else if (threadIdx.x < 128) {
        const uint32_t k = bin > 0 ? least_of_bin(bin - 1) : top_key + 1;
        if (threadIdx.x == 64) s.range[1] = k - 1;
      } else if (threadIdx.x == 128) {
        s.listed = 0;
      }
      __syncthreads();
      uint32_t lo = s.range[0], hi = s.range[1];
      auto take = [&](uint32_t k) {
        if (k >= lo && k <= hi) {
          const uint32_t i = atomicAdd(&s.listed, 1u);
          if (i < kList) s.list[i] = k;
        }
      };
      for (uint32_t j = threadIdx.x; row_listed && j < s.in_row; j += kThreads) take(s.row[j]);
      for (uint32_t n = 0; !row_listed && n < keys.loads; ++n) {
        keys.load(n);
        keys.each([&](u32x4 v, uint32_t) {
          bool any = false;
#pragma unroll
          for (int e = 0; e < 4; ++e) any |= v[e] - lo <= hi - lo;
          if (any) keys.tokens(v, take);
        });
      }
      __syncthreads();
      if (stage == kMinP) {
        Sums inside = {0u, 0ull}, sum;
        members([&](uint32_t k) { inside.mass += k >= from_p ? weight_of(k) : 0ull; });
        before_thread(s.waves, inside, &sum);
        kept = min(kept, s.mass[bin] + sum.mass);
        continue;
      }
      Sums before = {s.count[bin], s.mass[bin]};
      uint32_t equal;
      const uint32_t few = s.listed;
      if (few <= kFew) {   // each key against every other, eight threads to a key
        if (threadIdx.x < few) {
          const uint32_t k = s.list[threadIdx.x];
          s.sub_mass[threadIdx.x] = by_count ? 1 : k >= least ? weight_of(k) : 0;
        }
        __syncthreads();
        const uint32_t i = min(threadIdx.x / 8, few - 1), k = s.list[i];
        u64 above = 0;
        uint32_t count = 0, same = 0;
        for (uint32_t j = threadIdx.x % 8; j < few; j += 8) {
          const uint32_t other = s.list[j];
          const u64 m = s.sub_mass[j];
          above += other > k ? m : 0;
          count += other > k ? 1u : 0u;
          same += other == k ? 1u : 0u;
        }
        above = of_eight(above);
        count = of_eight(count);
        same = of_eight(same);
        const u64 from = (by_count ? (u64)before.count : before.mass) + above;
        if (from < threshold && threshold <= from + same * s.sub_mass[i]) {   // those with one key write the same
          s.range[0] = k;
          s.sub_count[0] = count;
          s.sub_count[1] = same;
          s.above = above;
        }
        __syncthreads();
        hi = s.range[0];
        before.count += s.sub_count[0];
        before.mass += by_count ? 0 : s.above;
        equal = s.sub_count[1];
      } else for (;;) {
        uint32_t shift = 0;
        while (((hi - lo) >> shift) >= kSub) ++shift;
        s.sub_count[threadIdx.x] = 0;
        s.sub_mass[threadIdx.x] = 0;
        __syncthreads();
        members([&](uint32_t k) {
          if (k < lo || k > hi) return;
          atomicAdd(&s.sub_count[(hi - k) >> shift], 1u);
          if (!by_count) atomicAdd(&s.sub_mass[(hi - k) >> shift], weight_of(k));
        });
        __syncthreads();
        Sums mine = {s.sub_count[threadIdx.x], s.sub_mass[threadIdx.x]}, sum;
        const Sums ahead = before_thread(s.waves, mine, &sum);
        const u64 from = by_count ? before.count + ahead.count : before.mass + ahead.mass, to = from + (by_count ? mine.count : mine.mass);
        if (from < threshold && threshold <= to) {
          s.found[1] = threadIdx.x;
          s.sub_count[0] = ahead.count;   // all have been read by their threads before the barriers in before_thread
          s.sub_mass[0] = ahead.mass;
          s.sub_count[1] = mine.count;
        }
        __syncthreads();
        before.count += s.sub_count[0];
        before.mass += s.sub_mass[0];
        equal = s.sub_count[1];
        const uint32_t f = s.found[1], top = hi - (f << shift), span = (1u << shift) - 1;
        __syncthreads();
        hi = top;
        lo = top - lo > span ? top - span : lo;
        if (shift == 0) break;
      }
      if (stage == kTopK) {
        least = hi;
        too_many = before.count + equal - (uint32_t)set.k;
        to_list = !row_listed && before.count + equal <= kList;
      } else {
        if (threadIdx.x == 0) {
          const auto t = w.parts(Key<F32>::value(hi));
          const u64 m = w.weight(t), n = tokens_to(threshold, before.mass, m);
          s.kept = min(kept, before.mass + n * m);
          s.key = hi;
          s.nth = (uint32_t)n;
          s.prob = (float)(w.scaled(t) / (double)kept);
        }
        __syncthreads();
        if (stage == kTopP) kept = s.kept;
      }
    }
  }
  __syncthreads();
  write_token(keys, s.waves, s.sub_count, s.found, s.key, s.nth, a.ids + r);
  if (threadIdx.x == 0 && a.prob) a.prob[r] = s.prob;
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
  const uint32_t vectors = N / (uint32_t)(16 / size);   // of a row
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(rows), dim3(kThreads), 0, (hipStream_t)hip_stream, a); };
  // one, four, eight or sixteen vectors a thread hold the row; a longer one is read four vectors a thread at a time
  if (dtype == BCT_F32) {
    if (vectors <= kThreads) launch(sample_f32_kernel<1, true>);
    else if (vectors <= 4 * kThreads) launch(sample_f32_kernel<4, true>);
    else if (vectors <= 8 * kThreads) launch(sample_f32_kernel<8, true>);
    else if (vectors <= 16 * kThreads) launch(sample_f32_kernel<16, true>);
    else launch(sample_f32_kernel<4, false>);
  } else {
    if (vectors <= kThreads) launch(sample_bf16_kernel<1, true>);
    else if (vectors <= 4 * kThreads) launch(sample_bf16_kernel<4, true>);
    else if (vectors <= 8 * kThreads) launch(sample_bf16_kernel<8, true>);
    else if (vectors <= 16 * kThreads) launch(sample_bf16_kernel<16, true>);
    else launch(sample_bf16_kernel<4, false>);
  }
  return launched("sample");
}
