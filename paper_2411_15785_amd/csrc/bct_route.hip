// Each token's experts from the router's logits, and the tokens in the order of their experts (gfx950):
//
//   p = softmax(l) or 1 / (1 + exp(-l)) over the experts a token may have (l neither NaN nor -inf)
//   the k experts with the largest l, or with a bias p + bias; equal ones by number
//   weight = scale * p / (sum of the chosen p, or 1)
//
// Sixteen lanes have a token, each some of its experts, and the choice is k times a maximum: over a lane's keys, then over the sixteen
// by the data-parallel primitives, so four tokens share the instructions of a wavefront, which is what bounds it.  With a bias, scores
// are worked out in 64 bits, as two experts' sums may lie closer than fp32 tells them apart: of sigmoids only those of the few that fp32 leaves
// near the border, of a softmax all, by a whole wavefront for a token.
//
// The plan is a counting sort of the pairs (token, slot) by expert that depends on no order of atomics: blocks of tokens count
// their experts, then each block adds up what the blocks before it counted and gives its pairs their places, a wavefront's
// 64 at a time by comparing their experts bit by bit.  Few tokens are one block, and one launch.
//
// us in a graph, choice and plan: 8 of 64 experts, 1 token 8.9, 64 11.8, 1024 13.2, 16384 16.0; 8 of 256, 16384 tokens 25.7, of sigmoids with a bias 37, of
// a softmax with one 47; 16 of 512, 4096 tokens 35, 63, 60.  The forms with a bias hold the wavefront's part too and spill: up to
// 512 experts 193 registers (192 of bf16 logits), up to 256 14 (8).  A token a wavefront, its k maxima
// over 64 lanes, took 40 for the sigmoids with a bias.  The plan is 13 of 16384 tokens' times, launch included.
#include <math.h>

#include "bct_device.h"
#include "bct_experts.h"
#include "bct_model_internal.h"

namespace bct {

namespace {

typedef unsigned long long u64;
constexpr uint32_t kThreads = 1024, kWaves = kThreads / 64;

// The value of the lane that the data-parallel-primitive control names, `none` where there is none or the row is not in ROWS.
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ uint32_t other_lane(uint32_t v, uint32_t none) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xF, false);
}
// The largest value of the wavefront, the same in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, other_lane<0x111>(v, 0));
  v = max(v, other_lane<0x112>(v, 0));
  v = max(v, other_lane<0x114>(v, 0));
  v = max(v, other_lane<0x118>(v, 0));
  v = max(v, other_lane<0x142, 0xA>(v, 0));
  v = max(v, other_lane<0x143, 0xC>(v, 0));
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ u64 wave_max(u64 v) {
  const uint32_t hi = wave_max((uint32_t)(v >> 32));
  return (u64)hi << 32 | wave_max((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
}
// What the lanes up to this one hold.
__device__ __forceinline__ uint32_t up_to_lane(uint32_t v) {
  v += other_lane<0x111>(v, 0);
  v += other_lane<0x112>(v, 0);
  v += other_lane<0x114>(v, 0);
  v += other_lane<0x118>(v, 0);
  v += other_lane<0x142, 0xA>(v, 0);
  v += other_lane<0x143, 0xC>(v, 0);
  return v;
}
__device__ __forceinline__ float wave_sum(float v) { return xor_sum<1, 32>(v); }
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o, 64);
  return v;
}

// Keys order like the numbers, as integers; zeros of either sign are equal.  0 is no key: of a NaN or -inf.
__device__ __forceinline__ uint32_t key_of(float v) {
  if (!(v > -INFINITY)) return 0;
  const int32_t b = __float_as_int(v);
  return (uint32_t)(b < 0 ? -(b & 0x7FFFFFFF) : b) ^ 0x80000000u;
}
__device__ __forceinline__ u64 key_of(double v) {
  if (!(v > -INFINITY)) return 0;
  const long long b = __double_as_longlong(v);
  return (u64)(b < 0 ? -(b & 0x7FFFFFFFFFFFFFFFll) : b) ^ 0x8000000000000000ull;
}

struct RouteArgs {
  const void* logits;
  size_t ld;
  const float* bias;
  int32_t* experts;
  float* weights;
  int32_t* plan;   // null: none is made
  uint32_t rows, E, k;
  float scale;
  uint32_t sigmoid, normalise;
};

__device__ __forceinline__ float value_of(uint32_t key) {
  const int32_t v = (int32_t)(key ^ 0x80000000u);
  return __int_as_float(v < 0 ? (int32_t)(0x80000000u | (0u - (uint32_t)v)) : v);
}

// A lane's V keys in descending order, equal ones as they were (neighbours are exchanged only where they have to be).
template <typename Key, int V>
__device__ __forceinline__ void sort_keys(Key (&key)[V], uint32_t (&id)[V]) {
#pragma unroll
  for (int n = V - 1; n > 0; --n)
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const bool turn = key[i] < key[i + 1];
      const Key k = turn ? key[i] : key[i + 1];
      const uint32_t d = turn ? id[i] : id[i + 1];
      key[i] = turn ? key[i + 1] : key[i];
      id[i] = turn ? id[i + 1] : id[i];
      key[i + 1] = k;
      id[i + 1] = d;
    }
}
// Takes the largest of all lanes' first keys, which are sorted, out of them: its key, 0 where none is left, and in *expert which it
// was.  Experts go to the lanes in runs, so of equal ones the lowest lane has the first.
template <typename Key, int V>
__device__ __forceinline__ Key take_largest(Key (&key)[V], uint32_t (&id)[V], uint32_t* expert) {
  const Key best = wave_max(key[0]);
  const uint32_t from = __builtin_ctzll(__ballot(key[0] == best));
  *expert = (uint32_t)__builtin_amdgcn_readlane((int)id[0], from);
  const bool mine = threadIdx.x % 64 == from;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    key[v] = mine ? (v + 1 < V ? key[v + 1] : Key(0)) : key[v];
    id[v] = mine && v + 1 < V ? id[v + 1] : id[v];
  }
  return best;
}

// The value of the lane of the same sixteen that the data-parallel-primitive control names, and what that makes of all sixteen: the other
// of a pair, the other pair of four, mirrored in eight and in sixteen.
template <int CTRL>
__device__ __forceinline__ uint32_t of_sixteen(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, of_sixteen<0xB1>(v));
  v = max(v, of_sixteen<0x4E>(v));
  v = max(v, of_sixteen<0x141>(v));
  return max(v, of_sixteen<0x140>(v));
}
__device__ __forceinline__ float sum16(float v) { return xor_sum<1, 8>(v); }
template <int L>
__device__ __forceinline__ double row_lane(double v) {
  const long long b = __double_as_longlong(v);
  return __longlong_as_double((long long)of_sixteen<0x150 + L>((uint32_t)(b >> 32)) << 32 | of_sixteen<0x150 + L>((uint32_t)b));
}

// Writes what was chosen for a token: a lane with has has the expert, its logit x and the slot where it goes; `empty`: the slot of a lane
// that has none, if it is one of the k.  most: of a softmax without normalising, the row's largest logit, and all the sum of exp(l - most).
// MAX, SUM: over the token's lanes.
// The scores come from the logits.  To be normalised, they may have any factor in common, and are taken against the largest chosen one,
// so that they do not all underflow: exp(l - m), or as a sigmoid exp(min(l, 0) - min(m, 0)) / (1 + exp(-|l|)).
template <typename MAX, typename SUM>
__device__ __forceinline__ void write_choice(const RouteArgs& a, uint32_t r, bool has, uint32_t expert, float x, uint32_t slot, bool empty,
                                             uint32_t lane, float most, float all, uint32_t* counts, MAX max_of, SUM sum_of) {
  if (a.normalise) {
    const uint32_t first = max_of(has ? key_of(x) : 0u);
    most = value_of(first);
  }
  float weight = 0.f, total = 1.f;
  if (a.sigmoid) {
    if (has) weight = expf(fminf(x, 0.f) - (a.normalise ? fminf(most, 0.f) : 0.f)) / (1.f + expf(-fabsf(x)));
  } else {
    if (has) weight = x == most ? 1.f : expf(x - most);
    total = all;
  }
  if (a.normalise) total = sum_of(weight);
  if (has || empty) {
    const size_t at = (size_t)r * a.k + (has ? slot : lane);
    a.experts[at] = has ? (int32_t)expert : -1;
    a.weights[at] = has ? weight / total * a.scale : 0.f;
    if (counts) atomicAdd(&counts[has ? expert : a.E], 1u);
  }
}

// The choice with a bias in 64 bits throughout, by a whole wavefront: a lane has V experts one after the other.
template <typename DT, int V>
__device__ __forceinline__ void route_whole(const RouteArgs& a, uint32_t r, uint32_t* counts) {
  const uint32_t lane = threadIdx.x % 64;
  const typename DT::elem* row = (const typename DT::elem*)a.logits + (size_t)r * a.ld;
  float l[V], most = -INFINITY;
  uint32_t id[V], top = 0;
  u64 sums[V];
  double p[V], all = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    id[v] = lane * V + v;
    l[v] = load_elem(row, min(id[v], a.E - 1));
    asm("" : "+v"(l[v]));
    if (id[v] >= a.E || !(l[v] > -INFINITY)) l[v] = -INFINITY;
    top = max(top, key_of(l[v]));
  }
  if (a.sigmoid) {
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = 1.0 / (1.0 + exp(-(double)l[v]));
  } else {
    top = wave_max(top);
    if (top) most = value_of(top);
#pragma unroll
    for (int v = 0; v < V; ++v) {   // infinite logits share with one another
      p[v] = l[v] == -INFINITY ? 0.0 : l[v] == most ? 1.0 : exp((double)l[v] - (double)most);
      all += p[v];
    }
    all = wave_sum(all);
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] /= all;
  }
#pragma unroll
  for (int v = 0; v < V; ++v) sums[v] = l[v] == -INFINITY ? 0 : key_of(p[v] + (double)a.bias[min(id[v], a.E - 1)]);
  sort_keys(sums, id);
  uint32_t expert = a.E, count = 0;
  for (; count < a.k; ++count) {
    uint32_t e;
    if (take_largest(sums, id, &e) == 0) break;
    if (lane == count) expert = e;
  }
  const bool has = lane < count;
  const float x = has ? load_elem(row, expert) : -INFINITY;
  write_choice(a, r, has, expert, x, lane, !has && lane < a.k, lane, most, (float)all, counts,
               [](uint32_t v) { return wave_max(v); }, [](float v) { return wave_sum(v); });
}

// The choice for four tokens from r on (those below r1) by a wavefront, V of a token's experts to each of its sixteen lanes: four side by
// side, so that four lanes read 64 bytes, and the four that are 64 further.  counts: how many of each expert there are is added to
// it, if it is not null.
template <typename DT, bool BIAS, int V>
__device__ __forceinline__ void route_four(const RouteArgs& a, uint32_t r, uint32_t r1, uint32_t* counts) {
  const uint32_t lane = threadIdx.x % 16, group = threadIdx.x % 64 / 16, mine = r + group;
  if (BIAS && !a.sigmoid) {
    for (uint32_t i = r; i < min(r + 4, r1); ++i) route_whole<DT, V / 4>(a, i, counts);
    return;
  }
  const bool there = mine < r1;
  const typename DT::elem* row = (const typename DT::elem*)a.logits + (size_t)min(mine, r1 - 1) * a.ld;
  uint32_t key[V];
  float most = -INFINITY, all = 1.f;
  auto expert_of = [&](uint32_t v) -> uint32_t { return 4 * lane + v / 4 * 64 + v % 4; };
  constexpr int AT_ONCE = BIAS && V > 16 ? 16 : BIAS && V > 8 ? 8 : V;   // what there are registers for
#pragma unroll
  for (int v0 = 0; v0 < V; v0 += AT_ONCE) {
    float l[AT_ONCE], bias[AT_ONCE];
#pragma unroll
    for (int v = 0; v < AT_ONCE; ++v) {
      const uint32_t at = min(expert_of(v0 + v), a.E - 1);
      l[v] = load_elem(row, at);
      if (BIAS) bias[v] = a.bias[at];
    }
#pragma unroll
    for (int v = 0; v < AT_ONCE; ++v) {
      // requested together: behind the branch that the compiler makes of what follows, they would be waited for one by one
      asm("" : "+v"(l[v]));
      if (BIAS) asm("" : "+v"(bias[v]));
    }
#pragma unroll
    for (int v = 0; v < AT_ONCE; ++v) {
      uint32_t& to = key[v0 + v];
      to = expert_of(v0 + v) < a.E ? key_of(l[v]) : 0;
      if constexpr (BIAS) to = to ? key_of(__builtin_amdgcn_rcpf(1.f + __expf(-l[v])) + bias[v]) : 0;
    }
    if (AT_ONCE < V) __builtin_amdgcn_sched_barrier(0);
  }
  if (!BIAS && !a.sigmoid && !a.normalise) {   // the softmax' sum over all experts
    uint32_t top = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) top = max(top, key[v]);
    top = max16(top);
    most = value_of(top);
    all = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (key[v]) all += key[v] == top ? 1.f : expf(value_of(key[v]) - most);
    all = sum16(all);
  }
  // With a bias the rounds go on, to the last lane, as long as a sum does not lie below the kth by more than both may be off: 2^-21 for a
  // sigmoid of fp32, 2^-23 of the sum.
  uint32_t count = 0, least = 1, expert = a.E;   // found; no smaller key is; what is in this lane's place
  bool more = false;
  for (uint32_t s = 0; s < (BIAS ? 17u : a.k); ++s) {
    uint32_t best = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) best = max(best, key[v]);
    best = max16(best);
    if (BIAS && s >= a.k && __ballot(best >= least && there) == 0) break;
    // the first expert that has it
    uint32_t at = V;
#pragma unroll
    for (int v = V - 1; v >= 0; --v) at = key[v] == best ? v : at;
    const uint32_t e = at < V ? expert_of(at) : ~0u, first = ~max16(~e);
    at = e == first ? at : V;
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = at == v ? 0 : key[v];
    if (best >= least) {
      if (lane == s) expert = first;
      ++count;
      more = BIAS && s == 16;
    }
    if constexpr (BIAS) {
      if (s + 1 == a.k) {
        const float kth = value_of(best), below = kth - (0x1p-19f + 0x1p-21f * fabsf(kth));
        least = best < least ? ~0u : below == below ? max(key_of(below), 1u) : best;   // none left; an infinite one: those
      }
    }
  }
  uint32_t slot = lane;
  const bool listed = lane < count && there;
  if (!listed) expert = a.E;
  const float x = listed ? load_elem(row, expert) : -INFINITY;
  if constexpr (BIAS) {
    double sum = -INFINITY;
    if (listed) sum = 1.0 / (1.0 + exp(-(double)x)) + (double)a.bias[expert];
    slot = 0;
    auto against = [&](auto j) {   // the slot is how many come before this one
      const double other = row_lane<decltype(j)::v>(sum);
      const uint32_t e = of_sixteen<0x150 + decltype(j)::v>(expert);
      slot += other > sum || (other == sum && e < expert) ? 1 : 0;
    };
    against(Int<0>{}), against(Int<1>{}), against(Int<2>{}), against(Int<3>{}), against(Int<4>{}), against(Int<5>{}), against(Int<6>{});
    against(Int<7>{}), against(Int<8>{}), against(Int<9>{}), against(Int<10>{}), against(Int<11>{}), against(Int<12>{}), against(Int<13>{});
    against(Int<14>{}), against(Int<15>{});
    const u64 whole = __ballot(more && there && lane == 0);   // more near the border than there are lanes
    count = min(count, a.k);
    const bool mine_done = there && !more;
    write_choice(a, mine, listed && !more && slot < a.k, expert, x, slot, mine_done && lane >= count && lane < a.k, lane, most, all, counts,
                 [](uint32_t v) { return max16(v); }, [](float v) { return sum16(v); });
    for (uint32_t g = 0; g < 4; ++g)
      if (whole >> (16 * g) & 1) route_whole<DT, V / 4>(a, r + g, counts);
  } else {
    write_choice(a, mine, listed, expert, x, slot, there && lane >= count && lane < a.k, lane, most, all, counts,
                 [](uint32_t v) { return max16(v); }, [](float v) { return sum16(v); });
  }
}

struct PlanShared {
  uint32_t wave[kWaves][kMaxExperts + 1];   // pairs of an expert in a wavefront's share, then where its next one goes
  uint32_t total[4 * kThreads], before[4 * kThreads];
  uint32_t tile[kTileLists][kMaxExperts + 1];   // an expert's first row tile
  uint32_t scan[kTileLists + 1][kWaves];
};

// Gives the pairs of one block of tokens their places.  experts: of all pairs.
__device__ __forceinline__ void plan_block(const int32_t* experts, int32_t* plan, const ExpertPlan& P, uint32_t rows, uint32_t k,
                                           uint32_t block, PlanShared& s) {
  const uint32_t lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), E = P.E, C = E + 1;
  const uint32_t per_block = P.block_rows(rows) * k, p0 = min(block * per_block, P.pairs), p1 = min(p0 + per_block, P.pairs);
  const uint32_t share = ((p1 - p0 + kWaves - 1) / kWaves + 63) / 64 * 64, w0 = min(p0 + wave * share, p1), w1 = min(w0 + share, p1);
  const uint32_t waves = share ? (p1 - p0 + share - 1) / share : 0;   // that have a share; a block behind the last token has none
  for (uint32_t w = 0; w < waves; ++w)
    if (threadIdx.x < C) s.wave[w][threadIdx.x] = 0;
  __syncthreads();
  for (uint32_t p = w0 + lane; p < w1; p += 64) {
    const uint32_t e = min((uint32_t)experts[p], E);   // a negative one is beyond E
    atomicAdd(&s.wave[wave][e], 1u);
    plan[P.expert + p] = e < E ? (int32_t)e + 1 : 0;
  }
  // What all blocks and the blocks before this one have of each expert: a thread adds up four experts of every groups-th block.
  if (P.blocks > 1) {
    const uint32_t quads = (C + 3) / 4, groups = kThreads / quads, g = threadIdx.x / quads, q = threadIdx.x % quads;
    const uint4* counts = (const uint4*)(plan + P.counts) + q;
    uint4 all = make_uint4(0, 0, 0, 0), before = all;
    if (g < groups) {
#pragma unroll 8
      for (uint32_t b = g; b < P.blocks; b += groups) {
        const uint4 n = counts[(size_t)b * quads];
        const uint32_t m = b < block ? ~0u : 0u;
        all = make_uint4(all.x + n.x, all.y + n.y, all.z + n.z, all.w + n.w);
        before = make_uint4(before.x + (n.x & m), before.y + (n.y & m), before.z + (n.z & m), before.w + (n.w & m));
      }
    }
    ((uint4*)s.total)[threadIdx.x] = all;
    ((uint4*)s.before)[threadIdx.x] = before;
    __syncthreads();
    uint32_t a = 0, f = 0;
    if (threadIdx.x < C)
      for (uint32_t i = 0; i < groups; ++i) {
        a += s.total[i * 4 * quads + threadIdx.x];
        f += s.before[i * 4 * quads + threadIdx.x];
      }
    __syncthreads();
    if (threadIdx.x < C) {
      s.total[threadIdx.x] = a;
      s.before[threadIdx.x] = f;
    }
  } else {
    __syncthreads();
    if (threadIdx.x < C) {
      uint32_t all = 0;
      for (uint32_t w = 0; w < waves; ++w) all += s.wave[w][threadIdx.x];
      s.total[threadIdx.x] = all;
      s.before[threadIdx.x] = 0;
    }
  }
  // Where each expert's pairs and row tiles begin; thread e has expert e, the last one the pairs without an expert.
  const uint32_t e = threadIdx.x, n = e < C ? s.total[e] : 0;
  uint32_t own[kTileLists + 1], run[kTileLists + 1];
#pragma unroll
  for (uint32_t i = 0; i <= kTileLists; ++i) {
    const uint32_t size = kPlanRows[i % kTileLists];
    own[i] = i == kTileLists ? n : e < E ? (n + size - 1) / size : 0;
    run[i] = up_to_lane(own[i]);
    if (lane == 63) s.scan[i][wave] = run[i];
  }
  __syncthreads();
#pragma unroll
  for (uint32_t i = 0; i <= kTileLists; ++i)
    for (uint32_t w = 0; w < wave; ++w) run[i] += s.scan[i][w];
  if (e < C) {
    const uint32_t first = run[kTileLists] - n;
    uint32_t at = first + s.before[e];
    s.before[e] = first;
    for (uint32_t w = 0; w < waves; ++w) {
      const uint32_t c = s.wave[w][e];
      s.wave[w][e] = at;
      at += c;
    }
#pragma unroll
    for (uint32_t i = 0; i < kTileLists; ++i) s.tile[i][e] = run[i] - own[i];
    if (block == 0) {
      plan[e] = (int32_t)first;
      if (e == E)
#pragma unroll
        for (uint32_t i = 0; i < kTileLists; ++i) plan[P.n_tiles + i] = (int32_t)run[i];
    }
  }
  __syncthreads();
  // the row tiles: experts are dealt out to the wavefronts of all blocks
  for (uint32_t x = block * kWaves + wave; x < E; x += P.blocks * kWaves) {
    const uint32_t count = s.total[x], first = s.before[x];
#pragma unroll
    for (uint32_t i = 0; i < kTileLists; ++i) {
      uint4* list = (uint4*)(plan + P.list[i]) + s.tile[i][x];
      for (uint32_t t = lane; t * kPlanRows[i] < count; t += 64)
        list[t] = make_uint4(x, first, count, t);
    }
  }
  // the pairs, 64 at a time: a pair's place is its expert's next one and how many lanes before have that expert too
  for (uint32_t p = w0; p < w1; p += 64) {
    const bool in = p + lane < w1;
    const uint32_t x = in ? min((uint32_t)experts[p + lane], E) : 0u;
    u64 same = __ballot(in);
    for (uint32_t bit = 1; bit <= E; bit *= 2) {
      const u64 set = __ballot((x & bit) != 0);
      same &= x & bit ? set : ~set;
    }
    if (!in) continue;
    const uint32_t leader = __builtin_ctzll(same);
    uint32_t at = 0;
    if (lane == leader) at = atomicAdd(&s.wave[wave][x], (uint32_t)__popcll(same));
    at = __shfl(at, leader, 64) + __popcll(same & ((1ull << lane) - 1));
    plan[P.order + at] = (int32_t)(p + lane);
  }
}

template <typename DT, bool BIAS, int V>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a, ExpertPlan P) {
  __shared__ union {
    uint32_t count[kMaxExperts + 1];
    PlanShared plan;
  } s;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), C = a.E + 1, per = P.block_rows(a.rows);
  const uint32_t r0 = min(blockIdx.x * per, a.rows), r1 = min(r0 + per, a.rows);
  const bool counts = a.plan && P.blocks > 1;
  if (counts) {
    if (threadIdx.x < C) s.count[threadIdx.x] = 0;
    __syncthreads();
  }
  for (uint32_t r = r0 + 4 * wave; r < r1; r += 4 * kWaves) route_four<DT, BIAS, V>(a, r, r1, counts ? s.count : nullptr);
  __syncthreads();
  if (counts) {
    if (threadIdx.x < C) a.plan[P.counts + (size_t)blockIdx.x * ((C + 3) / 4 * 4) + threadIdx.x] = (int32_t)s.count[threadIdx.x];
  } else if (a.plan) {
    plan_block(a.experts, a.plan, P, a.rows, a.k, 0, s.plan);
  }
}

// What each block of tokens has of each expert, where the experts are given.
__global__ __launch_bounds__(kThreads) void count_kernel(const int32_t* experts, int32_t* plan, ExpertPlan P, uint32_t rows, uint32_t k) {
  __shared__ uint32_t count[kMaxExperts + 1];
  const uint32_t C = P.E + 1, per = P.block_rows(rows) * k, p0 = min(blockIdx.x * per, P.pairs), p1 = min(p0 + per, P.pairs);
  if (threadIdx.x < C) count[threadIdx.x] = 0;
  __syncthreads();
  for (uint32_t p = p0 + threadIdx.x; p < p1; p += kThreads) atomicAdd(&count[min((uint32_t)experts[p], P.E)], 1u);
  __syncthreads();
  if (threadIdx.x < C) plan[P.counts + (size_t)blockIdx.x * ((C + 3) / 4 * 4) + threadIdx.x] = (int32_t)count[threadIdx.x];
}
__global__ __launch_bounds__(kThreads) void plan_kernel(const int32_t* experts, int32_t* plan, ExpertPlan P, uint32_t rows, uint32_t k) {
  __shared__ PlanShared s;
  plan_block(experts, plan, P, rows, k, blockIdx.x, s);
}

template <typename DT, bool BIAS>
void launch_route(const RouteArgs& a, const ExpertPlan& P, hipStream_t s) {
  const dim3 grid(P.blocks), block(kThreads);
  if (a.E <= 64) hipLaunchKernelGGL((route_kernel<DT, BIAS, 4>), grid, block, 0, s, a, P);
  else if (a.E <= 128) hipLaunchKernelGGL((route_kernel<DT, BIAS, 8>), grid, block, 0, s, a, P);
  else if (a.E <= 256) hipLaunchKernelGGL((route_kernel<DT, BIAS, 16>), grid, block, 0, s, a, P);
  else hipLaunchKernelGGL((route_kernel<DT, BIAS, 32>), grid, block, 0, s, a, P);
}

}  // namespace

bct_status check_plan_sizes(uint32_t rows, uint32_t k, uint32_t E) {
  if (rows == 0 || k == 0 || E == 0) return mfail(BCT_ERR_INVALID_ARG, "zero size");
  if (E > kMaxExperts || k > kMaxPerToken || k > E) return mfail(BCT_ERR_UNSUPPORTED, "at most 512 experts, 16 of them and not more than there are a token");
  if ((uint64_t)rows * k > 0x7FFFFFFFull - 0xFFFF) return mfail(BCT_ERR_UNSUPPORTED, "too many tokens");
  return BCT_OK;
}

bct_status check_expert_plan(const void* plan, uint32_t rows, uint32_t k, uint32_t E) {
  if (!plan) return mfail(BCT_ERR_INVALID_ARG, "NULL plan");
  if (!al16(plan)) return mfail(BCT_ERR_MISALIGNED, "pointers must be 16-byte aligned");
  return check_plan_sizes(rows, k, E);
}

}  // namespace bct

using namespace bct;

extern "C" {

bct_status bctm_expert_plan_bytes(uint32_t rows, uint32_t k, uint32_t n_experts, size_t* bytes, size_t* order) {
  if (!bytes) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer");
  const bct_status st = check_plan_sizes(rows, k, n_experts);
  if (st != BCT_OK) return st;
  const ExpertPlan P = ExpertPlan::of(rows, k, n_experts);
  *bytes = P.ints * 4;
  if (order) *order = P.order;
  return BCT_OK;
}

bct_status bctm_route(const void* logits, size_t ld, const float* bias, int32_t* experts, float* weights, void* plan,
                      size_t plan_bytes, uint32_t rows, uint32_t n_experts, uint32_t k, float scale, int32_t dtype, uint32_t flags,
                      void* hip_stream) {
  if (!logits || !experts || !weights) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer or zero size");
  const bct_status st = check_plan_sizes(rows, k, n_experts);
  if (st != BCT_OK) return st;
  if (dtype != BCT_F32 && dtype != BCT_BF16) return mfail(BCT_ERR_UNSUPPORTED, "logits are float32 or bf16");
  if (flags & ~(BCTM_ROUTE_SIGMOID | BCTM_ROUTE_NORMALISE)) return mfail(BCT_ERR_INVALID_ARG, "unknown flag");
  if (ld < n_experts || ld >> 56) return mfail(BCT_ERR_INVALID_ARG, "ld must be at least n_experts");
  if (!(fabsf(scale) < INFINITY)) return mfail(BCT_ERR_INVALID_ARG, "scale must be finite");
  if (((uintptr_t)logits & (dtype == BCT_F32 ? 3u : 1u)) || ((uintptr_t)bias & 3u) || ((uintptr_t)experts & 3u) || ((uintptr_t)weights & 3u) || !al16(plan))
    return mfail(BCT_ERR_MISALIGNED, "pointers must be aligned to their type, the plan to 16 bytes");
  const ExpertPlan P = ExpertPlan::of(rows, k, n_experts);
  if (plan && plan_bytes < P.ints * 4) return mfail(BCT_ERR_BUFFER_TOO_SMALL, "the plan is smaller than bctm_expert_plan_bytes says");
  const RouteArgs a = {logits, ld, bias, experts, weights, (int32_t*)plan, rows, n_experts, k, scale, flags & BCTM_ROUTE_SIGMOID ? 1u : 0u,
                       flags & BCTM_ROUTE_NORMALISE ? 1u : 0u};
  hipStream_t s = (hipStream_t)hip_stream;
  if (dtype == BCT_F32) bias ? launch_route<F32, true>(a, P, s) : launch_route<F32, false>(a, P, s);
  else bias ? launch_route<BF16, true>(a, P, s) : launch_route<BF16, false>(a, P, s);
  if (plan && P.blocks > 1)
    hipLaunchKernelGGL(plan_kernel, dim3(P.blocks), dim3(kThreads), 0, s, (const int32_t*)experts, (int32_t*)plan, P, rows, k);
  return launched("route");
}

bct_status bctm_expert_plan(const int32_t* experts, void* plan, size_t plan_bytes, uint32_t rows, uint32_t n_experts, uint32_t k,
                            void* hip_stream) {
  if (!experts || !plan) return mfail(BCT_ERR_INVALID_ARG, "NULL pointer or zero size");
  const bct_status st = check_plan_sizes(rows, k, n_experts);
  if (st != BCT_OK) return st;
  if (((uintptr_t)experts & 3u) || !al16(plan)) return mfail(BCT_ERR_MISALIGNED, "pointers must be aligned to their type, the plan to 16 bytes");
  const ExpertPlan P = ExpertPlan::of(rows, k, n_experts);
  if (plan_bytes < P.ints * 4) return mfail(BCT_ERR_BUFFER_TOO_SMALL, "the plan is smaller than bctm_expert_plan_bytes says");
  hipStream_t s = (hipStream_t)hip_stream;
  if (P.blocks > 1) hipLaunchKernelGGL(count_kernel, dim3(P.blocks), dim3(kThreads), 0, s, experts, (int32_t*)plan, P, rows, k);
  hipLaunchKernelGGL(plan_kernel, dim3(P.blocks), dim3(kThreads), 0, s, experts, (int32_t*)plan, P, rows, k);
  return launched("expert_plan");
}

}  // extern "C"
