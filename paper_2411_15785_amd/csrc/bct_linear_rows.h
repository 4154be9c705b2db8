// The matrix-core projection kernel of many token rows and its launch; bct_linear_rows.hip says how it works and what it measured.
#ifndef BCT_LINEAR_ROWS_H
#define BCT_LINEAR_ROWS_H

#include "bct_device.h"
#include "bct_experts.h"
#include "bct_linear.h"

namespace bct {

// The tile of a shape (rows_shape in bct_linear_rows.hip).
enum RowsShape { kTile256, kTile128x512, kTile128x256, kTile128, kTile128K2, kTile128x64K2, kTile64K2 };
RowsShape rows_shape(uint32_t rows, uint32_t bcols, uint32_t K, bool x_tiled);

namespace {

// Where a row's four chunks of a K step lie, with experts: chunk c of row r at place c ^ row_turn(r / 4).
__device__ __forceinline__ int row_turn(int q) { return ((q ^ q >> 1) & 1) << 1 | q >> 1; }   // 0, 2, 3, 1

// KS groups of WR x WC wavefronts; a wavefront owns 16 * MI token rows x 16 * NJ B-tile columns (SwiGLU: gate and
// up tiles alternate, so half as many output features); group g sums the K steps [KT * g / KS, ...).
// PAIR (row-major activations): the two K steps of a line are requested together, see request_rows.
// TERM: none, or one of
//   LoraTerm      the rows' low-rank term is added to the accumulators
//   EpilogueTerm  bias and activation before the residual, bf16 or fp32 outputs
//   ExpertTerm    the rows of a row tile are gathered, those of one expert, and meet its weights
// (A pack, so that the kernels without one are compiled as if there were none with it.)
template <bool SWIGLU, bool XT, bool PAIR, int MI, int NJ, int WR, int WC, int KS, typename... TERM>
__global__ __launch_bounds__(64 * WR * WC * KS, 2) void linear_rows_kernel(
    const uint16_t* __restrict__ x, const u32x4* __restrict__ w, const u32x4* __restrict__ w2, const uint16_t* residual,
    LinearOut dst, uint32_t rows, uint32_t K, uint32_t NT, uint32_t out_tiled, TERM... term) {
  constexpr bool kLora = kHas<LoraTerm, TERM...>, kEpilogue = kHas<EpilogueTerm, TERM...>, kExperts = kHas<ExpertTerm, TERM...>;
  static_assert(!kExperts || (!XT && !PAIR && 64 * WR * WC * KS >= 16 * MI * WR && NJ == 4), "gathered rows are row-major; a thread has one");
  constexpr int NW = WR * WC;                      // wavefronts of a group
  constexpr int TA = MI * WR, TB = NJ * WC, TT = TA + TB;  // 1 KB tiles of a K step: activations, weights
  constexpr int ND = TT / NW, NA = TA / NW, NB = TB / NW;  // of them per wavefront
  static_assert(TA % NW == 0 && TB % NW == 0, "tiles must divide among the wavefronts");
  static_assert(!PAIR || !XT, "tiled activations have no half lines");
  // LDS stages.  Three leave room for two workgroups of 128 x 256 on a compute unit, and one begins and ends under the other's
  // products: with experts, whose tiles are many, 4096 tokens of 8 in 64 1376 -> 4096 670 -> 630 us, gated 4096 -> 1376 827 -> 792.
  constexpr int S = kExperts && MI == 4 && NW == 8 ? 3 : 4;
  constexpr bool PING = NW * KS == 8;              // two wavefronts per SIMD that take turns
  constexpr uint32_t HB = 4;                       // row tiles of a band
  constexpr uint32_t BM = 16 * MI * WR;            // token rows of a workgroup
  constexpr uint32_t CW = 16 * NJ;                 // B columns of a wavefront
  constexpr uint32_t BNF = CW * WC / (SWIGLU ? 2 : 1);  // output features of a workgroup
  __shared__ __attribute__((aligned(16))) u32x4 st0[KS * TT * 64];
  __shared__ __attribute__((aligned(16))) u32x4 st1[KS * TT * 64];
  __shared__ __attribute__((aligned(16))) u32x4 st2[KS * TT * 64];
  __shared__ __attribute__((aligned(16))) u32x4 st3[S > 3 ? KS * TT * 64 : 1];
  __shared__ uint32_t pair_of[kExperts ? BM : 1];   // the pairs of the tile's rows

  uint32_t RT = (rows + BM - 1) / BM;
  if constexpr (kExperts) {   // the grid is for the most tiles there can be
    RT = min(*only(term...).n_tiles, only(term...).most_tiles);
    if (blockIdx.x / 8 >= (RT * NT + 7) / 8) return;
  }
  const uint32_t total = RT * NT, per = (total + 7) / 8;
  const uint32_t vid = (blockIdx.x % 8) * per + blockIdx.x / 8;
  if (vid >= total) return;   // the grid is 8 * per workgroups: every id below total comes up once
  // The last band takes the remainder as well (HB to 2 * HB - 1 row tiles): a band of one row tile of its own would read
  // every weight for that row tile alone.  us, own band | this: 320 rows, 11008 -> 4096 89.5 | 82.5, 4096 -> 12288 73 | 67,
  // 640 rows 107 | 102; 330 shapes 0.95 to 1.2, in the mean 1.004 to 1.02 for each tile (64 x 64: 434, 6464 -> 2176 35.6 |
  // 37.6, 283, 10752 -> 6016 125 | 106).  Not where two workgroups share a compute
  // unit (no turns): the two are 32 ids of their XCD apart, so in bands of HB they have the same row tile and its activations
  // from L1, in others not.  1060 rows, 928 -> 4480 21.0 | 24.3, 1598, 4000 -> 3456 56.2 | 62.6, 515, 10464 -> 7296 132 | 151 (but
  // 616, 8704 -> 6784 131 | 110).
  // With experts bands are those of one expert, so that its weights are read by workgroups side by side and come from memory once (in
  // bands over the experts' borders, 4096 tokens of 8 in 64 experts, 4096 -> 1376, read 3.1 GB for 1.5).
  uint32_t own = vid;
  ExpertTile tile = {0, 0, 0, 0};
  if constexpr (kExperts) {
    const uint32_t any = vid / NT;   // one of the expert's tiles
    tile = expert_tile(only(term...), any);
    if (tile.pairs == 0) return;
    own = vid - (any - tile.tile) * NT;
    RT = (tile.pairs + BM - 1) / BM;
  }
  const uint32_t nfull = !PING ? RT / HB : RT < 2 * HB ? 0u : RT / HB - 1;
  uint32_t rt, nt;
  if (own < nfull * HB * NT) {
    const uint32_t band = own / (HB * NT), rem = own % (HB * NT);
    nt = rem / HB;
    rt = band * HB + rem % HB;
  } else {
    const uint32_t rem = own - nfull * HB * NT, cnt = RT - nfull * HB;
    nt = rem / cnt;
    rt = nfull * HB + rem % cnt;
  }
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, jl = lane % 16, kg = lane / 16;
  const int grp = KS > 1 ? wv / NW : 0, wave = wv % NW, wr = wave / WC, wc = wave % WC;
  uint32_t r0 = rt * BM;
  const uint32_t KT = K / 32;
  // with experts rows count from the tile's first one, and end with it
  const int32_t* order = nullptr;
  if constexpr (kExperts) {
    const ExpertTerm& T = only(term...);
    // as many rows for each of its tiles, so that those that share weights run side by side to the end
    const uint32_t each = ((tile.pairs + RT - 1) / RT + 15) / 16 * 16;
    r0 = rt * each;
    if (r0 >= tile.pairs) return;
    rows = min(tile.pairs - r0, each);
    order = T.order + tile.begin + r0;
    if (threadIdx.x < rows) pair_of[threadIdx.x] = expert_pair(T, order, threadIdx.x);   // read behind the K loop's barriers
    w += tile.expert * T.stride;
    if (SWIGLU) w2 += tile.expert * T.stride;
    r0 = 0;
  }
  const uint32_t kfirst = grp ? (KT + 1) / 2 : 0u;                       // this group's K steps
  const uint32_t kcount = KS > 1 ? (grp ? KT / 2 : (KT + 1) / 2) : KT;
  const uint32_t kboth = KS > 1 ? KT / 2 : KT, kmost = KS > 1 ? (KT + 1) / 2 : KT;  // steps all groups / some group have

  // An expert's last row tile is partly used: the 16-row tiles of a wavefront are every WR-th one, so that those there are divide
  // evenly, and the others are not multiplied.
  const int active = kExperts ? __builtin_amdgcn_readfirstlane((int)(((rows + 15) / 16 + WR - 1 - wr) / WR)) : MI;

  // this lane's 16 bytes of the tiles wave, wave + NW, ... of a K step
  const char* src[ND];
  uint32_t step[ND];
#pragma unroll
  for (int j = 0; j < ND; ++j) {
    const uint32_t tile = wave + NW * j;
    if (tile < (uint32_t)TA) {
      if (XT) {
        const uint32_t g = min(r0 / 32 + tile / 2, (rows + 31) / 32 - 1);   // row groups past the end: a valid one
        src[j] = (const char*)(x + (((size_t)g * KT * 2 + tile % 2) * 64 + lane) * 8);
        step[j] = 2048;
      } else if constexpr (kExperts) {
        // Four lanes to a row, so that the address unit takes a row's 64 bytes at once (16 rows side by side, as an operand lies, it takes
        // lane by lane).  Chunk c of row r lies at place c ^ r / 4 of the row's four, so that an operand read finds its 16 rows
        // in different banks.
        const ExpertTerm& T = only(term...);
        const uint32_t r = min(tile * 16 + lane / 4, rows - 1);
        src[j] = (const char*)(x + (size_t)(expert_pair(T, order, r) / T.per_row) * K + (lane % 4 ^ row_turn(lane / 16)) * 8);
        step[j] = 64;
      } else {
        const uint32_t r = min(r0 + tile * 16 + jl, rows - 1);
        src[j] = (const char*)(x + (size_t)r * K + kg * 8);
        step[j] = 64;
      }
    } else {
      // features past the end: the last ones again, not stored
      const uint32_t bt = tile - TA, most = dst.start[3] / 16 - 1;
      if (SWIGLU) src[j] = (const char*)(((bt % 2) ? w2 : w) + (size_t)min(nt * (TB / 2) + bt / 2, most) * KT * 64 + lane);
      else src[j] = (const char*)(w + (size_t)min(nt * TB + bt, most) * KT * 64 + lane);
      step[j] = 1024;
    }
  }

  f32x4 acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto lora_tiles = [&](const auto& lora) {
    // B tile j of the wavefront: features past the end take the last tile's, as their weights do
    auto tile = [&](int j) -> uint32_t {
      const uint32_t bt = NJ * wc + j, most = dst.start[3] / 16 - 1;
      return SWIGLU ? min(nt * (TB / 2) + bt / 2, most) : min(nt * TB + bt, most);
    };
    auto segment = [=](int j) -> uint32_t {
      if (SWIGLU) return j % 2;   // a wavefront's tiles begin with a gate tile
      const uint32_t n = 16 * tile(j);
      return n >= dst.start[2] ? 2 : n >= dst.start[1] ? 1 : 0;
    };
    return LoraTiles<NJ, SWIGLU ? 2 : 1, decltype(segment), decltype(tile)>{lora, dst.start[3], segment, tile};
  };

  auto stage = [&](auto c) -> u32x4* {
    if constexpr (decltype(c)::v % S == 0) return st0;
    else if constexpr (decltype(c)::v % S == 1) return st1;
    else if constexpr (decltype(c)::v % S == 2) return st2;
    else return st3;
  };
  // one index into the stage each: the compiler loses track of which array an access belongs to when the
  // address is a long chain
  const int put0 = (grp * TT + wave) * 64, geta = (grp * TT + (kExperts ? wr : MI * wr)) * 64 + (kExperts ? jl * 4 + (kg ^ row_turn(jl / 4)) : lane), getb = (grp * TT + TA + NJ * wc) * 64 + lane;
  auto at = [&](uint32_t kt) { return min(kfirst + kt, KT - 1); };   // past the end: the last step again, never multiplied
  auto request = [&](auto c, uint32_t kt, auto first, auto last) {   // loads first .. last - 1 of step kt
    u32x4* s = stage(c);
    const uint32_t k = at(kt);
#pragma unroll
    for (int j = decltype(first)::v; j < decltype(last)::v; ++j) load_to_lds(src[j] + (size_t)k * step[j], s + put0 + NW * 64 * j);
  };
  // PAIR: a row's 64 bytes of a K step are half a line; the two steps of a line are requested together, before its other
  // half is evicted.
  auto request_rows = [&](auto c, uint32_t kt) {
    u32x4 *s0 = stage(c), *s1 = stage(Int<decltype(c)::v + 1>{});
    const uint32_t k0 = at(kt), k1 = at(kt + 1);
#pragma unroll
    for (int j = 0; j < NA; ++j) {
      load_to_lds(src[j] + (size_t)k0 * step[j], s0 + put0 + NW * 64 * j);
      load_to_lds(src[j] + (size_t)k1 * step[j], s1 + put0 + NW * 64 * j);
    }
    __builtin_amdgcn_sched_barrier(0);   // before the weights that are requested next: the waits count on it
  };
  // K step kt from stage c; requests step kt + S - 1 (PAIR: of the activations, in even steps, kt + 2 and kt + 3) into
  // stages whose reads all wavefronts have finished (they waited for them before the barrier that ended their step
  // kt - 1).  Left in flight at the end: what steps kt + 2 and kt + 3 need (PAIR: after an odd step only their weights,
  // as the activations of kt + 1 came with those of kt + 2).
  auto k_step = [&](auto c, uint32_t kt, auto last) {
    u32x4* s = stage(c);
    bf16x8 a[MI], b[NJ];
#pragma unroll
    for (int i = 0; i < NJ; ++i) b[i] = __builtin_bit_cast(bf16x8, s[getb + 64 * i]);
#pragma unroll
    for (int i = 0; i < MI; ++i) a[i] = __builtin_bit_cast(bf16x8, s[geta + 64 * i * (kExperts ? WR : 1)]);
    constexpr bool even = decltype(c)::v % 2 == 0;   // of kt as well
    constexpr int left = (S - 2) * (PAIR && !even ? NB : ND);
    if constexpr (PAIR && even) request_rows(Int<decltype(c)::v + 2>{}, kt + 2);
    request(Int<decltype(c)::v + S - 1>{}, kt + S - 1, Int<PAIR ? NA : 0>{}, Int<ND>{});
    if constexpr (PING) {
      __builtin_amdgcn_s_waitcnt(kWaitLds);
      __builtin_amdgcn_s_waitcnt(wait_vm(left));
      bare_barrier();
    }
    auto products = [&] {
      if constexpr (PING) __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        if (kExperts && i >= active) break;
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], acc[i][j], 0, 0, 0);
      }
      if constexpr (PING) __builtin_amdgcn_s_setprio(0);
    };
    if constexpr (decltype(last)::v == 0) products();
    else if (kt < kcount) products();   // the second group of an odd number of steps has one fewer
    if constexpr (!PING) {
      // the operands have been read: a wavefront's products wait for them and come before the barrier
      __builtin_amdgcn_s_waitcnt(kWaitLds);
      __builtin_amdgcn_s_waitcnt(wait_vm(left));
    }
    bare_barrier();
  };

  // The wait counts requests from the last one back, here and in the loop, so the stages' order has to stand: nothing
  // is moved across the scheduling barriers (in the loop, bare_barrier has them).
  if constexpr (PAIR) request_rows(Int<0>{}, 0);
  request(Int<0>{}, 0, Int<PAIR ? NA : 0>{}, Int<ND>{});
  __builtin_amdgcn_sched_barrier(0);
  request(Int<1>{}, 1, Int<PAIR ? NA : 0>{}, Int<ND>{});
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (S > 3) request(Int<2>{}, 2, Int<PAIR ? NA : 0>{}, Int<ND>{});
  __builtin_amdgcn_sched_barrier(0);
  // The low-rank term first, while the stages fill: what it loads is waited for together with them.  With two groups, the first
  // takes that of the first half of the row tiles.
  if constexpr (kLora) {
    if constexpr (KS == 1) {
      lora_add<MI>(lora_tiles(term...), r0 + wr * (16 * MI), rows, [&](int i, int j) -> f32x4& { return acc[i][j]; });
    } else {
      f32x4 half[MI / KS][NJ];
#pragma unroll
      for (int i = 0; i < MI / KS; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) half[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      lora_add<MI / KS>(lora_tiles(term...), r0 + wr * (16 * MI) + grp * (16 * MI / KS), rows, [&](int i, int j) -> f32x4& { return half[i][j]; });
#pragma unroll
      for (int i = 0; i < MI / KS; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            acc[i][j][v] = grp ? 0.f : half[i][j][v];
            acc[MI / KS + i][j][v] = grp ? half[i][j][v] : 0.f;
          }
    }
  }
  __builtin_amdgcn_s_waitcnt(wait_vm((S - 2) * (PAIR ? NB : ND)));
  bare_barrier();
  const bool second = PING && wv >= 4;   // the wavefront of a SIMD that is half a step behind
  if (second) bare_barrier();
  uint32_t kt = 0;
  for (; kt + S <= kboth; kt += S) {
    k_step(Int<0>{}, kt, Int<0>{});
    k_step(Int<1>{}, kt + 1, Int<0>{});
    k_step(Int<2>{}, kt + 2, Int<0>{});
    if constexpr (S > 3) k_step(Int<3>{}, kt + 3, Int<0>{});
  }
  if (kt < kmost) k_step(Int<0>{}, kt, Int<1>{});
  if (kt + 1 < kmost) k_step(Int<1>{}, kt + 1, Int<1>{});
  if ((S > 3 || KS > 1) && kt + 2 < kmost) k_step(Int<2>{}, kt + 2, Int<1>{});
  if constexpr (S > 3)
    if (KS > 1 && kt + 3 < kmost) k_step(Int<3>{}, kt + 3, Int<1>{});
  if (PING && !second) bare_barrier();   // every wavefront passes the same number of barriers
  __builtin_amdgcn_s_waitcnt(wait_vm(0));   // the stages are free once the last requests have arrived
  __syncthreads();

  // the row tiles this wavefront writes out: with two groups, the first half is summed and written by group 0,
  // the second by group 1
  constexpr int MO = MI / KS;
  f32x4 res[MO][NJ];
  if constexpr (KS > 1) {
    f32x4* ex = (f32x4*)(wave % 2 ? st1 : st0) + (wave / 2) * (2 * MO * NJ * 64);   // [for group][tile][lane]
#pragma unroll
    for (int i = 0; i < MO; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const f32x4 lo = acc[i][j], hi = acc[MO + i][j];
        f32x4 other;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          other[v] = grp ? lo[v] : hi[v];
          res[i][j][v] = grp ? hi[v] : lo[v];
        }
        ex[((1 - grp) * MO * NJ + i * NJ + j) * 64 + lane] = other;
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MO; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const f32x4 o = ex[(grp * MO * NJ + i * NJ + j) * 64 + lane];
#pragma unroll
        for (int v = 0; v < 4; ++v) res[i][j][v] += o[v];   // group 0's sum + group 1's, either way round
      }
    __syncthreads();
  } else {
#pragma unroll
    for (int i = 0; i < MO; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) res[i][j] = acc[i][j];
  }

  // Output, one row tile of every wavefront at a time, through an LDS strip of the wavefront's own (so no
  // barriers).  Accumulator element v of a lane: token row 4 * kg + v of the row tile, column jl of B tile j.  Staging
  // columns: plain, B tile j at 16 * j; SwiGLU, B tile j = 2 * f + matrix at CW / 2 * matrix + 16 * f.
  constexpr int ES = CW + 4;                       // floats per staged row
  constexpr int CPR = (SWIGLU ? CW / 2 : CW) / 8;  // 16-byte output chunks per row
  constexpr int RPP = 64 / CPR < 16 ? 64 / CPR : 16;   // rows per pass
  static_assert((NW * KS + 1) / 2 * 16 * ES * 4 <= KS * TT * 1024, "the strips of four wavefronts fit a stage");
  float(*e)[ES] = (float(*)[ES])((wv % 2 ? (char*)st1 : (char*)st0) + (wv / 2) * (16 * ES * 4));
#pragma unroll
  for (int i = 0; i < MO; ++i) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int col = SWIGLU ? (int)(CW / 2) * (j % 2) + 16 * (j / 2) + jl : 16 * j + jl;
#pragma unroll
      for (int v = 0; v < 4; ++v) e[4 * kg + v][col] = res[i][j][v];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if constexpr (kExperts && !SWIGLU) {
      // Products that wait for their weighted sum stay fp32; sixteen lanes have a row's 256 bytes, so a store fills whole lines.
#pragma unroll
      for (int ps = 0; ps < 4; ++ps) {
        const int rr = ps * 4 + lane / 16;
        const uint32_t row = ((grp * MO + i) * WR + wr) * 16 + rr, n = nt * BNF + wc * CW + 4 * (lane % 16);
        if (row < rows && n < dst.start[3])
          *(f32x4*)(only(term...).sums + (size_t)pair_of[row] * dst.start[3] + n) = *(const f32x4*)&e[rr][4 * (lane % 16)];
      }
      continue;
    }
    const int cc = lane % CPR;
#pragma unroll kEpilogue || kExperts ? 1 : 16 / RPP
    for (int ps = 0; ps < 16 / RPP; ++ps) {
      const int rr = ps * RPP + lane / CPR;
      const uint32_t row = kExperts ? ((grp * MO + i) * WR + wr) * 16 + rr : r0 + wr * (16 * MI) + (grp * MO + i) * 16 + rr;
      const uint32_t n = nt * BNF + wc * (BNF / WC) + 8 * cc;
      if (rr < 16 && row < rows && n < dst.start[3]) {
        float y[8];
        *(f32x4*)&y[0] = *(const f32x4*)&e[rr][8 * cc];
        *(f32x4*)&y[4] = *(const f32x4*)&e[rr][8 * cc + 4];
        const int which = n >= dst.start[2] ? 2 : n >= dst.start[1] ? 1 : 0;
        const uint32_t width = dst.start[which + 1] - dst.start[which], col = n - dst.start[which];
        size_t oo = (size_t)row * width + col;
        if constexpr (kExperts) oo = (size_t)pair_of[row] * width + col;
        if constexpr (kEpilogue) only(term...).apply(y, n);
        if (SWIGLU) {
          float u[8];
          *(f32x4*)&u[0] = *(const f32x4*)&e[rr][CW / 2 + 8 * cc];
          *(f32x4*)&u[4] = *(const f32x4*)&e[rr][CW / 2 + 8 * cc + 4];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            if constexpr (kExperts) y[k] = y[k] * __builtin_amdgcn_rcpf(1.0f + __expf(-y[k])) * u[k];
            else y[k] = y[k] / (1.0f + __expf(-y[k])) * u[k];
          }
        } else if (residual) {
          float rv[8];
          unpack16<BF16>(*(const u32x4*)(residual + oo), rv);
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] += rv[k];
        }
        if constexpr (kEpilogue) {
          if (only(term...).out32) {
            float* out = (float*)dst.ptr[0];
            *(f32x4*)(out + oo) = *(const f32x4*)&y[0];
            *(f32x4*)(out + oo + 4) = *(const f32x4*)&y[4];
            continue;
          }
        }
        const u32x4 o = pack16_round<BF16>(y);
        if (out_tiled) ((u32x4*)dst.ptr[which])[tiled_chunk(row, col, width)] = o;
        else *(u32x4*)(dst.ptr[which] + oo) = o;
      }
    }
  }
}

template <bool SWIGLU, bool XT, int MI, int NJ, int WR, int WC, int KS, bool PAIR, typename... TERM>
void launch_shape(const void* x, const void* w, const void* w2, const void* residual, const LinearOut& dst, uint32_t rows,
                  uint32_t K, uint32_t bcols, bool out_tiled, hipStream_t s, TERM... term) {
  const uint32_t NT = (bcols + 16 * NJ * WC - 1) / (16 * NJ * WC), RT = (rows + 16 * MI * WR - 1) / (16 * MI * WR);
  const dim3 grid(8 * ((RT * NT + 7) / 8)), block(64 * WR * WC * KS);
  hipLaunchKernelGGL((linear_rows_kernel<SWIGLU, XT, PAIR, MI, NJ, WR, WC, KS, TERM...>), grid, block, 0, s, (const uint16_t*)x,
                     (const u32x4*)w, (const u32x4*)w2, (const uint16_t*)residual, dst, rows, K, NT, out_tiled ? 1u : 0u, term...);
}

template <bool SWIGLU, bool XT, typename... TERM>
void launch_rows(const void* x, const void* w, const void* w2, const void* residual, const LinearOut& dst, uint32_t rows,
                 uint32_t K, uint32_t N, bool out_tiled, hipStream_t s, TERM... term) {
  const uint32_t bcols = SWIGLU ? 2 * N : N;
  const RowsShape shape = rows_shape(rows, bcols, K, XT);
  if constexpr (!SWIGLU && !XT) {
    // Row-major activations under 128 x 128 tiles (feature counts that 256 does not divide), many of them, and weights
    // that the last-level cache does not keep: in pairs.  us, in pairs | step by step, 70 shapes: 2894 rows, 10400 -> 11904
    // 872 | 972; 7647, 9120 -> 13184 2217 | 2411; 1172, 9792 -> 23936 794 | 839; 3463, 4416 -> 27520 1109 | 1205; 781, 5440 ->
    // 22912 300 | 298.  Fewer weights: 2236, 4288 -> 17280 415 | 390; K below 4000 up to 13 % slower.  Fewer
    // tiles (the activations of odd steps come later): 677, 10688 -> 11392 328 | 301.
    const uint64_t tiles = (uint64_t)((rows + 127) / 128) * ((N + 127) / 128);
    if (shape == kTile128 && (uint64_t)K * N >= (100u << 20) && tiles >= 850)
      return launch_shape<false, false, 4, 4, 2, 2, 1, true, TERM...>(x, w, w2, residual, dst, rows, K, bcols, out_tiled, s, term...);
  }
  switch (shape) {
    case kTile256: return launch_shape<SWIGLU, XT, 8, 4, 2, 4, 1, false, TERM...>(x, w, w2, residual, dst, rows, K, bcols, out_tiled, s, term...);
    case kTile128x512: return launch_shape<SWIGLU, XT, 4, 8, 2, 4, 1, false, TERM...>(x, w, w2, residual, dst, rows, K, bcols, out_tiled, s, term...);
    case kTile128x256: return launch_shape<SWIGLU, XT, 4, 4, 2, 4, 1, false, TERM...>(x, w, w2, residual, dst, rows, K, bcols, out_tiled, s, term...);
    case kTile128: return launch_shape<SWIGLU, XT, 4, 4, 2, 2, 1, false, TERM...>(x, w, w2, residual, dst, rows, K, bcols, out_tiled, s, term...);
    case kTile128K2: return launch_shape<SWIGLU, XT, 4, 4, 2, 2, 2, false, TERM...>(x, w, w2, residual, dst, rows, K, bcols, out_tiled, s, term...);
    case kTile128x64K2: return launch_shape<SWIGLU, XT, 2, 4, 4, 1, 2, false, TERM...>(x, w, w2, residual, dst, rows, K, bcols, out_tiled, s, term...);
    case kTile64K2: return launch_shape<SWIGLU, XT, 2, 2, 2, 2, 2, false, TERM...>(x, w, w2, residual, dst, rows, K, bcols, out_tiled, s, term...);
  }
}

}  // namespace

}  // namespace bct

#endif
