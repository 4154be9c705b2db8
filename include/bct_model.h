/* libbct -- the Llama-shaped glue around the bounded-cache attention layer.
 *
 * The paper applies its mechanism to the attention layers of a decoder-only
 * Transformer and obtains the write query and the write key-value vector from
 * the layer input with two learnable matrices (section 3.2 step 1, Algorithm 1:
 * wq_t = W_wq x_t, wv_t = W_wv x_t).  These entry points are the dense pieces
 * of such a stack, so that a token can go through whole layers on the GPU:
 * embedding lookup, RMS normalisation, the projections (W_q, W_wq, W_wv, W_o,
 * the SwiGLU MLP, the output head) and the greedy arg-max.  The attention
 * itself stays bct_decode_step / bct_prefill (include/bct.h).  For what each
 * request of a batch brings of its own: head norms with the rotation by its
 * position (bctm_qk_norm_rope), low-rank adapters beside the projections
 * (bctm_lora) and sampled instead of greedy tokens (bctm_sample).  For layers with
 * experts in place of the dense MLP: the router's product (bctm_linear_act), its
 * choice (bctm_route) and the experts' products (bctm_expert_swiglu,
 * bctm_expert_linear).
 *
 * All data pointers are DEVICE memory owned by the caller, bf16, row-major,
 * 16-byte aligned, unless a call says otherwise; token ids are int32.  Calls enqueue on the given stream and
 * return.  Status codes are those of include/bct.h.
 */
#ifndef BCT_MODEL_H
#define BCT_MODEL_H

#include <stddef.h>
#include <stdint.h>

#include "bct.h"

#ifdef __cplusplus
extern "C" {
#endif

/* out[r][:] = table[ids[r]][:], r < rows.  table [vocab][dim]; dim a multiple of 8.
 * Ids outside [0, vocab) give a zero row. */
bct_status bctm_embed(const int32_t* ids, const void* table, void* out, uint32_t rows, uint32_t vocab,
                      uint32_t dim, void* hip_stream);

/* Tiled activations.  A [rows][K] activation matrix that feeds a projection can be kept in the order the
 * projection's MFMA reads it, so that every wavefront load is one contiguous kilobyte: rows in groups of
 * 32, columns in groups of 32; group (r / 32, k / 32) is the 2 KB block number (r / 32) * (K / 32) + k / 32,
 * made of two 1 KB halves (rows 0-15, rows 16-31 of the group); in a half, element (r, k) sits at bf16
 * offset 8 * (16 * ((k % 32) / 8) + r % 16) + k % 8.  K must be a multiple of 32 and the buffer holds
 * 32 * ceil(rows / 32) * K bf16; rows past the end are never read for a stored result. */
#define BCTM_X_TILED 1u   /* the input x is tiled */
#define BCTM_OUT_TILED 2u /* the output is written tiled */

/* Row-major x [rows][K] -> tiled (above).  tiled must not be x. */
bct_status bctm_pack_rows(const void* x, void* tiled, uint32_t rows, uint32_t K, void* hip_stream);

/* out[r][:] = x[r][:] * rsqrt(mean(x[r][:]^2) + eps) * gain[:]   (fp32 arithmetic, bf16 in/out).
 * dim a multiple of 8, at most 16384.  flags: BCTM_OUT_TILED (then dim a multiple of 32, out not x). */
bct_status bctm_rmsnorm(const void* x, const void* gain, void* out, uint32_t rows, uint32_t dim, float eps,
                        uint32_t flags, void* hip_stream);

/* Queries and write queries of every head, normalised and turned by their token's position in one pass: what stands between
 * W_q, W_wq (section 3.2 step 1) and the bounded cache (bct_decode_step, bct_prefill).  For head x of row r:
 *   y = x * rsqrt(mean(x^2) + eps) * gain                               with BCTM_HEAD_NORM
 *   (y_a, y_b) = (y_a cos t - y_b sin t, y_a sin t + y_b cos t)         t = positions[r] * inv_freq[j], j < rotary_dim / 2
 * a = j and b = j + rotary_dim / 2, or with BCTM_ROPE_INTERLEAVED a = 2 j and b = 2 j + 1; elements from rotary_dim on pass.
 * fp32 arithmetic (the angle in 64 bits, for any position of an int32), one rounding.  The memory's keys do not turn, so scores
 * depend on a token's own position, not on a distance.
 * q: rows of n_q_heads heads side by side, q_ld elements from row to row (any distance of 64 bits), so heads are taken out of a
 * wider row (q | wq | wv) where they lie; k likewise, or NULL with n_kv_heads = 0.  An output may be its own input (same row distance); apart from
 * that no output shares memory with an input or the other output.  q_gain, k_gain [head_dim], NULL = ones.  positions int32
 * [rows], inv_freq float64 [rotary_dim / 2] in radians per position, both NULL with rotary_dim = 0.  All device memory.
 * head_dim and rotary_dim multiples of 16, at most 256; dtype: BCT_F32 or BCT_BF16, that of q, k, the gains and the outputs. */
#define BCTM_HEAD_NORM 4u
#define BCTM_ROPE_INTERLEAVED 8u
bct_status bctm_qk_norm_rope(const void* q, void* q_out, const void* q_gain, uint32_t n_q_heads, size_t q_ld,
                             size_t q_out_ld, const void* k, void* k_out, const void* k_gain, uint32_t n_kv_heads,
                             size_t k_ld, size_t k_out_ld, const int32_t* positions, const double* inv_freq,
                             uint32_t rotary_dim, uint32_t rows, uint32_t head_dim, float eps, int32_t dtype,
                             uint32_t flags, void* hip_stream);

/* Repacks a row-major weight matrix w [N][K] (one output feature per row) into the streaming layout
 * bctm_linear and bctm_swiglu read: 1 KB tiles of 16 features x 32 inputs, tile (n / 16, k / 32) at tile
 * index (n / 16) * (K / 32) + k / 32; inside a tile, element (n, k) sits at bf16 offset
 * 8 * (16 * ((k % 32) / 8) + n % 16) + k % 8.  Done once when weights are loaded.
 * N a multiple of 16, K a multiple of 32; packed holds N * K bf16 and must not be w. */
bct_status bctm_pack_weight(const void* w, void* packed, uint32_t N, uint32_t K, void* hip_stream);

/* out[r][n] = (residual ? residual[r][n] : 0) + sum_k x[r][k] * w[n][k].
 * x [rows][K] row-major, or tiled with flags = BCTM_X_TILED; w_packed = bctm_pack_weight of w [N][K];
 * out/residual [rows][N] row-major;
 * K a multiple of 32, N a multiple of 16; fp32 accumulation (MFMA), one rounding to bf16 at the end.  With few rows an infinite
 * activation may come out as a NaN (K tiles that fill up a round are multiplied by zero weights).
 * out may alias residual; x must not alias out.  Two kernels: up to 127 rows (a decode batch) the weights
 * are streamed once per 32 rows against activations read from cache; from 128 rows on (a prompt chunk), a tiled matrix-core
 * kernel runs instead where N is a multiple of 128 (bctm_swiglu: 64), or N is 128 to 16384 and the streaming kernel would have
 * more than 256 workgroups of 32 rows x 16 features (bctm_linear with K beyond 3072: 512), with workgroup tiles of
 * 64 x 64, 128 x 64, 128 x 128, 128 x 256, 256 x 256 and 128 x 512 chosen to fill the chip - fastest with a tiled x.  Both sum in fp32,
 * K in one or more parts added in order.  The tile depends on rows, N, K and x's order, the number of parts on rows, N and K
 * (bctm_linear_plan, bctm_linear_tile): equal calls give equal
 * bits, a tiled and a row-major x give the same bits, and so do calls of other rows or N with as many parts; calls with
 * other parts may differ in the last bits, a chunk's rows from the same rows alone or the parts of a bctm_linear_split
 * from separate projections. */
bct_status bctm_linear(const void* x, const void* w_packed, const void* residual, void* out, uint32_t rows,
                       uint32_t K, uint32_t N, uint32_t flags, void* hip_stream);

/* One projection with up to three row-major outputs: w_packed holds N0 + N1 + N2 features (packed as one
 * matrix, or matrix by matrix into consecutive parts of one buffer), the first N0 go to out0 [rows][N0], the
 * next N1 to out1 [rows][N1], the last N2 to out2 [rows][N2] (N2 may be 0, out2 then unused).  Every width a
 * multiple of 16.  For W_q, W_wq and W_wv, which read the same input. */
bct_status bctm_linear_split(const void* x, const void* w_packed, void* out0, uint32_t N0, void* out1, uint32_t N1,
                             void* out2, uint32_t N2, uint32_t rows, uint32_t K, uint32_t flags, void* hip_stream);

/* out[r][n] = silu(sum_k x[r][k] w_gate[n][k]) * (sum_k x[r][k] w_up[n][k]),  silu(a) = a / (1 + exp(-a)).
 * Both weights packed; same shape rules as bctm_linear.  flags: BCTM_X_TILED, BCTM_OUT_TILED (the output
 * as tiled activations of N columns, N a multiple of 32, ready to feed the next projection). */
bct_status bctm_swiglu(const void* x, const void* w_gate_packed, const void* w_up_packed, void* out, uint32_t rows,
                       uint32_t K, uint32_t N, uint32_t flags, void* hip_stream);

/* Low-rank adapters of many requests beside one shared projection: row r belongs to a request with the adapter
 * a = adapter[r], and its output has scale_a (x[r] A_a^T) B_a^T added before the one rounding.  Rows whose adapter is outside
 * [0, n_adapters) are those of the plain projection, bit for bit.
 *   a       the matrices A of all adapters, one below the other: [n_adapters][segments][rank][K], packed by one bctm_pack_weight of
 *           n_adapters * segments * rank features.  segments: 1 (bctm_linear_lora), the number of outputs (bctm_linear_split_lora:
 *           each output has an A of its own) or 2 (bctm_swiglu_lora: gate, then up)
 *   b       the matrices B, [n_adapters][N][rank], packed by one bctm_lora_pack of n_adapters * N features; N all features of
 *           the projection (all outputs together).  b_up: those of the up matrix in bctm_swiglu_lora, else NULL
 *   scale   float32 [n_adapters], NULL = 1;  adapter: int32 [rows]
 *   rank    a multiple of 16, at most 256; adapters of fewer ranks are filled up with zeros
 *   used    how many of these ranks are the adapters' own, 0 = all: x A^T is 0 for the others, whatever x holds (an infinity times
 *           a row of zeros would be a NaN)
 * workspace: 16-byte aligned, at least bctm_lora_workspace bytes, holds nothing between calls; it must not be in use by a call
 * on another stream.  All but the struct is device memory.  x A^T is summed in fp32 and enters the second product as that.
 * A row's bits depend on the sizes of the call and on its own adapter, not on the other rows'.
 * A NaN or an infinity in one adapter reaches the rows of that adapter alone. */
typedef struct {
  const void* a;
  const void* b;
  const void* b_up;
  const float* scale;
  const int32_t* adapter;
  uint32_t n_adapters, rank;
  void* workspace;
  size_t workspace_bytes;
  uint32_t used;
} bctm_lora;

/* Bytes of workspace a call of these sizes, or of fewer rows, needs (host call, no GPU needed). */
bct_status bctm_lora_workspace(uint32_t rows, uint32_t K, uint32_t rank, uint32_t segments, size_t* bytes);

/* Repacks row-major b [N][rank] into 16-byte chunks of 8 ranks of one feature, chunk (n / 16 * rank / 8 + k / 8) * 16 + n % 16.
 * Done once when adapters are loaded.  N and rank multiples of 16; packed holds N * rank bf16 and must not be b. */
bct_status bctm_lora_pack(const void* b, void* packed, uint32_t N, uint32_t rank, void* hip_stream);

/* bctm_linear, bctm_linear_split and bctm_swiglu with adapters; everything else as in those. */
bct_status bctm_linear_lora(const void* x, const void* w_packed, const void* residual, void* out, uint32_t rows, uint32_t K,
                            uint32_t N, uint32_t flags, const bctm_lora* lora, void* hip_stream);
bct_status bctm_linear_split_lora(const void* x, const void* w_packed, void* out0, uint32_t N0, void* out1, uint32_t N1,
                                  void* out2, uint32_t N2, uint32_t rows, uint32_t K, uint32_t flags, const bctm_lora* lora,
                                  void* hip_stream);
bct_status bctm_swiglu_lora(const void* x, const void* w_gate_packed, const void* w_up_packed, void* out, uint32_t rows,
                            uint32_t K, uint32_t N, uint32_t flags, const bctm_lora* lora, void* hip_stream);

/* out[r][n] = (residual ? residual[r][n] : 0) + act((bias ? bias[n] : 0) + sum_k x[r][k] * w[n][k]), everything after the sum in fp32 and
 * rounded once.  bias: bf16 [N].  act: one of BCTM_ACT_.  flags: BCTM_X_TILED as in bctm_linear; BCTM_OUT_F32: out is float32
 * (a router's logits), else bf16; BCTM_OUT_TILED: bf16 as tiled activations (N a multiple of 32).  residual: bf16, row-major; a
 * row-major bf16 out may be the residual.  Shapes as in bctm_linear, and its kernels and sums but for N a multiple of 64 and 17 rows or
 * more, where a kernel for few features, which sums K in eight parts, runs if one round of its workgroups (16 or 32 rows x 64
 * features) is enough, or N is 64; up to 127 rows for N up to 256.  A tiled and a row-major x give the same bits. */
#define BCTM_OUT_F32 16u
#define BCTM_ACT_NONE 0u
#define BCTM_ACT_RELU 1u
#define BCTM_ACT_SILU 2u      /* y / (1 + exp(-y)) */
#define BCTM_ACT_GELU 3u      /* y (1 + erf(y / sqrt 2)) / 2, the factor of y within 2e-7 */
#define BCTM_ACT_GELU_TANH 4u /* y (1 + tanh(sqrt(2 / pi) (y + 0.044715 y^3))) / 2 */
#define BCTM_ACT_SIGMOID 5u   /* 1 / (1 + exp(-y)) */
bct_status bctm_linear_act(const void* x, const void* w_packed, const void* bias, const void* residual, void* out, uint32_t rows,
                           uint32_t K, uint32_t N, uint32_t act, uint32_t flags, void* hip_stream);

/* Layers with experts: a token goes through k of n_experts MLPs, chosen by a router, and gets the sum of their outputs, weighted.
 * A pair is a token and one of its slots, number token * k + slot.  n_experts at most 512, k at most 16 and n_experts.
 *
 * bctm_route: each token's experts and their weights from its logits [rows], n_experts each, ld >= n_experts elements from row to
 * row, float32 or bf16 (dtype), aligned to their type.
 *   p       softmax of the logits, or with BCTM_ROUTE_SIGMOID 1 / (1 + exp(-logit)) of each
 *   chosen  the k experts with the largest logit, or with a bias (float32 [n_experts]) the largest p + bias, which is compared
 *           in 64 bits; in descending order, equal ones by number.  A logit of NaN or -inf (or a bias of these) is never chosen.
 *   weight  scale * p, with BCTM_ROUTE_NORMALISE divided by the sum of the chosen p
 * experts int32 [rows][k], weights float32 [rows][k]: -1 and 0 in slots for which no expert is left (a padding row: all logits -inf).
 * plan: the pairs by expert, for the calls below (or NULL).
 *
 * bctm_expert_plan: the same plan for experts that the caller chose; outside [0, n_experts): none.
 *
 * A plan is 16-byte aligned device memory of at least bctm_expert_plan_bytes bytes and holds for the sizes it was made for; calls only read
 * it.  As int32 it begins with offsets [n_experts + 1], and at *order (if that is asked for) is order [rows * k]:
 * the pairs of expert e are order[offsets[e]] .. order[offsets[e + 1] - 1], by number, and those without an expert follow the last.
 */
#define BCTM_ROUTE_SIGMOID 1u
#define BCTM_ROUTE_NORMALISE 2u
bct_status bctm_expert_plan_bytes(uint32_t rows, uint32_t k, uint32_t n_experts, size_t* bytes, size_t* order);
bct_status bctm_route(const void* logits, size_t ld, const float* bias, int32_t* experts, float* weights, void* plan,
                      size_t plan_bytes, uint32_t rows, uint32_t n_experts, uint32_t k, float scale, int32_t dtype, uint32_t flags,
                      void* hip_stream);
bct_status bctm_expert_plan(const int32_t* experts, void* plan, size_t plan_bytes, uint32_t rows, uint32_t n_experts, uint32_t k,
                            void* hip_stream);

/* out[p][n] = silu(g) * u for every pair p with an expert e: g = sum_j x[p / k][j] w_gate[e][n][j], u likewise with w_up; rows of
 * pairs without one are left as they were.  x [rows][K], out [rows * k][N], row-major; w_gate, w_up: the matrices [N][K] of
 * all experts one below the other, each packed by one bctm_pack_weight of n_experts * N features (or expert by expert).  K a multiple
 * of 32, N of 16.  fp32 accumulation, one rounding.  A row's bits depend on the sizes of the call alone, not on the other tokens'
 * experts. */
bct_status bctm_expert_swiglu(const void* x, const void* w_gate_packed, const void* w_up_packed, void* out, const void* plan,
                              uint32_t rows, uint32_t k, uint32_t n_experts, uint32_t K, uint32_t N, void* hip_stream);

/* Which tile of pairs x features the launch of that call or of the next one gives a workgroup (swiglu = 1: bctm_expert_swiglu, 0:
 * bctm_expert_linear); host logic only. */
bct_status bctm_expert_tile(uint32_t rows, uint32_t k, uint32_t n_experts, uint32_t K, uint32_t N, uint32_t swiglu, uint32_t* tile_rows,
                            uint32_t* tile_features);

/* out[r][n] = (residual ? residual[r][n] : 0) + sum over the slots s of r with an expert e of weights[r][s] * sum_j h[r k + s][j] w[e][n][j].
 * h [rows * k][K] (rows of pairs without an expert are not read), weights float32 [rows][k], out and residual [rows][N]; out may be the
 * residual.  Products, weights and sums in fp32, slots in their order, rounded once at the end.  workspace: 16-byte aligned, at least
 * bctm_expert_workspace bytes, holds nothing between calls; it must not be in use by a call on another stream. */
bct_status bctm_expert_workspace(uint32_t rows, uint32_t k, uint32_t N, size_t* bytes);
bct_status bctm_expert_linear(const void* h, const void* w_packed, const void* plan, const float* weights, const void* residual, void* out,
                              void* workspace, size_t workspace_bytes, uint32_t rows, uint32_t k, uint32_t n_experts, uint32_t K,
                              uint32_t N, void* hip_stream);

/* Which kernel bctm_linear / bctm_linear_split (swiglu = 0, N their widths together) or bctm_swiglu (swiglu = 1) launches
 * for a shape: host logic only, no GPU call.  *kernel receives one of the values below.  The last two of them
 * name the same matrix-core kernel in two ranges of shapes; which tile it gives a workgroup there is
 * bctm_linear_tile's answer. */
#define BCTM_KERNEL_STREAMING 0u /* weights streamed once per 32 rows (one 16-feature tile per workgroup) */
#define BCTM_KERNEL_STREAMING_WIDE 1u /* the same with two feature tiles per workgroup (wide output heads) */
#define BCTM_KERNEL_STREAMING_TRIPLE 4u /* streaming with three feature tiles per workgroup */
#define BCTM_KERNEL_TILE128 2u   /* matrix-core kernel, 128 to 1023 rows or N no multiple of 256 (SwiGLU: 128) */
#define BCTM_KERNEL_TILE256 3u   /* matrix-core kernel, from 1024 rows on and N a multiple of 256 (SwiGLU: 128) */
bct_status bctm_linear_plan(uint32_t rows, uint32_t K, uint32_t N, uint32_t swiglu, uint32_t* kernel);

/* What that launch gives one workgroup: *tile_rows token rows x *tile_features features, K summed in *k_parts parts.
 * flags: BCTM_X_TILED as in the call.  Host logic only, the launches go by the same functions. */
bct_status bctm_linear_tile(uint32_t rows, uint32_t K, uint32_t N, uint32_t swiglu, uint32_t flags, uint32_t* tile_rows,
                            uint32_t* tile_features, uint32_t* k_parts);

/* ids[r] = index of the largest logits[r][:] (the lowest index among equal maxima). */
bct_status bctm_argmax(const void* logits, int32_t* ids, uint32_t rows, uint32_t N, void* hip_stream);

/* The next token of each sequence drawn from its logits, with settings of its own and one uniform number
 * (bctm_argmax is the greedy choice).  logits [rows], N tokens each, ld >= N elements from row to row, float32 or
 * bf16 (dtype; aligned to their type, fastest where rows are 16-byte aligned).  Tokens in descending order of their logit, equal
 * ones by index; a logit of NaN or -inf is never drawn.  With w = exp((l - max) / temperature) and cum(j) the sum of the first j:
 *   kept   the first n: the least of top_k (0 or less: all), the fewest with cum(n) >= top_p * cum(top_k) (1 or more: all) and
 *          how many have w >= min_p (0 or less: all); at least 1
 *   drawn  the first j with cum(j) > u * cum(n)
 * temperature, top_p, min_p: float32 [rows], top_k int32 [rows], each NULL = 1, 1, 0, 0 for all; u float32 [rows] in [0, 1), below
 * taken as 0, above as the last number before 1; all device memory.  A temperature of 0 (or below, or NaN) draws the most likely
 * token, bctm_argmax's but for NaN; NaN elsewhere switches that setting off.  Infinite logits share the draw equally.
 * ids int32 [rows]: the tokens, -1 in a row that has none left; prob float32 [rows] or NULL: w / cum(n) of each, 0 with -1.
 * Weights and sums have 46 bits behind the binary point of the largest weight (62 less log2 N beyond 65536 tokens), added as integers:
 * equal calls draw equal tokens, and a tail of smaller weights is not there.  N at most 4194304. */
bct_status bctm_sample(const void* logits, size_t ld, const float* temperature, const int32_t* top_k, const float* top_p,
                       const float* min_p, const float* u, int32_t* ids, float* prob, uint32_t rows, uint32_t N,
                       int32_t dtype, void* hip_stream);

/* Thread-local detail of the last failure of a bctm_ call. */
const char* bctm_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* BCT_MODEL_H */
