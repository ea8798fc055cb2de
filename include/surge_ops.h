/*
 * surge_ops.h - stage-level entry points of the SuperBatch encoder.
 *
 * Each call runs one stage of the encode path on caller-provided device
 * buffers, with the same kernels surge_encode_superbatch launches, so every
 * stage can be checked on its own.  The call is synchronous unless its
 * comment says otherwise: it enqueues on `hip_stream` (NULL = null stream)
 * and waits for it before returning.
 * bf16 tensors are passed as uint16_t bit patterns.  Text boundaries are
 * given as host int64 cu_seqlens [n_texts+1] (cu[0] = 0, increasing), checked
 * on the host and copied to the device by the call.  Returns the status
 * codes of surge.h.
 */
#ifndef SURGE_OPS_H_
#define SURGE_OPS_H_

#include <stdint.h>

#include "surge.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Embedding gather + LayerNorm (encoder input; positions restart at 0 for
 * every text): out[t] = LN(word[id_t] + pos[t - cu_i]).
 * d_tokens int32 [cu[n]]; d_word bf16 [vocab, d]; d_pos bf16 [max_pos, d];
 * gamma/beta fp32 [d]; d_out bf16 [cu[n], d].  d % 128 == 0, d <= 1024,
 * every text length <= min(max_pos, 4096).  Out-of-vocabulary IDs are read
 * as ID 0 and reported with SURGE_ERR_INVALID_ARGUMENT after the stage ran.
 */
surge_status surge_op_embed_ln(int64_t n_texts, const int64_t* h_cu_seqlens, const int32_t* d_tokens,
                               const uint16_t* d_word, int32_t vocab, const uint16_t* d_pos,
                               int32_t max_pos, const float* d_gamma, const float* d_beta,
                               float eps, int32_t d, uint16_t* d_out, void* hip_stream);

/*
 * Linear layer over packed tokens: Y = epi(X W^T + b).
 * d_x bf16 [M, K]; d_w bf16 [N, K] (out, in); d_bias fp32 [N];
 * epilogue 0 = bias, 1 = bias then exact GELU, 2 = bias then + d_res
 * (bf16 [M, N]); d_y bf16 [M, N].  M >= 1, N % 128 == 0, K % 64 == 0.
 */
surge_status surge_op_linear(int64_t M, int32_t N, int32_t K, const uint16_t* d_x,
                             const uint16_t* d_w, const float* d_bias, const uint16_t* d_res,
                             int32_t epilogue, uint16_t* d_y, void* hip_stream);

/*
 * The linear layer's LayerNorm-fused forms (post-LN encoder with every
 * LayerNorm except the last folded into its neighbours; LN(v) = gamma (v -
 * mu) / sqrt(var + eps) + beta over a row, biased variance):
 *   epilogue 3: y = LN(x) W^T + b for raw rows x of d_x, computed as
 *               rstd (x W'^T - mu s) + b' with d_w = W' = bf16(W diag(gamma)),
 *               d_col_s = s = row sums of W' [N] and d_bias = b' = b + W beta;
 *               the row statistics of x come from d_stats_in;
 *   epilogue 4: epilogue 3, then exact GELU;
 *   epilogue 5: y = x W^T + b + res, and the statistics of y's rows are
 *               written to d_stats_out;
 *   epilogue 6: y = x W^T + b + LN(res) with res's statistics in d_stats_in
 *               and LN's gamma, beta in d_gamma, d_beta [N]; statistics of y
 *               to d_stats_out.
 *   epilogues 0-2 as surge_op_linear.
 * Statistics are partials of W = surge_op_linear_stats_width(M, N) (64)
 * consecutive features of a row: fp32 pairs (mean, variance) at
 * [(p * M + row) * 2], p < N / W.  d_stats_in holds parts_in partials of
 * equal width per row (the producer's N / W).  Shapes as surge_op_linear;
 * float vectors 16-byte aligned.
 */
surge_status surge_op_linear_ln(int64_t M, int32_t N, int32_t K, const uint16_t* d_x,
                                const uint16_t* d_w, const float* d_bias, const uint16_t* d_res,
                                int32_t epilogue, const float* d_stats_in, int32_t parts_in,
                                const float* d_col_s, const float* d_gamma, const float* d_beta,
                                float eps, float* d_stats_out, uint16_t* d_y, void* hip_stream);

/*
 * surge_op_linear_ln without any allocation, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc): the per-row LayerNorm factors that the
 * folded and residual-LayerNorm epilogues (3, 4, 6) read live in a static
 * device array of the library (4 MiB: at most 524,288 rows), not in a buffer
 * allocated per call.  Same arguments, checks, kernels and results as
 * surge_op_linear_ln, but asynchronous: the call only enqueues on
 * `hip_stream` (no synchronisation).  M above 524,288 with epilogue 3, 4 or
 * 6 returns SURGE_ERR_CAPACITY before anything is enqueued.  Every call on
 * one GPU shares that GPU's array (each call overwrites the rows it uses
 * before reading them): calls on one stream are ordered, calls that overlap
 * on different streams of one GPU race.  Calls no hipMalloc/hipFree.
 */
surge_status surge_op_linear_ln_noalloc(int64_t M, int32_t N, int32_t K, const uint16_t* d_x,
                                        const uint16_t* d_w, const float* d_bias,
                                        const uint16_t* d_res, int32_t epilogue,
                                        const float* d_stats_in, int32_t parts_in,
                                        const float* d_col_s, const float* d_gamma,
                                        const float* d_beta, float eps, float* d_stats_out,
                                        uint16_t* d_y, void* hip_stream);

/* Features per statistics partial of an [M, N] linear output (host-only). */
int32_t surge_op_linear_stats_width(int64_t M, int32_t N);

/*
 * The tile that the linear layer's launch takes for an [M, N] output of K
 * inputs on a device of n_cus compute units, rows << 16 | features (host-only;
 * 0 for shapes that the layer refuses).  Where N is not a multiple of the
 * features, the last 128 take 128 x 128 tiles.  Every tile gives the same
 * bits.
 */
int32_t surge_op_linear_tile(int64_t M, int32_t N, int32_t K, int32_t n_cus);

/*
 * Packed varlen multi-head self-attention within each text:
 * out[rows of text i, head h] = softmax(Q_h K_h^T / sqrt(d_head)) V_h.
 * d_qkv bf16 [T, 3 n_heads d_head] (Q | K | V blocks, head h at columns
 * h d_head of each); d_out bf16 [T, n_heads d_head]; T = cu[n_texts].
 * d_head is 32 or 64; n_heads * d_head % 128 == 0; every text length in
 * [1, 4096].
 */
surge_status surge_op_attention(int64_t n_texts, const int64_t* h_cu_seqlens, int32_t n_heads,
                                int32_t d_head, const uint16_t* d_qkv, uint16_t* d_out,
                                void* hip_stream);

/* Row LayerNorm: y = gamma (x - mean) / sqrt(var + eps) + beta, biased
 * variance.  d_x, d_y bf16 [M, d]; d % 8 == 0, d <= 1024. */
surge_status surge_op_layernorm(int64_t M, int32_t d, const uint16_t* d_x, const float* d_gamma,
                                const float* d_beta, float eps, uint16_t* d_y, void* hip_stream);

/* Masked mean pooling + L2 normalisation: out[i] = e_i / max(||e_i||, 1e-12)
 * with e_i the mean of text i's rows of d_x (bf16 [T, d]); d_out fp32
 * [n_texts, d], 16-byte aligned.  d % 128 == 0, d <= 1024. */
surge_status surge_op_pool_l2(int64_t n_texts, const int64_t* h_cu_seqlens, int32_t d,
                              const uint16_t* d_x, float* d_out, void* hip_stream);

/*
 * Operators of models that read the encoder's token states (a reranker, a
 * pooling head with latent queries, a decoder of answers): the linear layer
 * in 8-bit integers, the norms around a block, and attention to a text's
 * states.  Unlike the stages above these calls only enqueue on `hip_stream`:
 * they do not synchronise, allocate or copy, so they can be captured into a
 * HIP graph (with buffers, workspace and plan that live as long as the
 * graph).  Buffers and stream belong to the current device.  A matrix has a
 * row stride `ld`, in elements, of at most 2^22, and 16-byte aligned rows
 * (ld a multiple of 8 for bf16, of 16 for int8).  M = 0 rows is a call that
 * does nothing.
 */

/*
 * Rows quantized to int8 with a scale per row (per token of activations, per
 * output channel of a weight): with a = max(max_k |x[m][k]|, 2^-100),
 *   q[m][k] = round(x[m][k] * (127 / a)) (ties to even), scale[m] = a / 127.
 * d_x bf16 [M, K]; d_q int8 [M, K rounded up to a multiple of 128], the
 * columns from K on set to 0; d_scale fp32 [M].  A row with an infinity or a
 * NaN gets q = 0 and scale = NaN, which marks every output made from it.
 * K % 8 == 0, K <= 16384.  d_q must not overlap d_x.
 */
surge_status surge_op_quantize_rows(int64_t M, int32_t K, const uint16_t* d_x, int64_t ld_x,
                                    int8_t* d_q, int64_t ld_q, float* d_scale, void* hip_stream);

/*
 * Linear layer in 8-bit integers with scales for each token and channel:
 *   y[m][n] = epi(x_scale[m] w_scale[n] sum_k x[m][k] w[n][k] + bias[n]),
 * in fp32 from the exact sum on: times x_scale, times w_scale, plus bias.
 * d_x int8 [M, K]; d_x_scale fp32 [M]; d_w int8 [N, K] contiguous (out, in);
 * d_w_scale, d_bias fp32 [N], 16-byte aligned; epilogue as surge_op_linear (0
 * bias, 1 exact GELU, 2 + d_res, bf16 [M, N]); d_y bf16 [M, N].  The sum over
 * k is exact (32-bit integers).  K % 128 == 0, K <= 65536 (pad both operands
 * with zeros, as surge_op_quantize_rows does); N % 8 == 0, N <= 2^20.  d_y
 * may be d_res with the same stride; it must not overlap the other inputs.
 */
surge_status surge_op_linear_i8(int64_t M, int32_t N, int32_t K, const int8_t* d_x, int64_t ld_x,
                                const float* d_x_scale, const int8_t* d_w, const float* d_w_scale,
                                const float* d_bias, const uint16_t* d_res, int64_t ld_res,
                                int32_t epilogue, uint16_t* d_y, int64_t ld_y, void* hip_stream);

/*
 * The tile that the layer's launch takes for an [M, N] output of K inputs on a
 * device of n_cus compute units, rows << 16 | channels (host-only; 0 for
 * shapes that the layer refuses).  Where 256-wide tiles leave some of N over,
 * the rest takes a launch of its own.  Every tile gives the same bits.
 */
int32_t surge_op_linear_i8_tile(int64_t M, int32_t N, int32_t K, int32_t n_cus);

/* Norms of surge_op_block_norm over a row v of d features. */
#define SURGE_NORM_LAYER 0 /* gamma (v - mean) / sqrt(var + eps) + beta, biased variance */
#define SURGE_NORM_RMS 1   /* gamma v / sqrt(mean of v^2 + eps) */

/*
 * What lies between two blocks of a model, in one pass over the rows:
 *   y = res_scale * x + gate * gate_rows * N_post(block)
 *   z = N_pre(y)
 * d_x, d_block, d_gate_rows bf16 [M, d]; the gammas, betas and d_gate fp32
 * [d], 16-byte aligned.  Outputs: d_y bf16 [M, d], the residual stream; d_z
 * bf16 [M, d], the next block's input; d_zq int8 with d_zq_scale fp32 [M],
 * the same rows as surge_op_quantize_rows gives them, before a rounding to
 * bf16 (d_zq has d rounded up to a multiple of 128 columns).  Each output may
 * be NULL, not all.  z is made from y before its rounding to bf16; a row whose
 * sum of features overflows fp32 has NaN in z under SURGE_NORM_LAYER.
 * NULL inputs: d_block (y = res_scale * x; then no post norm or gate),
 * d_post_gamma (no norm after the block), either beta (0; always NULL for
 * SURGE_NORM_RMS), d_gate, d_gate_rows (1).  d_pre_gamma is needed for z.
 * d_gate is multiplied into d_post_gamma and d_post_beta first: it is finite
 * wherever that beta is not 0.
 * d % 8 == 0, d <= 8192; eps in [0, 1].  d_y and d_z may each be d_x, d_block
 * or d_gate_rows with the same stride (not the same one); otherwise outputs
 * must not overlap inputs or each other.
 */
surge_status surge_op_block_norm(int64_t M, int32_t d, int32_t kind, const uint16_t* d_x,
                                 int64_t ld_x, const uint16_t* d_block, int64_t ld_block,
                                 const float* d_post_gamma, const float* d_post_beta,
                                 const float* d_gate, const uint16_t* d_gate_rows, int64_t ld_gate,
                                 float res_scale, const float* d_pre_gamma, const float* d_pre_beta,
                                 float eps, uint16_t* d_y, int64_t ld_y, uint16_t* d_z, int64_t ld_z,
                                 int8_t* d_zq, int64_t ld_zq, float* d_zq_scale, void* hip_stream);

/*
 * The work list of cross attention for a batch's lengths, on the current
 * device.  Sequence i has the queries cu_q[i] .. cu_q[i+1]-1 and the states
 * cu_kv[i] .. cu_kv[i+1]-1 of its text (host int64 [n_seqs+1], from 0, never
 * decreasing: either length may be 0).  n_heads query heads share n_kv_heads
 * key heads in equal groups (head h reads key head h / (n_heads /
 * n_kv_heads)); d_head is 32, 64 or 128.  The lengths of a text's states stay
 * what they are over the layers and steps of its reader, so a plan is made
 * once.  It is not changed by the calls that use it, from any thread or
 * stream; destroy it after the last of them has finished.  Create and
 * destroy allocate, copy and free device memory and cannot be captured.
 */
typedef struct surge_cross_plan surge_cross_plan;
surge_status surge_cross_plan_create(int64_t n_seqs, const int64_t* h_cu_q, const int64_t* h_cu_kv,
                                     int32_t n_heads, int32_t n_kv_heads, int32_t d_head,
                                     surge_cross_plan** out);
void surge_cross_plan_destroy(surge_cross_plan* plan);

/* Bytes of workspace that a call needs, the units of work it launches and
 * how many of them hold a part of their rows' keys.  Each pointer may be
 * NULL. */
surge_status surge_cross_plan_info(const surge_cross_plan* plan, int64_t* workspace_bytes,
                                   int64_t* n_units, int64_t* n_parts);

/*
 * Cross attention: out[t][h] = sum_k p_k v[k] / sum_k p_k over the states k
 * of t's text, p_k = exp(scale q[t][h] . k[k]); a sequence without states, or
 * with none left by the mask, gives zeros.  Scores, log2(e) scale q . k, are
 * fp32: a row of which one is a NaN, the largest overflows or none is above
 * -infinity gives NaN.  Maxima, sums and outputs are fp32; each p_k is rounded
 * to bf16, the type of v, for its product with v, but not in the sum of p_k:
 * outputs are off by up to 2^-8 of sum_k p_k |v[k]| / sum_k p_k, and their own
 * rounding.
 * d_q, d_out bf16 [cu_q[n], n_heads d_head]; d_k, d_v bf16 [cu_kv[n],
 * n_kv_heads d_head] (two column ranges of one projection's output, say, with
 * its stride); d_key_mask one byte per state, 0 leaves it out (what stands in
 * its rows of k and v does not matter), or NULL; scale positive, below 2^127.
 * d_workspace: 16-byte aligned, of at least the plan's bytes (NULL where
 * that is 0), used until the call's work is done: calls that may run at the
 * same time, graph replays among them, need one each.  d_out must not
 * overlap an input.
 */
surge_status surge_op_cross_attention(const surge_cross_plan* plan, const uint16_t* d_q, int64_t ld_q,
                                      const uint16_t* d_k, int64_t ld_k, const uint16_t* d_v,
                                      int64_t ld_v, const uint8_t* d_key_mask, float scale,
                                      void* d_workspace, int64_t workspace_bytes, uint16_t* d_out,
                                      int64_t ld_out, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* SURGE_OPS_H_ */
