/*
 * rlhf_ops.h -- kernel-level entry points of the same library, for per-kernel parity tests
 * and roofline measurements.  The stage API in rlhf.h is built from exactly these kernels.
 *
 * All pointers are DEVICE pointers owned by the caller; `stream` is a hipStream_t (NULL =
 * the default stream).  Calls enqueue work and return without waiting.  Return values are
 * rlhf_status codes (0 = OK, RLHF_EINVAL for unsupported shapes, RLHF_EDEVICE for a failed
 * launch).  dtype is an rlhf_dtype: the storage type of the weights.
 */
#ifndef RLHF_OPS_H
#define RLHF_OPS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Linear projection y = W x of a decoder block (the matrix work of both the memory-bound
 * decoding phase, Section 4.2, and the prefill-like inference forward, Section 2.1):
 * C[s][m][n] = sum over the s-th K range of A[m][k] * W[n][k].  W [N,K] row-major in dtype;
 * A [M,K] in dtype, or (act_half != 0, bf16 weights only) in IEEE half, the activation type
 * of prefill / scoring passes; C float32 [nsplit][M][N]; the caller sums the nsplit partial
 * planes.  K must be a multiple of 8 (bf16) or 4 (fp32).  variant 0 takes the tiling the
 * stage uses for M rows; a positive value forces one of the library's tilings (benchmarks;
 * RLHF_EINVAL if it does not exist or cannot split K).  rlhf_op_gemm_nsplit returns the split
 * the stage itself would choose for this shape, at most max_split. */
/* Half copies of the weights: rlhf_op_bf16_to_half converts n (even) bf16 elements to IEEE half the
 * way the kernels do on the fly (exact for magnitudes >= 2^-14, toward zero on half's subnormal
 * grid below).  With such a copy as W, rlhf_op_gemm takes dtype = 2 (A must be half, K a multiple
 * of 64; the 256 x 256 tiling with both operands loaded global -> LDS directly, any nsplit whose
 * ranges are non-empty; A and W each smaller than 4 GiB, else RLHF_EINVAL), and
 * rlhf_op_gemm_swiglu / rlhf_op_gemm_rope / rlhf_op_lm_head_logprob take act_half = 2 under the
 * same conditions.  This is what the stage runs in passes of more than 256 rows when the engine
 * option half_weight_copies is set; results are bit-identical to the bf16-weight path. */
int rlhf_op_bf16_to_half(const void* src, void* dst, int64_t n, void* stream);
int rlhf_op_gemm_nsplit(int dtype, int M, int N, int K, int max_split);
int rlhf_op_gemm(int dtype, int act_half, const void* A, const void* W, float* C, int M, int N, int K,
                 int nsplit, int variant, void* stream);

/* Host-side copy of the workgroup -> tile mapping of the compute-bound (256 x 256) launches, for
 * tests of that mapping: rlhf_op_gemm_tall_grid is the number of workgroups launched for a grid of
 * tiles_m x tiles_n tiles; rlhf_op_gemm_tall_tile returns 1 and the tile (*tm, *tn) workgroup bid
 * computes, 0 if it has none, RLHF_EINVAL on bad arguments.  The 8 XCDs (bid modulo 8) walk the same
 * panel of 8 tile rows at the same time, each over a contiguous group of tile columns of its own. */
int rlhf_op_gemm_tall_grid(int tiles_m, int tiles_n);
int rlhf_op_gemm_tall_tile(int bid, int tiles_m, int tiles_n, int* tm, int* tn);

/* Gate||up projection of the SwiGLU MLP with the activation fused into the epilogue, as the
 * stage runs it in prefill / scoring passes: act[m][c] = silu(<A[m], W[c]>) * <A[m], W[ffn + c]>.
 * W_gate_up bf16 [2*ffn, K] (gate rows, then up rows); A and act IEEE half (act_half != 0) or
 * bf16, [M, K] and [M, ffn].  Needs M >= 512, ffn and K multiples of 8 (else RLHF_EINVAL); or
 * 1 <= M <= 16 and K a multiple of 256: the few-row kernel of decode steps, whose workgroups walk
 * the whole K range (no split) so that SwiGLU can ride in the epilogue there too. */
int rlhf_op_gemm_swiglu(int act_half, const void* A, const void* W_gate_up, void* act, int M, int ffn, int K,
                        void* stream);

/* QKV projection of a prefill / scoring pass with the rotary embedding fused into the epilogue,
 * as the stage runs it for bf16 models (Section 2.1, the attention input of a decoder block):
 * row m of A [M, K] (IEEE half if act_half != 0, else bf16) times W_qkv bf16
 * [(n_q_heads + 2*n_kv_heads)*head_dim, K] (query rows, key rows, value rows); query and key
 * heads are rotated by position pos[m] (pair (i, i + head_dim/2), cosine and sine taken from
 * table, float32 [max position][head_dim/2][cos, sin]); results are rounded to A's type and
 * written to q [M, n_q_heads*head_dim] and, where non-NULL, to k, v [M, n_kv_heads*head_dim] and
 * to the paged pool (layout as in rlhf_op_paged_decode_attention) at token slot kv_dst[m] =
 * page*16 + offset.  Needs M >= 512, K a multiple of 64, head_dim 64 or 128 (else RLHF_EINVAL); or
 * 1 <= M <= 16 and K a multiple of 256: the few-row kernel of decode steps (no K split, rotary and
 * the KV-cache append in its epilogue). */
int rlhf_op_gemm_rope(int act_half, const void* A, const void* W_qkv, const int32_t* pos, const int32_t* kv_dst,
                      const float* table, void* q, void* k, void* v, void* pool, int M, int K, int layer,
                      int n_layers, int n_q_heads, int n_kv_heads, int head_dim, void* stream);

/* Decode attention of one step (Section 2.1, decoding phase): row r holds one query
 * [n_q_heads * head_dim] and attends to the ctx_len[r] cached tokens of the sample whose
 * page-table row is row_sample[r].  pool layout: [page][layer][K|V][kv_head][16][head_dim].
 * Here dtype is the element type of q, pool and out: RLHF_FP32, RLHF_BF16, or 2 = IEEE half
 * (what the stage uses for bf16 models).
 * part_acc / part_ml are float32 scratch of rows*n_q_heads*nsplit*head_dim and
 * rows*n_q_heads*nsplit*2 entries (unused when nsplit == 1). */
int rlhf_op_paged_decode_attention(int dtype, const void* q, const void* pool, const int32_t* page_table,
                                   int pt_stride, const int32_t* row_sample, const int32_t* ctx_len,
                                   void* out, float* part_acc, float* part_ml, int rows, int layer,
                                   int nsplit, int n_layers, int n_q_heads, int n_kv_heads, int head_dim,
                                   void* stream);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): the same decode attention with the split-KV partials
 * kept in a scratch array built into the library instead of caller-supplied part_acc / part_ml.
 * The call allocates nothing.  Limits: rows * n_q_heads * nsplit <= 16384 and head_dim <= 128
 * (the scratch is 16384 * 130 floats = 8.1 MiB per GPU, held until the process ends); beyond them
 * RLHF_EINVAL, with the reason available from rlhf_last_error(NULL).  All calls on one GPU share
 * that scratch: two such calls whose work overlaps in time on one GPU (different streams or
 * threads) race; calls ordered on one stream are safe.  Same kernels, same results as
 * rlhf_op_paged_decode_attention for the same nsplit. */
int rlhf_op_paged_decode_attention_noalloc(int dtype, const void* q, const void* pool, const int32_t* page_table,
                                           int pt_stride, const int32_t* row_sample, const int32_t* ctx_len,
                                           void* out, int rows, int layer, int nsplit, int n_layers,
                                           int n_q_heads, int n_kv_heads, int head_dim, void* stream);

/* Packed variable-length causal attention of the prefill / inference forward (Section 2.1):
 * float32 q [T, n_q_heads*head_dim], k, v [T, n_kv_heads*head_dim]; row r belongs to the
 * sequence that starts at row row_start[r] and is its row_pos[r]-th token.  out is IEEE half
 * (out_half != 0) or float32. */
int rlhf_op_varlen_attention(int out_half, const float* q, const float* k, const float* v,
                             const int32_t* row_start, const int32_t* row_pos, void* out, int rows,
                             int n_q_heads, int n_kv_heads, int head_dim, void* stream);

/* The same attention on the matrix units, as used for bf16 models: q, k, v, out IEEE half.
 * Queries are cut into tiles of 128 rows that do not straddle sequences: tile i covers rows
 * tile_start[i] + tile_q0[i] .. (at most 128, up to the end) of the sequence that starts at
 * row tile_start[i] and has tile_len[i] rows.  rows = rows of the packed buffers.
 * head_dim must be 64 or 128. */
int rlhf_op_flash_attention(const void* q, const void* k, const void* v, const int32_t* tile_start,
                            const int32_t* tile_q0, const int32_t* tile_len, void* out, int n_tiles,
                            int rows, int n_q_heads, int n_kv_heads, int head_dim, void* stream);

/* ---- attention that reads less of its cache: a sliding window with a few first tokens that stay visible (sinks), for packed passes
 * and for decode steps, and a KV cache held in 4 bits.
 *
 * The query at position i sees key j where j <= i and (j > i - window or j < sinks): the newest `window` tokens, itself among them,
 * and the first `sinks` ones.  window >= 1, sinks >= 0; a window of at least the longest context (INT32_MAX will do) is causal attention.
 * Scores are scaled by 1/sqrt(head_dim).  head_dim 64 or 128, n_q_heads a multiple of n_kv_heads (query head h reads KV head
 * h / (n_q_heads / n_kv_heads)).  act_dtype: RLHF_FP32, RLHF_BF16 or 2 = IEEE half, of all matrices of a call.  Scores, softmax and sums are
 * float.  In 16-bit calls a weight is rounded once for its product with V: in the packed form to the type (outputs are divided by the sum of the rounded
 * weights, and off by up to half a step of how far the visible values lie apart), over a cache of 4 bits, times the scale of a token's values, to half;
 * outputs are rounded once.  Matrices have rows of their own stride (ld_*, elements); addresses and strides are multiples of 16 bytes.  What a query does not see does not reach it, whatever it holds (infinities and NaN too).  At most 2^30 rows
 * (decode 2^24) and tiles, 2^16 heads and layers, fewer than 2^27 pages. */

/* Packed causal attention of a pass with a window: q, out [rows, n_q_heads*head_dim], k, v [rows, n_kv_heads*head_dim], e.g. columns
 * of one QKV buffer.  Tiles as in rlhf_op_flash_attention: tile i covers rows tile_start[i] + tile_q0[i] .. (at most 128, up to the
 * end) of the sequence that starts at row tile_start[i] and has tile_len[i] rows.  Rows of no tile are left as they are; a tile that
 * does not lie within the `rows` rows is skipped.  out must not overlap q, k or v; ld_k and ld_v are below 2^25. */
int rlhf_op_window_attention(int act_dtype, const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                             const int32_t* tile_start, const int32_t* tile_q0, const int32_t* tile_len, void* out, int64_t ld_out,
                             int n_tiles, int rows, int window, int sinks, int n_q_heads, int n_kv_heads, int head_dim,
                             void* stream);

/* Decode attention of one step with a window: row r holds one query at position ctx_len[r] - 1 of the sample whose row of page_table
 * [n_samples, pt_stride] is row_sample[r]; pool as in rlhf_op_paged_decode_attention, n_pages of them, in act_dtype.  Page-table entries of
 * pages without a visible token are not read: their pages may have been given back.  ctx_len[r] <= 0 gives a row of zeros.  A row
 * whose context, sample or visible pages lie outside page table or pool gives NaN; nothing is read out of bounds.  out overlaps neither q nor the pool.  How the
 * rows are launched goes by pt_stride and the window: with many rows of short contexts a table no wider than they need is up to 2.5 times as fast.
 * nsplit (1..64): into how many parts a row's visible pages are cut; rlhf_op_window_decode_nsplit gives the library's choice for a step
 * whose longest context has max_ctx tokens.  scratch: rlhf_op_window_decode_scratch_floats(rows, n_q_heads, head_dim, nsplit) floats,
 * 16-byte aligned (none for nsplit == 1: NULL will do); it belongs to one call at a time. */
int rlhf_op_window_decode_nsplit(int rows, int n_q_heads, int n_kv_heads, int max_ctx, int window, int sinks);
int64_t rlhf_op_window_decode_scratch_floats(int rows, int n_q_heads, int head_dim, int nsplit);
int rlhf_op_window_decode_attention(int act_dtype, const void* q, int64_t ld_q, const void* pool, int n_pages,
                                    const int32_t* page_table, int pt_stride, int n_samples, const int32_t* row_sample,
                                    const int32_t* ctx_len, void* out, int64_t ld_out, float* scratch, int rows, int layer, int nsplit,
                                    int window, int sinks, int n_layers, int n_q_heads, int n_kv_heads, int head_dim, void* stream);

/* A paged KV cache of 4 bits (4.5 with scales: 3.6 times the tokens of a half cache).  64 consecutive dims of one head's K or V of one token
 * share a scale and a center, IEEE half both: with lo and hi their least and greatest value
 *   s = half((hi - lo) * (1/15)),  c = half(lo + 8 s)     each operation and 1/15 rounded to float, then to half
 *   u = (x - c) / s rounded to the nearest whole number (half way: the even one) and clamped to -8 .. 7; 0 where s == 0
 * and the value held is c + s u.  A group with a NaN, or a magnitude above 65504, becomes NaN as a whole.
 * The outermost step of a group next to 65504 may lie beyond it: read or averaged in half it counts as 65504.
 * A page is 16 tokens, [page][layer][kv_head][18 * head_dim bytes], rlhf_op_kv4_page_bytes in all:
 *   8 head_dim bytes   K codes: 4 bits u + 8 of token t, dim d = 32 a + 8 b + i, in bits 4 (i % 2) of byte ((16 b + t) * head_dim / 32 + a) * 4 + i / 2
 *   8 head_dim bytes   V codes: token t = 4 b + i, dim d = 32 a + 16 e + g, in bits 4 e of byte ((16 b + g) * head_dim / 32 + a) * 4 + i
 *   head_dim bytes     (s, c) of K [head_dim / 64][16 tokens];  head_dim bytes   the same of V
 * (what a lane of the matrix units needs lies together).  Pools are 16-byte aligned. */
int64_t rlhf_op_kv4_page_bytes(int n_layers, int n_kv_heads, int head_dim);

/* Appends rows of k, v [rows, n_kv_heads*head_dim] to token slots kv_dst[r] = page*16 + offset of `layer`.  A negative slot, or one
 * beyond the pool's n_pages, is left out.  The slots of a call are distinct; k and v do not overlap the pool. */
int rlhf_op_kv4_append(int act_dtype, const void* k, int64_t ld_k, const void* v, int64_t ld_v, const int32_t* kv_dst, void* pool,
                       int n_pages, int rows, int layer, int n_layers, int n_kv_heads, int head_dim, void* stream);

/* Reads token slots back into rows of k, v, in act_dtype (to look at a cache, move it, or run a pass over it): c + s u rounded to float, which is exact unless
 * s is below 2^-9 of c, and from there to the type.  A negative slot gives a row of zeros, one beyond the pool a row of NaN.  k, v and the pool do not overlap. */
int rlhf_op_kv4_read(int act_dtype, const void* pool, int n_pages, const int32_t* kv_src, void* k, int64_t ld_k, void* v, int64_t ld_v,
                     int rows, int layer, int n_layers, int n_kv_heads, int head_dim, void* stream);

/* rlhf_op_window_decode_attention over such a cache; act_dtype is the type of q and out.  nsplit and scratch as there. */
int rlhf_op_kv4_decode_attention(int act_dtype, const void* q, int64_t ld_q, const void* pool, int n_pages,
                                 const int32_t* page_table, int pt_stride, int n_samples, const int32_t* row_sample,
                                 const int32_t* ctx_len, void* out, int64_t ld_out, float* scratch, int rows, int layer, int nsplit,
                                 int window, int sinks, int n_layers, int n_q_heads, int n_kv_heads, int head_dim, void* stream);

/* ---- row-wise kernels of the decoder block and of the heads.  act_dtype is the element type of
 * the 16-bit (or float) activations a kernel writes or reads: RLHF_FP32, RLHF_BF16, or 2 = IEEE
 * half.  "nsplit / sstride": a float input given as nsplit partial planes, plane s at x + s *
 * sstride elements (the split-K output of rlhf_op_gemm, summed in plane order by the consumer). */

/* RMSNorm of a decoder block (the reading of "LLaMA", Section 7: y = x * rsqrt(mean(x^2) + eps) * g,
 * statistics in float), fused with the residual add: v = h[src] + sum of the partial planes at
 * row src; xn[r] = norm(v) * g.  row_idx == NULL: src = r and v is written back to h (the residual
 * stream); otherwise src = row_idx[r] and h is left alone.  d a multiple of 8, at most 8192;
 * nsplit in [0, 16] (0: no planes). */
int rlhf_op_rmsnorm(int act_dtype, float* h, const float* part, int nsplit, int64_t sstride,
                    const int32_t* row_idx, const float* g, void* xn, int rows, int d, float eps, void* stream);

/* Rotary embedding and KV-cache append of decode steps and short passes: qkv [rows, (Hq + 2 Hkv)
 * * hd] float planes; query and key heads are rotated by pos[r] (pair (i, i + hd/2); table float32
 * [max position][hd/2][cos, sin]); q [rows, Hq*hd] and, if non-NULL, k, v [rows, Hkv*hd] are
 * written in act_dtype, and k, v also to token slot kv_dst[r] = page*16 + offset of `layer` in
 * the paged pool when pool != NULL (layout as in rlhf_op_paged_decode_attention). */
int rlhf_op_rope_kv(int act_dtype, const float* qkv, int nsplit, int64_t sstride, const int32_t* pos,
                    const int32_t* kv_dst, const float* table, void* q, void* k, void* v, void* pool,
                    int layer, int rows, int n_layers, int n_q_heads, int n_kv_heads, int head_dim,
                    void* stream);

/* SwiGLU of decode steps: gu [rows, 2*ffn] float planes (gate columns, then up columns);
 * act[r][c] = silu(gate) * up in act_dtype.  ffn a multiple of 8. */
int rlhf_op_swiglu(int act_dtype, const float* gu, int nsplit, int64_t sstride, void* act, int rows, int ffn,
                   void* stream);

/* Greedy choice of the generation stage (Section 2.1; lowest id on ties) over float logit planes
 * [rows, vocab]: token y = argmax (or forced[r] if forced != NULL and forced[r] >= 0) is written to
 * tokens[tok_dst[r]] (and picked[r] if non-NULL) and log_softmax(logits[r])[y] to lp[lp_dst[r]].
 * scratch: rlhf_op_pick_scratch_floats(rows) floats. */
int64_t rlhf_op_pick_scratch_floats(int rows);
int rlhf_op_pick(const float* logits, int nsplit, int64_t sstride, int rows, int vocab, const int32_t* forced,
                 int32_t* tokens, const int32_t* tok_dst, float* lp, const int32_t* lp_dst, int32_t* picked,
                 float* scratch, void* stream);

/* Log-prob of given tokens (inference stage, Section 2.1): out[out_dst[r]] =
 * log_softmax(logits[r])[tokens[target_idx[r]]]. */
int rlhf_op_gather_lp(const float* logits, int nsplit, int64_t sstride, int rows, int vocab,
                      const int32_t* tokens, const int32_t* target_idx, float* out, const int32_t* out_dst,
                      void* stream);

/* LM head of the inference stage fused with the log-softmax gather (Section 2.1: the Reference
 * and Actor log-probabilities of the generated tokens), as the stage runs it for bf16 models: for
 * row m of A [M, K] (IEEE half if act_half != 0, else bf16) and W_head bf16 [vocab, K],
 *   out[out_dst[m]] = log_softmax(W_head A[m])[tokens[target_idx[m]]]
 * without the [M, vocab] logits ever being written: the GEMM's epilogue keeps, per row and per 128
 * vocabulary columns, the maximum and the sum of exponentials, and a merge kernel finishes.
 * scratch: rlhf_op_lm_head_logprob_scratch_floats(M, vocab) floats.  K a multiple of 64. */
int64_t rlhf_op_lm_head_logprob_scratch_floats(int M, int vocab);
int rlhf_op_lm_head_logprob(int act_half, const void* A, const void* W_head, const int32_t* tokens,
                            const int32_t* target_idx, float* out, const int32_t* out_dst, float* scratch, int M,
                            int vocab, int K, void* stream);

/* Value / reward head (Section 2.1: the Critic evaluates each action, the Reward model scores the
 * sample): out[out_dst[r]] = <xn[r], w>, xn [rows, d] in act_dtype, w [d] in w_dtype (RLHF_FP32 or
 * RLHF_BF16).  Supported pairs: (fp32, fp32), (fp32, bf16), (half, bf16), (bf16, bf16). */
int rlhf_op_head_dot(int act_dtype, int w_dtype, const void* xn, const void* w, int rows, int d, float* out,
                     const int32_t* out_dst, void* stream);

/* ---- the Actor's update, as the training stage takes it up from the stage's results: the loss on the logits of a
 * forward pass with its gradient, the embedding lookup with its gradient, and the norm and clipping of all
 * gradients.  Columns of one buffer, side by side, do not overlap (row strides of the same number of bytes; of different ones, matrices
 * that interleave count as overlapping).  All of them can be captured into a graph; a scratch buffer belongs to one call at a time (calls
 * ordered on one stream may share it, graphs that may run at the same time may not). */

/* Clipped policy loss with a KL term towards the Reference, on logits, forward and gradient in one pass.  Row r of logits
 * [rows, vocab] (logit_dtype RLHF_FP32, RLHF_BF16 or 2 = IEEE half; row stride ld elements) is what predicts
 * y = tokens[r].  With l = log_softmax(logits[r])[y], A = adv[r], w = weight[r] (1 where weight == NULL),
 *   rho = exp(l - lp_old[r]),   policy_r = -min(rho * A, clamp(rho, 1 - clip_low, 1 + clip_high) * A),
 *   x = lp_ref[r] - l,          kl_r = exp(x) - x - 1    (0 where lp_ref == NULL, which needs kl_coef == 0),
 * the loss is the sum over the rows of w * (policy_r + kl_coef * kl_r): weights 1/n give the mean over n tokens.
 *   stats[4] = loss, sum of w * policy_r, sum of w * kl_r, sum of w over the rows whose gradient the clamp cut off
 *   lp[r]    = l
 *   dlogits[r] = grad_scale * d loss / d logits[r], in logit_dtype, row stride ld_grad; NULL: no gradient is taken.  It may be
 *              the logits themselves (same ld), else the two must not overlap.
 * Everything is float until the gradient is rounded once, the sums over rows double.  All sums have a fixed order (which columns meet
 * first goes by where a row lies between 16-byte boundaries): the same call gives the same bits.
 * A row with weight 0 or a negative token is left out: its logits and its other inputs, whatever they hold, are not used,
 * lp[r] = 0, its gradient is zero.  Logits of -inf have probability 0; where the token's own is, lp[r] = -inf, the ratio is 0 and the
 * KL towards lp_ref infinite, and with kl_coef > 0 the row's gradient is not finite.  A row whose result is not a number (all
 * logits -inf, a logit of +inf, NaN among its inputs, a token of vocab or more) makes lp[r], its gradient and stats NaN; lp[r] is a
 * number where it does not depend on what is none (adv; lp_old of -inf beside l = -inf), and so is the KL's sum (0 without lp_ref).
 * Columns of dlogits behind vocab are left as they are.  clip_low in [0, 1], clip_high >= 0, kl_coef >= 0.  rows and vocab at most
 * 2^30.
 * scratch: rlhf_op_policy_loss_scratch_floats(rows, vocab) floats. */
int64_t rlhf_op_policy_loss_scratch_floats(int rows, int vocab);
int rlhf_op_policy_loss(int logit_dtype, const void* logits, int64_t ld, const int32_t* tokens, const float* lp_old,
                        const float* lp_ref, const float* adv, const float* weight, float clip_low, float clip_high,
                        float kl_coef, float grad_scale, float* lp, float* stats, void* dlogits, int64_t ld_grad,
                        float* scratch, int rows, int vocab, void* stream);

/* Embedding lookup with scaling: out[r] = scale * table[tokens[r]], table [vocab, d] and out [rows, d] each in its own
 * type (RLHF_FP32, RLHF_BF16, 2 = IEEE half) and row stride; d at most 2^22, rows and vocab 2^30.  One rounding, to out's type.  A negative token gives
 * a row of zeros (padding), one of vocab or more a row of NaN. */
int rlhf_op_embed(int table_dtype, int out_dtype, const void* table, int64_t ld_table, const int32_t* tokens, float scale,
                  void* out, int64_t ld_out, int rows, int d, int vocab, void* stream);

/* Its gradient: dtable[v] = scale * (sum of dout[r] over the rows r with tokens[r] == v), every row of dtable written
 * (zeros where no row has the token); with accumulate != 0 that sum is added to dtable[v] instead and rows of other
 * tokens are left as they are.  The rows of a token are summed in float, in an order that depends on the tokens and sizes alone:
 * the same call gives the same bits.  Rows with tokens outside [0, vocab) count for nothing.  Types and strides as
 * above, dout in dout_dtype, dtable in table_dtype.  dout and dtable must not overlap.  Matrices of hundreds of GB, which no launch
 * covers, are refused before anything is written.
 * scratch: rlhf_op_embed_grad_scratch_bytes(rows, d, vocab) bytes, 16-byte aligned (none for few rows: NULL will do). */
int64_t rlhf_op_embed_grad_scratch_bytes(int rows, int d, int vocab);
int rlhf_op_embed_grad(int dout_dtype, int table_dtype, const void* dout, int64_t ld_dout, const int32_t* tokens, float scale,
                       int accumulate, void* dtable, int64_t ld_table, void* scratch, int rows, int d, int vocab,
                       void* stream);

/* The gradients of a model: n_tensors entries in HOST memory, read before a call returns.  src: n elements (fewer than
 * 2^40) of dtype (RLHF_FP32, RLHF_BF16, 2 = IEEE half), contiguous.  dst: where the clipped gradient goes, in the same type: src itself,
 * or memory that no entry's src or other dst shares; NULL where only the norm is taken.  Clipping refuses a list whose
 * dst are not so, the same gradient listed twice in place among them; the norm counts each entry, whatever it shares. */
typedef struct rlhf_tensor {
    const void* src;
    void* dst;
    int64_t n;
    int32_t dtype;
} rlhf_tensor;

/* norm[0] (device float) = the square root of the sum of the squares of all elements.  Sums are held in double: no square overflows or
 * vanishes.  scratch: rlhf_op_grad_norm_scratch_doubles(tensors, n_tensors) doubles. */
int64_t rlhf_op_grad_norm_scratch_doubles(const rlhf_tensor* tensors, int n_tensors);
int rlhf_op_grad_norm(const rlhf_tensor* tensors, int n_tensors, float* norm, double* scratch, void* stream);

/* dst = src * f with f = max_norm / norm[0] where norm[0] is finite and above max_norm, else 1: the gradients of a step
 * whose norm is not finite pass unchanged, for the caller to drop.  Between the two calls norm may be combined with that of other
 * ranks.  max_norm > 0. */
int rlhf_op_clip_grads(const rlhf_tensor* tensors, int n_tensors, const float* norm, float max_norm, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* RLHF_OPS_H */
