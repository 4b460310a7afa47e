/*
 * libgrat — token sequences: attention within a window, and over caches in 8 bits.
 *
 * What the local layers of a language model need beside the attention over selected blocks of grat_sequence.h: every query attends the
 * newest keys up to its own position and a few first ones that stay visible.  And what serves such a model, token by token or by trees of
 * drafted tokens, from caches that are read once a step.
 *
 *   grat_window_attention_fwd / _bwd    prompts, chunks of them and single tokens, and the gradient
 *   grat_cache_append / grat_cache_read the new tokens' K, turned, and V written into a cache, in 8 bits too; 8 bits read back
 *   grat_cache_attention_fwd            attention of the newest tokens over a cache
 *
 * Conventions, tensors and grat_sequence are those of grat_sequence.h; of grat_sequence q_group and block are not read.
 */
#ifndef GRAT_WINDOW_H
#define GRAT_WINDOW_H

#include "grat_sequence.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * O = softmax(scale * Q K^T over the keys that the row sees) V, row by row.
 *   The query in row i is at position p = d_q_pos[b] + i (d_q_pos NULL: k_len - n_q + i), the key in row j at j.
 *   causal: it sees the valid keys j <= p with p - j < window or j < sinks.
 *   not causal: the valid keys with |p - j| < window, and those with j < sinks.  (d_q_pos counts here too.)
 *   window     >= 1, or 0: no limit (sinks then says nothing)
 *   sinks      >= 0
 *   O          strides of its own; must not alias Q, K or V.  A row that sees no key gets 0.
 *   d_lse      [batch][q_heads][n_q] (fp32, or NULL): the natural logarithm of the row's sum of exp(scale q.k), -infinity for a row that
 *              sees no key
 *   d_work     scratch memory of grat_window_attention_work(seq, window, sinks, 0) bytes (NULL where that is 0), 16-byte aligned
 * Supported: GRAT_BF16, GRAT_F16; head_dim 64 or 128; stride_n < 2^24; every other stride as in grat.h; scale > 0; n_q, n_k < 2^30;
 * batch * kv_heads, q_heads <= 65535; batch * q_heads * n_q < 2^29; batch * kv_heads * n_k < 2^28; sinks <= 2^20 where that is below n_k.
 * Scores, reference maximum, sum and output accumulate in fp32; the weights are rounded to the element type (nearest-even) for the product
 * with V, their sum is not.  Rows are worked on together, 32 to 256 of neighbouring positions and of the heads that share a K/V head: a NaN or infinite V that one of
 * them sees can reach all of them (0 * NaN).  Keys that none of them sees are never read.
 */
int64_t grat_window_attention_work(const grat_sequence* seq, int32_t window, int32_t sinks, int32_t backward);
grat_status grat_window_attention_fwd(const grat_sequence* seq, const grat_tensor* Q, const grat_tensor* K, const grat_tensor* V,
                                      const grat_tensor* O, float* d_lse, float scale, int32_t window, int32_t sinks, void* d_work,
                                      void* hip_stream);

/*
 * The gradient of grat_window_attention_fwd: dQ, dK, dV for dO, with O and d_lse as the forward call wrote them.  Heads that share a K/V
 * head add up in its dK and dV.  Rows of dK and dV that no query sees, also those behind the valid keys, get 0.  Every output is written
 * once, nothing is added atomically: the same inputs give the same bits.
 *   d_work     grat_window_attention_work(seq, window, sinks, 1) bytes, 16-byte aligned: 8 bytes a query row, and 2 * 64 * head_dim * 4 for every part
 *              of the 64-key tiles that many rows see (those of the first keys; all of them where there are few), of which there are fewer than 2 560
 * Supported: as the forward call.  The softmax weights and the score gradients are rounded to the element type for the products; all sums
 * in fp32.  GRAT_F16: with the powers of two of grat_selected_attention_bwd.
 */
grat_status grat_window_attention_bwd(const grat_sequence* seq, const grat_tensor* dO, const grat_tensor* Q, const grat_tensor* K,
                                      const grat_tensor* V, const grat_tensor* O, const float* d_lse, const grat_tensor* dQ,
                                      const grat_tensor* dK, const grat_tensor* dV, float scale, int32_t window, int32_t sinks,
                                      void* d_work, void* hip_stream);

/*
 * Caches in 8 bits.  Of each row (one token of one K/V head) the head_dim numbers x are kept as e4m3 values (1 + 4 + 3 bits, largest 448, no
 * infinity), one byte each, rounded to nearest-even from x / s, beside s, one float a row: the least power of two with max |x| <= 448 s,
 * at least 2^-126, over the finite x; 1 for a row of zeros.  NaN and infinities become NaN.  A value is off by at most 2^-4 of itself, or 2^-10 s.
 * (GRAT_F16: 240 2^8 is the largest that a number below 65 520 becomes: 256 2^8 would be infinite when it is read back.)
 * grat_cache_read and grat_cache_attention_fwd take any finite scale.
 *   The cache's grat_tensor is in bytes (strides in elements of one byte, as its pointer multiples of 16); a scale's (b, h, n) at data +
 *   b*stride_b + h*stride_h + n*stride_n floats, strides >= 0 and below 2^46, stride_n >= 1 and below 2^24; scales that are written as in grat_sequence.h.
 */

/*
 * Serving: Q_out = Q turned by its positions; row i of sequence b of K (turned) and V (as it is) goes to row d_start[b] + i of K_cache and
 * V_cache, which have n_cache rows; rows outside [0, n_cache) are dropped.
 *   K_scale, V_scale   not NULL: caches in 8 bits.  Both NULL: caches of args->dtype.
 *   args   as grat_rotary_append takes them, but positions may be given too (a drafted token's row follows from its place in the tree's order,
 *          its position from its depth): axes and d_positions as for grat_rotary; NULL: row i is at position d_start[b] + i.  d_table NULL:
 *          nothing is turned; rot, axes, positions and n_pos are not read.
 *   Q, Q_out   both NULL: K and V alone; q_heads is not read.  Q_out may be Q.  Else no output may overlap an input.
 * Turned in fp32 and rounded once, to the cache's type.  Supported: as grat_rotary; head_dim 64 or 128; n_cache < 2^30; batch * n_tokens * (q_heads + 2 kv_heads) < 2^35.
 */
grat_status grat_cache_append(const grat_rotary_args* args, const grat_tensor* Q, const grat_tensor* Q_out, const grat_tensor* K,
                              const grat_tensor* V, const grat_tensor* K_cache, const grat_tensor* V_cache, const grat_tensor* K_scale,
                              const grat_tensor* V_scale, int32_t n_cache, void* hip_stream);

/*
 * out[b][h][n] = value * scale of the rows n < d_k_len[b] (NULL: all n_rows) of a cache in 8 bits, rounded once; rows behind them get 0 and are not
 * read.  `cache`, `scale` and `out` have `heads` heads and n_rows rows; out is of `dtype` (all three).
 * Supported: head_dim 64 or 128; strides and pointers of out as in grat.h; batch * heads <= 65535, n_rows < 2^30, batch * heads * n_rows < 2^28.
 */
grat_status grat_cache_read(grat_dtype dtype, int32_t batch, int32_t heads, int32_t n_rows, int32_t head_dim, const grat_tensor* cache,
                            const grat_tensor* scale, const int32_t* d_k_len, const grat_tensor* out, void* hip_stream);

/*
 * O of the newest tokens over a cache: those of sequence b have their K and V in the rows [k_len - n_q, k_len) of the caches, the tokens ahead of
 * them (the committed ones) in [0, k_len - n_q).  seq->causal and d_q_pos are not read.
 *   d_parent   NULL: a chain.  The token in row i is at position k_len - n_q + i and sees what grat_window_attention_fwd (causal) has it see.
 *              int32 [batch or 1][n_q], sequences parent_stride_b elements apart (0: shared): a tree.  Token t goes on from token parent[t] < t,
 *              or, where that is -1 (and any other number that is not in [0, t)), from the newest committed one.  Its position is k_len - n_q + its
 *              depth (0 for those that go on from a committed token).  It sees the committed tokens, its ancestors and itself, of these the ones at a
 *              position less than `window` ahead of its own, or below `sinks`.  (Tokens whose row k_len - n_q + t is negative have no key.)
 *   K_scale, V_scale   not NULL: caches in 8 bits.  Both NULL: caches of seq->dtype.
 *   window, sinks, O, d_lse, scale   as for grat_window_attention_fwd
 *   d_work     scratch memory of grat_cache_attention_work(seq, window, sinks, eight) bytes, eight: caches in 8 bits; 16-byte aligned
 * Supported: as grat_window_attention_fwd; trees: n_q <= 256.  For few rows (n_q * q_heads / kv_heads up to a few hundred); more are correct, but
 * every 128 or 256 rows (32 where their keys are few) read the cache anew.
 * Arithmetic as there.  8 bits, few rows a K/V head (up to 64; up to 256 where their keys are few): K's scale is taken to the scores in fp32, and the weights times
 * V's scales are rounded to bfloat16 (GRAT_F16: to the sum of two such numbers, 2^-17).  More rows: values times scales are rounded to seq->dtype first (scales that are powers of two leave bfloat16
 * nothing to round; half saturates at 65 504), and the weights as there.  A NaN or infinite V that one of a sequence's new tokens sees
 * can reach all of them (0 * NaN).
 */
int64_t grat_cache_attention_work(const grat_sequence* seq, int32_t window, int32_t sinks, int32_t eight);
grat_status grat_cache_attention_fwd(const grat_sequence* seq, const grat_tensor* Q, const grat_tensor* K_cache, const grat_tensor* V_cache,
                                     const grat_tensor* K_scale, const grat_tensor* V_scale, const grat_tensor* O, float* d_lse, float scale,
                                     int32_t window, int32_t sinks, const int32_t* d_parent, int64_t parent_stride_b, void* d_work,
                                     void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* GRAT_WINDOW_H */
