/*
 * libgrat — token sequences: attention within a window.
 *
 * What the local layers of a language model need beside the attention over selected blocks of grat_sequence.h: every query attends the
 * newest keys up to its own position and a few first ones that stay visible.
 *
 *   grat_window_attention_fwd / _bwd    prompts, chunks of them and single tokens, and the gradient
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
 * them sees reaches all of them (0 * NaN).  Keys that none of them sees are never read.
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
 *              of the 64-key tiles that many rows see (those of the first keys; all of them where there are few)
 * Supported: as the forward call.  The softmax weights and the score gradients are rounded to the element type for the products; all sums
 * in fp32.  GRAT_F16: with the powers of two of grat_selected_attention_bwd.
 */
grat_status grat_window_attention_bwd(const grat_sequence* seq, const grat_tensor* dO, const grat_tensor* Q, const grat_tensor* K,
                                      const grat_tensor* V, const grat_tensor* O, const float* d_lse, const grat_tensor* dQ,
                                      const grat_tensor* dK, const grat_tensor* dV, float scale, int32_t window, int32_t sinks,
                                      void* d_work, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* GRAT_WINDOW_H */
