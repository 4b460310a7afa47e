/*
 * libgrat — token sequences: rotary positions, and attention over key blocks that a score selects.
 *
 * grat.h attends lists of key groups that follow from positions on a grid.  Here the lists follow from the data, as
 * long sequences of a language model need them: every group of queries attends the key blocks whose mean key it
 * scores highest, beside the first blocks and its own neighbourhood.  The steps, each an entry point of its own:
 *
 *   grat_rotary / grat_rotary_append    Q and K turned by their positions (a grid's axes included), appended to a cache
 *   grat_block_means                    mean key of every key block
 *   grat_block_scores                   score of every query group for every key block
 *   grat_select_blocks                  the lists
 *   grat_selected_attention_fwd / _bwd  attention over the lists, and its gradient
 *
 * Conventions of grat.h hold: plain C, device pointers owned by the caller, nothing allocated, nothing synchronised,
 * work enqueued on `hip_stream`, every check on the host ahead of the first launch, errors as return codes.  The
 * structs below and what their `data` members do not point to are HOST memory, read before the call returns.
 *
 * A batch of sequences
 *   Q has n_q rows and q_heads heads, K and V have n_k rows and kv_heads heads (a divisor of q_heads): query head h
 *   goes with K/V head h / (q_heads / kv_heads).
 *   d_k_len[b] keys of sequence b are valid (NULL: all n_k); values outside [0, n_k] are forced into it.  What lies
 *   behind them (a cache that is not full) is never read by these entry points.
 *   causal: the query in row i is at position p = d_q_pos[b] + i (d_q_pos NULL: k_len - n_q + i, the queries are the
 *   newest tokens) and sees the keys [0, p].  A row at a negative position sees nothing.  Not causal: every row sees
 *   every valid key.
 *   q_group consecutive rows, [g q_group, (g + 1) q_group), of all heads that share a K/V head are query group g and
 *   have one list; n_groups = ceil(n_q / q_group).  Key block j is the keys [j block, (j + 1) block), n_blocks =
 *   ceil(n_k / block).  The blocks that group g SEES are those with a key that one of its rows sees, blocks [0, s).
 *   A list is common to its group, and so is what it is made of: scores take the mean of all of the group's queries, and of all valid keys of a
 *   block.  With q_group > 1 the CHOICE of a causal row's blocks thus depends on up to q_group - 1 later tokens (the values that it attends
 *   do not), and single tokens that are served later cannot make the same choice.  With q_group = 1 and local >= 1 (grat_select_blocks) it
 *   depends on no later token: the one block whose mean reaches beyond the row is selected whatever its score.
 * Everywhere batch * kv_heads <= 65535, n_q, n_k < 2^30 (GRAT_ERR_UNSUPPORTED).
 */
#ifndef GRAT_SEQUENCE_H
#define GRAT_SEQUENCE_H

#include "grat.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element (b, h, n, c) at data + b*stride_b + h*stride_h + n*stride_n + c, strides in elements.  Inputs may repeat (stride_b, stride_h 0);
 * tensors that are written to may not (GRAT_ERR_BAD_DIMS where that axis has more than one element). */
typedef struct {
    void* data;
    int64_t stride_b, stride_h, stride_n;
} grat_tensor;

typedef struct {
    grat_dtype dtype;
    int32_t batch, q_heads, kv_heads, head_dim;
    int32_t n_q, n_k;          /* rows of the tensors */
    int32_t q_group, block;
    int32_t causal;
    const int32_t* d_k_len;    /* [batch] or NULL */
    const int32_t* d_q_pos;    /* [batch] or NULL; read only where causal */
} grat_sequence;

/*
 * Rotary positions.  Of a row's head_dim elements the first `rot` are turned as rot / 2 pairs, the others pass through:
 *     y[a] = c x[a] - s x[b],  y[b] = s x[a] + c x[b],   (c, s) = table[position][p] of pair p,
 * a = 2p, b = 2p + 1 (interleaved) or a = p, b = p + rot/2.  `inverse` takes -s for s: the gradient of the rotation.
 *
 *   axes, axis_pairs[axes]  pairs are dealt to axes in order, axis_pairs[k] to axis k (sum rot / 2); pair p takes the
 *                           table's row of its axis' position.  One axis for a sequence, 2 or 3 for a grid.
 *   d_positions             int32 [batch or 1][n_tokens][axes], batches positions_stride_b elements apart (0: shared);
 *                           or NULL (axes = 1): token i of sequence b is at d_start[b] + i (d_start NULL: i).
 *   d_table                 float [n_pos][rot / 2][2], e.g. from grat_rotary_table.  Positions outside [0, n_pos)
 *                           are forced into it.
 * Products and sums in fp32 (pairs of bf16 / half are exact there), rounded once.
 * Supported: all three dtypes; head_dim and rot multiples of 16, rot <= head_dim <= 1024; strides and pointers in 16
 * bytes as in grat.h; batch * n_tokens < 2^24 floor(w / head_dim), w = 2048 (fp32) or 4096 (16 bits), and < 2^30.
 */
typedef struct {
    grat_dtype dtype;
    int32_t batch, q_heads, kv_heads, head_dim, n_tokens;
    int32_t rot, interleaved, inverse;
    int32_t axes, axis_pairs[3];
    const float* d_table;
    int32_t n_pos;
    const int32_t* d_positions;
    int64_t positions_stride_b;
    const int32_t* d_start;    /* [batch] or NULL */
} grat_rotary_args;

/*
 * The table of cos and sin: row n, pair p of axis k (the i-th of its axis_pairs[k]) holds m cos(n f), m sin(n f),
 *     f0 = base ^ (-i / axis_pairs[k]),  f by `scaling`, worked out in fp64 and rounded once:
 *       GRAT_ROTARY_PLAIN   f = f0
 *       GRAT_ROTARY_LINEAR  f = f0 / factor                        (positions interpolated)
 *       GRAT_ROTARY_BASE    base * factor ^ (P / (P - 1)) for base (P = axis_pairs[k] > 1): the slowest pair is slowed by `factor`, the fastest not
 *       GRAT_ROTARY_RAMP    with t = trained f0 / 2 pi, the turns within the trained length, and
 *                           w = clamp((t - low) / (high - low), 0, 1):  f = f0 (w + (1 - w) / factor)
 *   m = magnitude.
 * factor > 0, magnitude > 0; RAMP also trained > 0 and low < high.  n_pos rows.
 */
typedef enum { GRAT_ROTARY_PLAIN = 0, GRAT_ROTARY_LINEAR = 1, GRAT_ROTARY_BASE = 2, GRAT_ROTARY_RAMP = 3 } grat_rotary_scaling;
typedef struct {
    grat_rotary_scaling scaling;
    double base, factor, magnitude, trained, low, high;
} grat_rotary_spec;
grat_status grat_rotary_table(const grat_rotary_spec* spec, int32_t n_pos, int32_t axes, const int32_t* axis_pairs,
                              float* d_table, void* hip_stream);

/*
 * Q_out = Q turned, K_out = K turned (K and K_out both NULL: Q alone; kv_heads is then not read).  An output may be its
 * input (same data and strides); any other overlap is undefined.
 */
grat_status grat_rotary(const grat_rotary_args* args, const grat_tensor* Q, const grat_tensor* Q_out, const grat_tensor* K,
                        const grat_tensor* K_out, void* hip_stream);

/*
 * Serving: as grat_rotary, but row i of sequence b of K (turned) and V (as it is) goes to row d_start[b] + i of
 * K_cache and V_cache, which have n_cache rows; rows outside [0, n_cache) are dropped.  d_start is required, one axis,
 * no d_positions, no inverse.  K, V have kv_heads heads.
 */
grat_status grat_rotary_append(const grat_rotary_args* args, const grat_tensor* Q, const grat_tensor* Q_out, const grat_tensor* K,
                               const grat_tensor* V, const grat_tensor* K_cache, const grat_tensor* V_cache, int32_t n_cache,
                               void* hip_stream);

/*
 * d_means[batch][kv_heads][n_blocks][head_dim] (fp32): the mean of the valid keys of every block, summed in fp32;
 * blocks without a valid key get 0.
 *   n_new = 0: all blocks.  n_new > 0: only the blocks that hold one of the last n_new valid keys of their sequence
 *   (means kept with a cache); the others are not touched.
 * Of `seq` dtype, batch, kv_heads, head_dim, n_k, block and d_k_len are read.
 * Supported: all three dtypes; head_dim 64 or 128; block a multiple of 32, <= 4096; n_blocks < 2^24.
 */
grat_status grat_block_means(const grat_sequence* seq, const grat_tensor* K, int32_t n_new, float* d_means, void* hip_stream);

/*
 * d_scores[batch][kv_heads][n_groups][n_blocks] (fp32): scale * (mean of the group's queries, over its rows and the heads
 * that share the K/V head) . (mean of the block's keys) for blocks that the group sees, -infinity for others.
 * Sums and products in fp32.
 *   d_means as grat_block_means writes them
 *   d_work  scratch memory of grat_block_scores_work(seq) bytes (NULL where that is 0), 16-byte aligned
 * Supported: as grat_block_means; n_groups <= 64 * 65535; scale any finite number.
 */
int64_t grat_block_scores_work(const grat_sequence* seq);
grat_status grat_block_scores(const grat_sequence* seq, const grat_tensor* Q, const float* d_means, float scale, float* d_scores,
                              void* d_work, void* hip_stream);

/*
 * The list of every query group: of the blocks that it sees the first `first`, the last `local`, and of the others those with
 * the highest scores, `top` blocks in all at most.  Equal scores: the lower block.  A score of NaN or -infinity is never
 * selected (the first and the last blocks are, whatever their scores).
 *   d_scores  as grat_block_scores writes them (or any others of that shape; those of blocks not seen do not count)
 *   d_count[batch][kv_heads][n_groups]       (out) length of the list, 0 for a group that sees nothing
 *   d_index[batch][kv_heads][n_groups][top]  (out) blocks in ascending order, then -1
 * top >= 1, first >= 0, local >= 0, first + local <= top (GRAT_ERR_BAD_DIMS); `local` of at least ceil(q_group / block) + 1
 * lets every row of a causal group see itself.
 * Supported: n_blocks <= 32768, top <= 8192, at most 2^26 - 4 lists, below 2^24 where n_blocks > 2048, below 2^23 where it is > 16384.  Of `seq` dtype and q_heads are not read, head_dim neither.
 */
grat_status grat_select_blocks(const grat_sequence* seq, const float* d_scores, int32_t top, int32_t first, int32_t local,
                               int32_t* d_count, int32_t* d_index, void* hip_stream);

/*
 * O = softmax(scale * Q K^T over the listed keys that the row sees) V, row by row.
 *   O          strides of its own; must not alias Q, K or V.  A row that sees no listed key gets 0.
 *   d_lse      [batch][q_heads][n_q] (fp32, or NULL): the natural logarithm of the row's sum of exp(scale q.k), -infinity
 *              for a row that sees no listed key
 *   d_count, d_index, max_blocks   lists as grat_select_blocks writes them (max_blocks = top).  Callers may make their
 *              own: any order, blocks of a list distinct.  Counts are forced into [0, max_blocks]; entries outside
 *              [0, n_blocks) are skipped.
 *   d_work     scratch memory of grat_selected_attention_work(seq, max_blocks, 0) bytes (NULL where that is 0), 16-byte
 *              aligned
 * Supported: GRAT_BF16, GRAT_F16; head_dim 64 or 128; block a multiple of 32; max_blocks * block <= 2^18; stride_n
 * < 2^24; every other stride as in grat.h.  scale > 0.  With L = batch * kv_heads * n_groups lists and R = q_group *
 * (q_heads / kv_heads) rows a list: L * max_blocks, L * R < 2^30, L * ceil(R / 32) < 2^23, batch * q_heads * n_q < 2^29,
 * batch * kv_heads * n_blocks < 2^24.
 * Scores, reference maximum, sum and output accumulate in fp32; the weights are rounded to the element type (nearest-even)
 * for the product with V, their sum is not.  A NaN or infinite V of a listed key that some row of a query group sees
 * reaches all rows of that group (0 * NaN); keys that the group does not list, or that none of its rows sees, are never read.
 */
int64_t grat_selected_attention_work(const grat_sequence* seq, int32_t max_blocks, int32_t backward);
grat_status grat_selected_attention_fwd(const grat_sequence* seq, const grat_tensor* Q, const grat_tensor* K, const grat_tensor* V,
                                        const grat_tensor* O, float* d_lse, float scale, const int32_t* d_count,
                                        const int32_t* d_index, int32_t max_blocks, void* d_work, void* hip_stream);

/*
 * The gradient of grat_selected_attention_fwd (the lists are given, not differentiated): dQ, dK, dV for dO, with O and
 * d_lse as the forward call wrote them.  Heads that share a K/V head add up in its dK and dV.  Rows of dK and dV that
 * no query attends, also those behind the valid keys, get 0.  Every output is written once, nothing is added
 * atomically: the same inputs give the same bits.
 *   d_work     grat_selected_attention_work(seq, max_blocks, 1) bytes, 16-byte aligned.  About four times the bytes of dK and dV (up to
 *              100 MB where that is less) for sums of parts, 8 bytes a query row, 4 an entry of a list, and a bit for
 *              every group and block of a K/V head, n_groups * n_blocks / 8 bytes: with a list per query (q_group = 1) that grows with
 *              the square of the length - 131 072 tokens in blocks of 64 keys: 34 MB a K/V head, 524 288 tokens 537 MB - and is
 *              cleared and read once a call
 * Supported: as the forward call; in addition the parts that the walk over keys is cut into, at most batch * kv_heads *
 * n_blocks + L * min(max_blocks, n_blocks) * R / 256, times the key tiles of 64 (or 32) of a block, stay below 2^23.
 * The softmax weights and the score gradients are rounded to the element type for the products; all sums in fp32.  GRAT_F16: both are
 * taken times powers of two that keep them within half's normal numbers - weights from 2^-26 on; score gradients by the size of
 * dO, of the row for dQ and of the K/V head's largest row for dK - so dO and V of any size lose nothing that half's results could hold.
 */
grat_status grat_selected_attention_bwd(const grat_sequence* seq, const grat_tensor* dO, const grat_tensor* Q, const grat_tensor* K,
                                        const grat_tensor* V, const grat_tensor* O, const float* d_lse, const grat_tensor* dQ,
                                        const grat_tensor* dK, const grat_tensor* dV, float scale, const int32_t* d_count,
                                        const int32_t* d_index, int32_t max_blocks, void* d_work, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* GRAT_SEQUENCE_H */
