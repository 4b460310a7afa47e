// Internal declarations of the token-sequence operators (grat_sequence.h).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fastdiv.h"
#include "grat_sequence.h"

namespace grat {

// A tensor as the kernels address it.
struct SeqTensor {
    uint8_t* data;
    int64_t stride_b, stride_h, stride_n;   // elements
};

// What the kernels know of a batch of sequences.
struct SeqShape {
    int32_t batch, q_heads, kv_heads, share;   // share = q_heads / kv_heads
    int32_t n_q, n_k, q_group, block, n_groups, n_blocks;
    int32_t causal;
    const int32_t* k_len;
    const int32_t* q_pos;
};

// Valid keys of sequence b, and the position of its first query row.
__device__ __forceinline__ int seq_len(const SeqShape& s, int b) {
    return s.k_len ? min(max(s.k_len[b], 0), s.n_k) : s.n_k;
}
__device__ __forceinline__ int64_t seq_pos(const SeqShape& s, int b, int len) {
    return s.causal && s.q_pos ? (int64_t)s.q_pos[b] : (int64_t)len - s.n_q;
}
// Keys [0, seen) that the query in row i sees.
__device__ __forceinline__ int row_seen(const SeqShape& s, int len, int64_t pos, int i) {
    return s.causal ? (int)max((int64_t)0, min((int64_t)len, pos + i + 1)) : len;
}
// ... that some row of query group g sees: those of its last row.
__device__ __forceinline__ int group_seen(const SeqShape& s, int len, int64_t pos, int g) {
    return row_seen(s, len, pos, (int)min((int64_t)(g + 1) * s.q_group, (int64_t)s.n_q) - 1);
}

template <typename T> struct Vec16;   // 16 bytes of an element type
template <> struct Vec16<float> { static constexpr int n = 4; typedef __attribute__((ext_vector_type(4))) float type; };
template <> struct Vec16<__bf16> { static constexpr int n = 8; typedef __attribute__((ext_vector_type(8))) __bf16 type; };
template <> struct Vec16<_Float16> { static constexpr int n = 8; typedef __attribute__((ext_vector_type(8))) _Float16 type; };

struct RotaryParams {
    SeqTensor in[3], out[3];   // Q, K, V
    int32_t heads[3];          // 0: not there
    int32_t batch, n_tokens, items;   // items: pieces of two 16-byte vectors that a row consists of
    int32_t rot, interleaved, inverse, n_pos;
    int32_t axes, axis_end[3];        // pairs of the axes up to and with each
    const float* table;
    const int32_t* positions;
    int64_t positions_stride_b;
    const int32_t* start;
    int32_t n_cache;           // > 0: K and V go to the rows of a cache, start[b] + i
    int32_t head_chunk;        // heads per workgroup
    FastDiv fd_items, fd_tokens;
};
hipError_t launch_rotary(const RotaryParams& p, grat_dtype dtype, hipStream_t stream);
hipError_t launch_rotary_table(const grat_rotary_spec& spec, int32_t n_pos, int32_t axes, const int32_t* axis_pairs, float* d_table,
                               hipStream_t stream);

hipError_t launch_block_means(const SeqShape& s, const SeqTensor& K, grat_dtype dtype, int32_t head_dim, int32_t n_new, float* d_means,
                              hipStream_t stream);
int64_t block_scores_work(const SeqShape& s, int32_t head_dim);
hipError_t launch_block_scores(const SeqShape& s, const SeqTensor& Q, grat_dtype dtype, int32_t head_dim, const float* d_means, float scale,
                               float* d_scores, float* d_work, hipStream_t stream);
int64_t select_blocks_threads(const SeqShape& s, int32_t top);   // of a launch
hipError_t launch_select_blocks(const SeqShape& s, const float* d_scores, int32_t top, int32_t first, int32_t local, int32_t* d_count,
                                int32_t* d_index, hipStream_t stream);

}  // namespace grat
