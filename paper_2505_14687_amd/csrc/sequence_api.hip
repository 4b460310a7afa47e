// Host side of the token-sequence operators: argument validation and dispatch.  No allocation, no synchronisation.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "sequence_attn.h"
#include "sequence_checks.h"

namespace grat {

grat_status make_rotary(const grat_rotary_args* a, bool with_k, RotaryParams* out) {
    if (!a || !a->d_table) return GRAT_ERR_NULL;
    if (a->batch < 1 || a->q_heads < 1 || a->n_tokens < 1 || a->head_dim < 1 || a->rot < 1 || a->rot > a->head_dim || a->n_pos < 1)
        return GRAT_ERR_BAD_DIMS;
    if (with_k && a->kv_heads < 1) return GRAT_ERR_BAD_DIMS;
    if (a->axes < 1 || a->axes > 3) return GRAT_ERR_BAD_DIMS;
    int64_t pairs = 0;
    RotaryParams p{};
    for (int k = 0; k < 3; ++k) {
        if (k < a->axes) {
            if (a->axis_pairs[k] < 1) return GRAT_ERR_BAD_DIMS;
            pairs += a->axis_pairs[k];
        }
        p.axis_end[k] = (int32_t)(pairs < kMaxRows ? pairs : kMaxRows);
    }
    if (2 * pairs != a->rot) return GRAT_ERR_BAD_DIMS;
    if (a->axes > 1 && !a->d_positions) return GRAT_ERR_NULL;
    if (a->positions_stride_b < 0) return GRAT_ERR_BAD_DIMS;
    if (!known(a->dtype)) return GRAT_ERR_UNSUPPORTED;
    if (a->head_dim % 16 || a->rot % 16 || a->head_dim > 1024 || !aligned16(a->d_table)) return GRAT_ERR_UNSUPPORTED;
    // (a workgroup of 256 threads takes at least 256 / pieces tokens, rounded down)
    const int64_t tokens = (int64_t)a->batch * a->n_tokens, per = 256 / (a->head_dim / (is16(a->dtype) ? 16 : 8));
    if (tokens >= kMaxRows || (tokens + per - 1) / per * 256 >= kMaxThreads) return GRAT_ERR_UNSUPPORTED;
    if ((int64_t)a->q_heads + 2 * (int64_t)(with_k ? a->kv_heads : 0) > 65535) return GRAT_ERR_UNSUPPORTED;
    p.heads[0] = a->q_heads;
    p.heads[1] = with_k ? a->kv_heads : 0;
    p.batch = a->batch;
    p.n_tokens = a->n_tokens;
    p.items = a->head_dim;   // (the launcher divides by what a piece holds)
    p.rot = a->rot;
    p.interleaved = a->interleaved ? 1 : 0;
    p.inverse = a->inverse ? 1 : 0;
    p.n_pos = a->n_pos;
    p.axes = a->axes;
    p.table = a->d_table;
    p.positions = a->d_positions;
    p.positions_stride_b = a->positions_stride_b;
    p.start = a->d_start;
    *out = p;
    return GRAT_OK;
}

namespace {

// The parts of a grat_sequence that every operator on lists reads.
grat_status make_shape(const grat_sequence* s, SeqShape* out) {
    if (!s) return GRAT_ERR_NULL;
    if (s->batch < 1 || s->kv_heads < 1 || s->q_heads < 1 || s->n_q < 1 || s->n_k < 1 || s->q_group < 1 || s->block < 1) return GRAT_ERR_BAD_DIMS;
    if (s->q_heads % s->kv_heads) return GRAT_ERR_BAD_DIMS;
    if (s->block % 32 || s->block > 4096) return GRAT_ERR_UNSUPPORTED;
    if (s->n_q >= kMaxRows || s->n_k >= kMaxRows || (int64_t)s->batch * s->kv_heads > 65535 || s->q_heads > 65535) return GRAT_ERR_UNSUPPORTED;
    *out = SeqShape{s->batch, s->q_heads, s->kv_heads, s->q_heads / s->kv_heads, s->n_q, s->n_k,
                    s->q_group < s->n_q ? s->q_group : s->n_q, s->block, 0, 0, s->causal ? 1 : 0, s->d_k_len, s->d_q_pos};
    out->n_groups = (out->n_q + out->q_group - 1) / out->q_group;
    out->n_blocks = (out->n_k + out->block - 1) / out->block;
    return GRAT_OK;
}

// For the operators that do not read all of it.
grat_sequence with_heads(const grat_sequence& s) {
    grat_sequence t = s;
    t.q_heads = t.kv_heads;
    return t;
}

// ---- attention over lists --------------------------------------------------------------------
// Rows of a forward workgroup, of the `rows` of a group: one tile where they fit, else 256 if that makes four rounds of the chip and wastes no half tile, else 128
// (groups of 64 x 4 heads, 16 blocks of 64 keys, us in tiles of 256 and of 128: 512 groups x 8 heads 580 and 590, 100 x 8 109 and 109, 82 x 8 93 and 91, 47 x 8
// 60 and 55).
int fwd_tile_rows(const SeqShape& s, int head_dim, int64_t rows) {
    if (rows <= 16) return 16;
    if (rows <= 32) return 32;
    if (rows <= 64) return 64;
    const int64_t lists = (int64_t)s.batch * s.kv_heads * s.n_groups;
    if (head_dim == 128 && (rows % 256 == 0 || rows % 256 > 128) && lists * ((rows + 255) / 256) >= 1024) return 256;
    return 128;
}
int bwd_tile_rows(int64_t rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128; }
// Keys of a workgroup of the walk over keys.  (128, four waves that each take all rows of a tile, spill: blocks of 128 keys, 2 048 tokens 187 us against 154,
// 8 192 tokens of half at head_dim 64 440 against 420; blocks of 256 in groups of 128 2 310 against 2 395.)
int bwd_tile_keys(int block) { return block % 64 == 0 ? 64 : 32; }

// A checked call on lists, with everything that is decided about its launches.
struct SelPlan {
    SelParams p{};
    GradParams g{};
    int tile_rows = 0, tile_keys = 0;
    int64_t work = 0;   // bytes of scratch memory
};

// Takes a share of the scratch memory: returns its place, counted from the start.
int64_t take(SelPlan& plan, int64_t bytes) {
    const int64_t at = plan.work;
    plan.work = at + (bytes + 255) / 256 * 256;
    return at;
}

grat_status make_plan(const grat_sequence* seq, float scale, int32_t max_blocks, bool backward, uint8_t* work, SelPlan* out) {
    SelPlan plan;
    SelParams& p = plan.p;
    const grat_status st = make_shape(seq, &p.s);
    if (st != GRAT_OK) return st;
    const SeqShape& s = p.s;
    if (max_blocks < 1) return GRAT_ERR_BUFFER_TOO_SMALL;
    if (!(scale > 0.f) || !std::isfinite(scale)) return GRAT_ERR_BAD_DIMS;
    if (!is16(seq->dtype) || (seq->head_dim != 64 && seq->head_dim != 128)) return GRAT_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)s.q_group * s.share, lists = (int64_t)s.batch * s.kv_heads * s.n_groups;
    const int64_t blocks = (int64_t)s.batch * s.kv_heads * s.n_blocks, D = seq->head_dim;
    if ((int64_t)max_blocks * s.block > (1 << 18) || lists * max_blocks >= kMaxRows || blocks >= (1 << 24)) return GRAT_ERR_UNSUPPORTED;
    if ((int64_t)s.batch * s.q_heads * s.n_q >= kMaxRows / 2 || lists * rows >= kMaxRows || lists * ((rows + 31) / 32) >= (1 << 23))
        return GRAT_ERR_UNSUPPORTED;
    p.max_blocks = max_blocks;
    p.scale = scale;
    p.scale_log2 = (float)((double)scale * 1.4426950408889634);
    p.rows = (int32_t)rows;
    plan.tile_rows = backward ? bwd_tile_rows(rows) : fwd_tile_rows(s, (int)D, rows);
    p.row_tiles = (int32_t)((rows + plan.tile_rows - 1) / plan.tile_rows);
    const int64_t items = lists * p.row_tiles, units = (int64_t)std::min(max_blocks, s.n_blocks) * (s.block / kUnit);
    const int64_t shares = plan.tile_rows == 16 ? (units + 3) / 4 : (units + 1) / 2;   // steps of a workgroup
    // A forward launch that leaves compute units idle has lists shared by several workgroups, one a compute unit (two cost more than they hide, 64 tokens of
    // half over 2 048 keys 28.0 us against 26.9, and with many rows their parts' results: 1 000 queries, 20 blocks of 64 keys, 42 against 30).  A part is
    // two steps or more, and a list of fewer than 8 is not split: the launch that joins costs as much (one token, us, not split and split: 4 steps 8.6 and
    // 9.5, 8 steps 13.0 and 8.7, 16 steps 21.7 and 8.9; 64 queries, 16 steps 23.5, in 8 parts 15.4, in 16 parts 21.1).
    p.splits = backward || shares < 8 ? 1 : (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min(256 / items, shares / 2), 64));
    p.items = (int32_t)(items * p.splits);
    p.per_xcd = (p.items + 7) / 8;
    p.fd_splits = make_fastdiv((uint32_t)p.splits);
    p.fd_row_tiles = make_fastdiv((uint32_t)p.row_tiles);
    p.fd_groups = make_fastdiv((uint32_t)s.n_groups);
    p.fd_kv_heads = make_fastdiv((uint32_t)s.kv_heads);
    p.fd_q_group = make_fastdiv((uint32_t)s.q_group);
    p.fd_units = make_fastdiv((uint32_t)(s.block / kUnit));
    if (p.splits > 1) {
        const int64_t part_rows = (int64_t)p.items * plan.tile_rows;
        p.part_o = (float*)(work + take(plan, part_rows * D * 4));
        p.part_ml = (float*)(work + take(plan, part_rows * 8));
    }
    if (backward) {
        GradParams& g = plan.g;
        plan.tile_keys = bwd_tile_keys(s.block);
        g.blocks = (int32_t)blocks;
        g.words = (s.n_groups + 31) / 32;
        g.fd_rows = make_fastdiv((uint32_t)rows);
        g.fd_top = make_fastdiv((uint32_t)max_blocks);
        g.fd_tiles = make_fastdiv((uint32_t)(s.block / plan.tile_keys));
        // Parts of the rows that a block has on average (entries of all lists times the rows of a group, over all blocks), or of fewer where
        // that leaves compute units idle: a launch takes as long as its longest part.  (Against parts of the average length, 512 rows or more, a training
        // step: 201 queries with a list each 127 -> 60 us, 6 218 of them 2 024 -> 1 550.  More workgroups, 1 024 or 1 536 for 768: 2 626 tokens 262 -> 252 and
        // 260, 2 047 of half at head_dim 64 67.8 -> 69.3.)  A part is a workgroup a key tile of its block and holds whole blocks in fp32, so it is key tiles
        // that are counted: with parts counted, 16 384 tokens in blocks of 4 096 keys took 5 960 MiB of scratch memory, not 264, and a step of 1 024 queries on 8 192
        // keys 1 170 us, not 636; 2 048 tokens in blocks of 128 keys 155, not 136, of 256 keys 163, not 139.
        const int64_t entries = lists * std::min(max_blocks, s.n_blocks), all_rows = entries * rows;
        const int64_t part = std::max<int64_t>(256, (std::min(std::max<int64_t>(all_rows / blocks, 512), all_rows * (s.block / plan.tile_keys) / 768) + 63) / 64 * 64);
        g.part_rows = (int32_t)std::min<int64_t>(part, kMaxRows / 2);
        g.fd_part = make_fastdiv((uint32_t)g.part_rows);
        const int64_t most_parts = blocks + all_rows / g.part_rows, most_slots = 2 * (all_rows / g.part_rows) + 1;
        if (most_parts * (s.block / plan.tile_keys) >= (1 << 23)) return GRAT_ERR_UNSUPPORTED;
        g.most_parts = (int32_t)most_parts;
        g.most_joins = (int32_t)std::min<int64_t>(blocks, most_slots / 2);
        g.stats = (int64_t)s.batch * s.q_heads * s.n_q;
        g.delta = (float*)(work + take(plan, (g.stats + 1) * 4));
        g.lse2 = (float*)(work + take(plan, (g.stats + 1) * 4));
        g.bits = (uint32_t*)(work + take(plan, blocks * g.words * 4));
        g.counters = (int32_t*)(work + take(plan, 5 * 4));
        g.groups = (int32_t*)(work + take(plan, entries * 4));
        g.parts = (int4*)(work + take(plan, most_parts * 16));
        g.part_slot = (int32_t*)(work + take(plan, most_parts * 4));
        g.joins = (int4*)(work + take(plan, g.most_joins * 16));
        g.slots = (float*)(work + take(plan, most_slots * s.block * 2 * D * 4));
        g.heads = s.batch * s.kv_heads;
        if (seq->dtype == GRAT_F16) {
            g.head_runs = s.n_groups * p.row_tiles * std::max(plan.tile_rows / 32, 1);   // (below 2^30: rows of a head)
            g.row_bits = (int32_t*)(work + take(plan, (int64_t)g.heads * g.head_runs * 4));
            g.head_bits = (int32_t*)(work + take(plan, (int64_t)g.heads * 4));
        }
    }
    *out = plan;
    return GRAT_OK;
}

}  // namespace
}  // namespace grat

using namespace grat;

extern "C" grat_status grat_rotary_table(const grat_rotary_spec* spec, int32_t n_pos, int32_t axes, const int32_t* axis_pairs,
                                         float* d_table, void* hip_stream) {
    if (!spec || !axis_pairs || !d_table) return GRAT_ERR_NULL;
    if (n_pos < 1 || axes < 1 || axes > 3) return GRAT_ERR_BAD_DIMS;
    int64_t pairs = 0;
    for (int k = 0; k < axes; ++k) {
        if (axis_pairs[k] < 1) return GRAT_ERR_BAD_DIMS;
        pairs += axis_pairs[k];
    }
    if (spec->scaling != GRAT_ROTARY_PLAIN && spec->scaling != GRAT_ROTARY_LINEAR && spec->scaling != GRAT_ROTARY_BASE &&
        spec->scaling != GRAT_ROTARY_RAMP)
        return GRAT_ERR_BAD_PATTERN;
    auto positive = [](double v) { return v > 0.0 && std::isfinite(v); };
    if (!positive(spec->base) || !positive(spec->magnitude)) return GRAT_ERR_BAD_DIMS;
    if (spec->scaling != GRAT_ROTARY_PLAIN && !positive(spec->factor)) return GRAT_ERR_BAD_DIMS;
    if (spec->scaling == GRAT_ROTARY_RAMP && (!positive(spec->trained) || !(spec->low < spec->high) || !std::isfinite(spec->high - spec->low)))
        return GRAT_ERR_BAD_DIMS;
    if (pairs > 512 || (int64_t)n_pos * pairs >= kMaxRows || !aligned16(d_table)) return GRAT_ERR_UNSUPPORTED;
    return status_of(launch_rotary_table(*spec, n_pos, axes, axis_pairs, d_table, (hipStream_t)hip_stream));
}

extern "C" grat_status grat_rotary(const grat_rotary_args* args, const grat_tensor* Q, const grat_tensor* Q_out, const grat_tensor* K,
                                   const grat_tensor* K_out, void* hip_stream) {
    RotaryParams p;
    const bool with_k = K || K_out;
    grat_status st = make_rotary(args, with_k, &p);
    const grat_tensor* const tensors[4] = {Q, Q_out, K, K_out};
    for (int i = 0; st == GRAT_OK && i < (with_k ? 4 : 2); ++i)
        st = i % 2 ? check_output(tensors[i], args->dtype, args->head_dim, args->batch, p.heads[i / 2]) : check_tensor(tensors[i], args->dtype, args->head_dim);
    if (st != GRAT_OK) return st;
    p.in[0] = of(Q);
    p.out[0] = of(Q_out);
    if (with_k) {
        p.in[1] = of(K);
        p.out[1] = of(K_out);
    }
    return status_of(launch_rotary(p, args->dtype, (hipStream_t)hip_stream));
}

extern "C" grat_status grat_rotary_append(const grat_rotary_args* args, const grat_tensor* Q, const grat_tensor* Q_out, const grat_tensor* K,
                                          const grat_tensor* V, const grat_tensor* K_cache, const grat_tensor* V_cache, int32_t n_cache,
                                          void* hip_stream) {
    RotaryParams p;
    grat_status st = make_rotary(args, true, &p);
    const grat_tensor* const tensors[6] = {Q, Q_out, K, K_cache, V, V_cache};
    for (int i = 0; st == GRAT_OK && i < 6; ++i)
        st = i % 2 ? check_output(tensors[i], args->dtype, args->head_dim, args->batch, p.heads[i < 2 ? 0 : 1]) : check_tensor(tensors[i], args->dtype, args->head_dim);
    if (st != GRAT_OK) return st;
    if (!args->d_start) return GRAT_ERR_NULL;
    if (n_cache < 1 || args->axes != 1 || args->d_positions || args->inverse) return GRAT_ERR_BAD_DIMS;
    for (int t = 0; t < 3; ++t) {
        p.in[t] = of(tensors[2 * t]);
        p.out[t] = of(tensors[2 * t + 1]);
    }
    p.heads[2] = p.heads[1];
    p.n_cache = n_cache;
    return status_of(launch_rotary(p, args->dtype, (hipStream_t)hip_stream));
}

extern "C" grat_status grat_block_means(const grat_sequence* seq, const grat_tensor* K, int32_t n_new, float* d_means, void* hip_stream) {
    if (!seq || !d_means) return GRAT_ERR_NULL;
    grat_sequence q = with_heads(*seq);   // what is not read here
    q.n_q = q.q_group = 1;
    SeqShape s;
    grat_status st = make_shape(&q, &s);
    if (st != GRAT_OK) return st;
    if (n_new < 0) return GRAT_ERR_BAD_DIMS;
    if (!known(seq->dtype) || (seq->head_dim != 64 && seq->head_dim != 128)) return GRAT_ERR_UNSUPPORTED;
    if ((int64_t)s.n_blocks * 256 >= kMaxThreads) return GRAT_ERR_UNSUPPORTED;
    st = check_tensor(K, seq->dtype, seq->head_dim);
    if (st != GRAT_OK) return st;
    return status_of(launch_block_means(s, of(K), seq->dtype, seq->head_dim, n_new, d_means, (hipStream_t)hip_stream));
}

extern "C" int64_t grat_block_scores_work(const grat_sequence* seq) {
    SeqShape s;
    return make_shape(seq, &s) == GRAT_OK && seq->head_dim > 0 ? block_scores_work(s, seq->head_dim) : 0;
}

extern "C" grat_status grat_block_scores(const grat_sequence* seq, const grat_tensor* Q, const float* d_means, float scale, float* d_scores,
                                         void* d_work, void* hip_stream) {
    if (!d_means || !d_scores) return GRAT_ERR_NULL;
    SeqShape s;
    grat_status st = make_shape(seq, &s);
    if (st != GRAT_OK) return st;
    if (!std::isfinite(scale)) return GRAT_ERR_BAD_DIMS;
    if (!known(seq->dtype) || (seq->head_dim != 64 && seq->head_dim != 128)) return GRAT_ERR_UNSUPPORTED;
    if ((int64_t)s.n_groups > 65535 * (int64_t)64 || !aligned16(d_means) || !aligned16(d_work)) return GRAT_ERR_UNSUPPORTED;
    st = check_tensor(Q, seq->dtype, seq->head_dim);
    if (st != GRAT_OK) return st;
    if (!d_work && block_scores_work(s, seq->head_dim) > 0) return GRAT_ERR_NULL;
    return status_of(launch_block_scores(s, of(Q), seq->dtype, seq->head_dim, d_means, scale, d_scores, (float*)d_work, (hipStream_t)hip_stream));
}

extern "C" grat_status grat_select_blocks(const grat_sequence* seq, const float* d_scores, int32_t top, int32_t first, int32_t local,
                                          int32_t* d_count, int32_t* d_index, void* hip_stream) {
    if (!seq || !d_scores || !d_count || !d_index) return GRAT_ERR_NULL;
    const grat_sequence q = with_heads(*seq);
    SeqShape s;
    const grat_status st = make_shape(&q, &s);
    if (st != GRAT_OK) return st;
    if (top < 1 || first < 0 || local < 0 || (int64_t)first + local > top) return GRAT_ERR_BAD_DIMS;
    if (s.n_blocks > 32768 || top > 8192 || (int64_t)s.batch * s.kv_heads * s.n_groups >= (1 << 26)) return GRAT_ERR_UNSUPPORTED;
    if (select_blocks_threads(s, top) >= kMaxThreads) return GRAT_ERR_UNSUPPORTED;
    return status_of(launch_select_blocks(s, d_scores, top, first, local, d_count, d_index, (hipStream_t)hip_stream));
}

extern "C" int64_t grat_selected_attention_work(const grat_sequence* seq, int32_t max_blocks, int32_t backward) {
    SelPlan plan;
    return make_plan(seq, 1.f, max_blocks, backward != 0, nullptr, &plan) == GRAT_OK ? plan.work : 0;
}

extern "C" grat_status grat_selected_attention_fwd(const grat_sequence* seq, const grat_tensor* Q, const grat_tensor* K, const grat_tensor* V,
                                                   const grat_tensor* O, float* d_lse, float scale, const int32_t* d_count,
                                                   const int32_t* d_index, int32_t max_blocks, void* d_work, void* hip_stream) {
    if (!d_count || !d_index) return GRAT_ERR_NULL;
    SelPlan plan;
    grat_status st = make_plan(seq, scale, max_blocks, false, (uint8_t*)d_work, &plan);
    for (const grat_tensor* t : {Q, K, V})
        if (st == GRAT_OK) st = check_tensor(t, seq->dtype, seq->head_dim);
    if (st == GRAT_OK) st = check_output(O, seq->dtype, seq->head_dim, seq->batch, seq->q_heads);
    if (st != GRAT_OK) return st;
    if (plan.work > 0 && !d_work) return GRAT_ERR_NULL;
    if (!aligned16(d_work)) return GRAT_ERR_UNSUPPORTED;
    SelParams& p = plan.p;
    p.Q = of(Q);
    p.K = of(K);
    p.V = of(V);
    p.O = of(O);
    p.lse = d_lse;
    p.count = d_count;
    p.index = d_index;
    const bool f16 = seq->dtype == GRAT_F16, wide = seq->head_dim == 128;
    const auto launch = f16 ? (wide ? launch_selected_fwd_f16_d128 : launch_selected_fwd_f16_d64)
                            : (wide ? launch_selected_fwd_bf16_d128 : launch_selected_fwd_bf16_d64);
    return status_of(launch(p, plan.tile_rows, (hipStream_t)hip_stream));
}

extern "C" grat_status grat_selected_attention_bwd(const grat_sequence* seq, const grat_tensor* dO, const grat_tensor* Q, const grat_tensor* K,
                                                   const grat_tensor* V, const grat_tensor* O, const float* d_lse, const grat_tensor* dQ,
                                                   const grat_tensor* dK, const grat_tensor* dV, float scale, const int32_t* d_count,
                                                   const int32_t* d_index, int32_t max_blocks, void* d_work, void* hip_stream) {
    if (!d_lse || !d_count || !d_index) return GRAT_ERR_NULL;
    SelPlan plan;
    grat_status st = make_plan(seq, scale, max_blocks, true, (uint8_t*)d_work, &plan);
    for (const grat_tensor* t : {dO, Q, K, V, O})
        if (st == GRAT_OK) st = check_tensor(t, seq->dtype, seq->head_dim);
    if (st == GRAT_OK) st = check_output(dQ, seq->dtype, seq->head_dim, seq->batch, seq->q_heads);
    for (const grat_tensor* t : {dK, dV})
        if (st == GRAT_OK) st = check_output(t, seq->dtype, seq->head_dim, seq->batch, seq->kv_heads);
    if (st != GRAT_OK) return st;
    if (!d_work) return GRAT_ERR_NULL;
    if (!aligned16(d_work)) return GRAT_ERR_UNSUPPORTED;
    SelParams& p = plan.p;
    p.Q = of(Q);
    p.K = of(K);
    p.V = of(V);
    p.O = of(O);
    p.lse = const_cast<float*>(d_lse);
    p.count = d_count;
    p.index = d_index;
    GradParams& g = plan.g;
    g.dO = of(dO);
    g.dQ = of(dQ);
    g.dK = of(dK);
    g.dV = of(dV);
    const bool f16 = seq->dtype == GRAT_F16, wide = seq->head_dim == 128;
    const auto launch = f16 ? (wide ? launch_selected_bwd_f16_d128 : launch_selected_bwd_f16_d64)
                            : (wide ? launch_selected_bwd_bf16_d128 : launch_selected_bwd_bf16_d64);
    return status_of(launch(p, g, plan.tile_rows, plan.tile_keys, (hipStream_t)hip_stream));
}
