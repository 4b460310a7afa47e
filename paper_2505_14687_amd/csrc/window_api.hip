// Host side of attention within a window and over caches: argument validation and dispatch.  No allocation, no synchronisation.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "cache_attn.h"
#include "cache_rows.h"
#include "grat_window.h"
#include "sequence_checks.h"

namespace grat {
namespace {

constexpr int64_t kMostFirst = (int64_t)1 << 20;   // first keys that stay visible

// What every operator here reads of a grat_sequence.
grat_status make_shape(const grat_sequence* s, SeqShape* out) {
    if (!s) return GRAT_ERR_NULL;
    if (s->batch < 1 || s->kv_heads < 1 || s->q_heads < 1 || s->n_q < 1 || s->n_k < 1 || s->q_heads % s->kv_heads) return GRAT_ERR_BAD_DIMS;
    if (!is16(s->dtype) || (s->head_dim != 64 && s->head_dim != 128)) return GRAT_ERR_UNSUPPORTED;
    if (s->n_q >= kMaxRows || s->n_k >= kMaxRows || (int64_t)s->batch * s->kv_heads > 65535 || s->q_heads > 65535) return GRAT_ERR_UNSUPPORTED;
    if ((int64_t)s->batch * s->q_heads * s->n_q >= kMaxRows / 2 || (int64_t)s->batch * s->kv_heads * s->n_k >= kMaxRows / 4) return GRAT_ERR_UNSUPPORTED;
    *out = SeqShape{s->batch, s->q_heads, s->kv_heads, s->q_heads / s->kv_heads, s->n_q, s->n_k, s->n_q, kUnit, 1, 0,
                    s->causal ? 1 : 0, s->d_k_len, s->d_q_pos};
    return GRAT_OK;
}

grat_status set_window(SelParams& p, float scale, int32_t window, int32_t sinks) {
    if (window < 0 || sinks < 0 || !(scale > 0.f) || !std::isfinite(scale)) return GRAT_ERR_BAD_DIMS;
    const bool all = window == 0 || sinks >= p.s.n_k;
    p.window = all ? kNoWindow : window;
    p.sinks = all ? 0 : sinks;
    if (p.sinks > kMostFirst) return GRAT_ERR_UNSUPPORTED;
    p.scale = scale;
    p.scale_log2 = (float)((double)scale * 1.4426950408889634);
    return GRAT_OK;
}

// Keys that `queries` neighbouring queries may see beside the first ones, and the other way round.
int64_t reach(const SelParams& p, int64_t queries, int64_t most) {
    return std::min(most, (p.s.causal ? 1 : 2) * (p.window - 1) + queries);
}

// Keys that they see, with the first ones.
int64_t seen(const SelParams& p, int64_t queries) { return std::min<int64_t>(p.s.n_k, reach(p, queries, p.s.n_k) + p.sinks); }

// Groups of neighbouring queries of at most `group_rows` rows (where one query has no more), in tiles.
void set_tiles(SelParams& p, int group_rows, int tile_rows) {
    SeqShape& s = p.s;
    s.q_group = std::max(1, std::min(s.n_q, group_rows / s.share));
    s.n_groups = (s.n_q + s.q_group - 1) / s.q_group;
    p.rows = s.q_group * s.share;
    p.row_tiles = (p.rows + tile_rows - 1) / tile_rows;
    p.fd_row_tiles = make_fastdiv((uint32_t)p.row_tiles);
    p.fd_groups = make_fastdiv((uint32_t)s.n_groups);
    p.fd_kv_heads = make_fastdiv((uint32_t)s.kv_heads);
    p.fd_q_group = make_fastdiv((uint32_t)s.q_group);
    p.fd_units = make_fastdiv(1);
}
void set_items(SelParams& p, int64_t items, int splits) {
    p.splits = splits;
    p.items = (int32_t)(items * splits);
    p.per_xcd = (p.items + 7) / 8;
    p.fd_splits = make_fastdiv((uint32_t)splits);
}

// ---- forward -------------------------------------------------------------------------------------
struct ForwardPlan {
    SelParams p{};
    int tile_rows = 0;
    int64_t work = 0;
};

// Prompts that tiles of 128 rows would spread over the chip about once: tiles of 64, whose two teams take half of the keys each.  us with tiles
// of 128 and of 64, forward of 8 heads on as many (16 tiles of 128 rows for 2 048 tokens of one):
//   window 129, 2 047 tokens of 1 to 4 sequences   head_dim 64   11.0 8.5   11.7 10.2   14.6 11.8   14.9 13.4   (training step 47.0 38.5   52.5 47.3   67.0 58.8   71.8 74.6)
//                                                  head_dim 128  13.3 11.7   14.0 14.1   18.4 21.5   19.3 24.9   (62.2 53.8   74.8 71.4   92.4 99.0   108 123)
// The gradient's dQ gains at any number of keys (2 048 queries of 1 and 2 sequences behind 6 144 tokens, gradient, window 1 000, 3 000, none: head_dim 64 58.5 51.3   112.5 94.4
// 247.5 201.4 and 70.2 66.8   142.8 134.1   308 285; head_dim 128 81.5 75.6   156.8 141.8   336.6 298.3 and 107.4 108.8   220.5 222.0   463 464).
int64_t tiles_of_128(const SelParams& p) { return (int64_t)p.s.batch * p.s.kv_heads * (((int64_t)p.s.n_q * p.s.share + 127) / 128); }
bool few_tiles(const SelParams& p, int head_dim) { return tiles_of_128(p) <= (head_dim == 64 ? 384 : 256); }

// ... forward, while rows see few keys: the same queries, windows
//   1 500, 1 800, 2 100          head_dim 128, 1 sequence   34.2 30.6   36.7 35.2   38.7 38.9     2   37.5 38.9   42.9 45.2   47.3 50.6   (1 300, 1 400: 32.8 32.7   33.7 33.8)
//   2 500, 2 900, 3 200, 6 000   head_dim 64, 1 sequence    32.8 31.9   35.5 35.6   37.1 38.0   56.0 65.5     2   43.6 38.8   48.7 43.3   51.9 46.4   90.6 80.8     3   56.3 51.4   63.1 57.9
//   67.3 62.1   117 110
bool few_tiles_forward(const SelParams& p, int head_dim) {
    const bool half_chip = tiles_of_128(p) <= 128;
    const int64_t most = head_dim == 128 ? (half_chip ? 2048 : 1536) : half_chip ? 2816 : p.s.n_k;
    return few_tiles(p, head_dim) && seen(p, 128) <= most;
}

// Rows of a workgroup, of the `rows` of all heads that share a K/V head.
// 16 and 32: the kernel of few rows, whose tiles each fetch all of the head's keys; so rows that see much the same keys, few of them (64; 96 in 8 bits) or with few keys.  us
// in tiles of 64 to 256 rows and of 32, 32 heads on 8: 64 rows over 4 000 keys 16 bits 17.1 15.4, 16 sequences over 8 192 112 108, head_dim 64 13.3 11.9 and 65.8 56.8;
// 96 rows of 16 sequences over 4 096 8 bits 65.3 56.8, 16 bits 64.1 80.6; 256 rows over 4 096 8 bits 29.2 21.8, 16 bits 27.9 21.7, head_dim 64 18.5 15.5; of 4 sequences
// 35.8 38.3, 35.5 35.3, 25.6 25.6; 128 rows of 4 sequences over 8 192, 16 bits, 40.1 48.5.  256 rows of 4 sequences, window 256 and 1 024, 4 096, 16 384 first keys, 16 bits 25.2 22.9   35.0
// 37.1   82.1 124.6, 8 bits 26.9 23.1   37.2 39.6   82.2 108.4; window 64 and 1 024 first keys 24.2 21.6.  head_dim 64 goes further: 256 rows of 4 sequences over 16 384 and
// 65 536 67.6 65.6   238 260, in 8 bits, whatever the number of keys, 78.8 65.7   285 233; of 16 sequences over 4 096 and 16 384 63.9 55.3   234 253, 8 bits 74.1 64.6   281 230.
// 256 if that is one tile, or makes four rounds of the chip and its walk is long, else 128, of which two share a compute unit and cover each other's start and end (32 768
// tokens, 32 heads on 8, us in tiles of 256 and of 128: window 64 204 161, 256 288 253, 512 398 371, 1 024 621 601, 2 048 1 056 1 051, 4 096 1 855 1 890; window 64 and 2 600, 4 096,
// 8 192 first keys 1 265 1 302, 1 830 1 906, 3 360 3 466).
int fwd_tile_rows(const SelParams& p, int head_dim, bool eight) {
    const SeqShape& s = p.s;
    const int64_t rows = (int64_t)s.n_q * s.share, tiles = (rows + 31) / 32, heads = (int64_t)s.batch * s.kv_heads;
    const bool alike = (p.window + p.sinks) / 4 >= s.n_q;
    const int64_t keys = heads * tiles * seen(p, s.n_q);   // that tiles of 32 rows fetch
    const bool few_keys = head_dim == 64 ? eight || keys <= 1 << 22 : keys <= 1 << 19;
    if (rows <= 32) return rows <= 16 ? 16 : 32;
    if ((rows <= 64 && eight) || (alike && (rows <= (eight ? 96 : 64) || (rows <= 256 && few_keys)))) return 32;
    if (rows <= 64) return 64;
    if (head_dim == 128 && rows > 128 && (rows <= 256 || (heads * ((rows + 255) / 256) >= 1024 && seen(p, 64) > 2560))) return 256;
    if (!eight && few_tiles_forward(p, head_dim)) return 64;
    return 128;
}

grat_status make_forward(const grat_sequence* seq, float scale, int32_t window, int32_t sinks, bool eight, bool tree, void* work, ForwardPlan* out) {
    ForwardPlan plan;
    SelParams& p = plan.p;
    const SeqShape& s = p.s;
    grat_status st = make_shape(seq, &p.s);
    if (st == GRAT_OK) st = set_window(p, scale, window, sinks);
    if (st != GRAT_OK) return st;
    if (tree && s.n_q > kMostDrafted) return GRAT_ERR_UNSUPPORTED;
    plan.tile_rows = fwd_tile_rows(p, seq->head_dim, eight);
    const bool few = plan.tile_rows <= 32;   // four waves that share the keys (cache_attn.h)
    set_tiles(p, tree || few ? s.n_q * s.share : plan.tile_rows, plan.tile_rows);   // (these are one group)
    const int64_t items = (int64_t)s.batch * s.kv_heads * s.n_groups * p.row_tiles;
    if (items >= (1 << 23)) return GRAT_ERR_UNSUPPORTED;
    const int keys = few ? 4 * cache_keys(eight, seq->head_dim, tree) : 64;   // of a workgroup's step
    const int64_t steps = (reach(p, s.q_group, s.n_k) + keys - 1) / keys + (p.sinks + keys - 1) / keys;
    // A launch that leaves compute units idle has keys shared by several workgroups, up to one a compute unit (two tiles of few rows: two).  Few rows: parts of one or two steps, about 16 of them,
    // or of more where that fills the chip; 4 steps or more (one token on 8 heads, us, in parts of 2 steps and by this rule: 17 steps 11.9 and 10.8, 8 steps
    // 10.3 and 9.3, 32 steps 12.3 both, in parts of one 13.4; 2 steps 7.5 in one part).  Many rows, whose parts' results weigh as much as their keys do:
    // 2 steps or more up to 8 parts, 4 or more beyond (64 rows over 4 000 keys in 31 and in 15 parts 19.0 and 16.9, 96 rows 21.1 and 19.1; 120 rows over 1 015 in 8 and 4 12.7 and 13.7).
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>((few && p.row_tiles > 1 ? 512 : 256) / items, 64));
    const int64_t per = std::max((steps + most - 1) / most, std::min<int64_t>(std::max<int64_t>((steps + 8) / 16, 1), 2));
    set_items(p, items, few ? (steps < 4 ? 1 : (int)std::min<int64_t>((steps + per - 1) / per, most)) : steps < 8 ? 1 : (int)std::min<int64_t>(steps < 32 ? std::min<int64_t>(steps / 2, 8) : steps / 4, most));
    if (p.splits > 1 && s.k_len && s.batch <= 64 && s.n_groups == 1) {   // lengths of their own: parts of about equal length
        p.slots = s.batch * p.splits;
        p.part_keys = few ? keys / 4 : kUnit;
        p.part_step = few ? 4 : 2;
        p.fd_splits = make_fastdiv((uint32_t)p.slots);
    }
    Scratch scratch{(uint8_t*)work};
    if (p.splits > 1) {
        p.part_o = scratch.take<float>((int64_t)p.items * plan.tile_rows * seq->head_dim);
        p.part_ml = scratch.take<float>((int64_t)p.items * plan.tile_rows * 2);
    }
    plan.work = scratch.bytes;
    *out = plan;
    return GRAT_OK;
}

grat_status launch_forward(const ForwardPlan& plan, const grat_sequence* seq, bool eight, void* hip_stream) {
    const bool f16 = seq->dtype == GRAT_F16, wide = seq->head_dim == 128;
    const auto launch = f16 ? (wide ? launch_cache_attention_f16_d128 : launch_cache_attention_f16_d64)
                            : (wide ? launch_cache_attention_bf16_d128 : launch_cache_attention_bf16_d64);
    return status_of(launch(plan.p, eight, plan.tile_rows, (hipStream_t)hip_stream));
}

// A cache's queries are the newest tokens.
grat_sequence newest(const grat_sequence& s) {
    grat_sequence t = s;
    t.causal = 1;
    t.d_q_pos = nullptr;
    return t;
}

// ---- gradient ------------------------------------------------------------------------------------
struct GradPlan {
    SelParams p{};
    GradParams g{};
    int tile_rows = 0;
    int64_t work = 0;
};

int bwd_tile_rows(const SelParams& p, int head_dim) {
    const SeqShape& s = p.s;
    const int64_t rows = (int64_t)s.n_q * s.share;
    return rows <= 32 ? 32 : rows <= 64 || few_tiles(p, head_dim) ? 64 : 128;
}

grat_status make_gradient(const grat_sequence* seq, float scale, int32_t window, int32_t sinks, void* work, GradPlan* out) {
    GradPlan plan;
    SelParams& p = plan.p;
    GradParams& g = plan.g;
    WindowGradParams& w = g.window;
    const SeqShape& s = p.s;
    grat_status st = make_shape(seq, &p.s);
    if (st == GRAT_OK) st = set_window(p, scale, window, sinks);
    if (st != GRAT_OK) return st;
    const int64_t D = seq->head_dim, heads = (int64_t)s.batch * s.kv_heads;
    plan.tile_rows = bwd_tile_rows(p, (int)D);
    set_tiles(p, plan.tile_rows, plan.tile_rows);
    const int64_t items = heads * s.n_groups * p.row_tiles;
    if (items >= (1 << 23)) return GRAT_ERR_UNSUPPORTED;
    set_items(p, items, 1);
    // Parts of the rows that see a key tile: a window's, or fewer where that leaves compute units idle, which take two workgroups each (2 048 tokens, 32 heads on 8, window
    // 512, training step 137 us in 1.5 rounds of parts, 124 in one).  The rows that see first keys are cut as the others, or into 32 where four rounds cover longer parts
    // (16 384 tokens, window 128 545 -> 523; on one K/V head 172 -> 227), and into no more than make two rounds of all first tiles: a part's sums are twice what dK and dV take of its
    // tile, in scratch memory.  Gradient of 16 384 tokens, 32 heads on 8, window 128, first keys 1 024 and 4 096: cut by their length alone 1 350 us and 273 MB, 4 171 and
    // 1 078; for one round 1 166 and 38, 3 311 and 4; two 1 186 and 71, 3 289 and 71; four 1 258 and 138, 3 346 and 138.  8 heads on one, 4 096: 1 280, 1 371, 1 178, 1 115 us.
    w.tiles = (s.n_k + 63) / 64;
    w.first_tiles = (p.sinks + 63) / 64;
    const int64_t near = reach(p, 64, s.n_q) * s.share, all = (int64_t)s.n_q * s.share;
    const int64_t part = std::max<int64_t>(256, (std::min(std::max<int64_t>(near, 512), heads * w.tiles * near / 512) + 63) / 64 * 64);
    const int64_t even = std::max(heads * w.tiles >= 2048 ? all / 32 : 0, std::min(all, heads * w.first_tiles * all / 1024));
    const int64_t first_part = std::max(part, (even + 63) / 64 * 64);
    w.near_parts = (int32_t)((near + part - 1) / part);
    w.first_parts = std::max(w.near_parts, (int32_t)((all + first_part - 1) / first_part));
    const int64_t firsts = (int64_t)w.first_tiles * w.first_parts, per_head = firsts + (int64_t)(w.tiles - w.first_tiles) * w.near_parts;
    const int64_t slots = w.near_parts > 1 ? per_head : w.first_parts > 1 ? firsts : 0;
    // (Fewer than 2^23 items in all for whatever is supported: heads * tiles < 2^22 + 2^16, and there is more than one part only of tiles that leave these few.)
    w.head_items = (int32_t)per_head;
    w.head_slots = (int32_t)slots;
    w.items = (int32_t)(heads * per_head);
    w.per_xcd = (w.items + 7) / 8;
    Scratch scratch{(uint8_t*)work};
    g.fd_tiles = make_fastdiv(1);
    g.stats = (int64_t)s.batch * s.q_heads * s.n_q;
    g.delta = scratch.take<float>(g.stats + 1);
    g.lse2 = scratch.take<float>(g.stats + 1);
    g.slots = scratch.take<float>(heads * slots * 128 * D);
    g.heads = (int32_t)heads;
    if (seq->dtype == GRAT_F16) {
        g.head_runs = s.n_groups * p.row_tiles * (plan.tile_rows / 32);
        g.row_bits = scratch.take<int32_t>(heads * g.head_runs);
        g.head_bits = scratch.take<int32_t>(heads);
        w.own_bits = g.head_runs <= 512;
    }
    plan.work = scratch.bytes;
    *out = plan;
    return GRAT_OK;
}

// ---- caches --------------------------------------------------------------------------------------
// Rows in 8 bits, and their scales.
grat_status check_eight(const grat_tensor* t, int32_t head_dim) {
    if (!t || !t->data) return GRAT_ERR_NULL;
    if (t->stride_n < head_dim || t->stride_b < 0 || t->stride_h < 0) return GRAT_ERR_BAD_DIMS;
    if (t->stride_n % 16 || t->stride_b % 16 || t->stride_h % 16 || !aligned16(t->data)) return GRAT_ERR_UNSUPPORTED;
    if (t->stride_n >= ((int64_t)1 << 24) || t->stride_b >= ((int64_t)1 << 46) || t->stride_h >= ((int64_t)1 << 46)) return GRAT_ERR_UNSUPPORTED;
    return GRAT_OK;
}
grat_status check_scale(const grat_tensor* t) {
    if (!t || !t->data) return GRAT_ERR_NULL;
    if (t->stride_n < 1 || t->stride_b < 0 || t->stride_h < 0) return GRAT_ERR_BAD_DIMS;
    if ((uintptr_t)t->data & 3) return GRAT_ERR_UNSUPPORTED;
    if (t->stride_n >= ((int64_t)1 << 24) || t->stride_b >= ((int64_t)1 << 46) || t->stride_h >= ((int64_t)1 << 46)) return GRAT_ERR_UNSUPPORTED;
    return GRAT_OK;
}
grat_status not_repeated(const grat_tensor* t, int32_t batch, int32_t heads) {   // what is written to
    return (batch > 1 && t->stride_b == 0) || (heads > 1 && t->stride_h == 0) ? GRAT_ERR_BAD_DIMS : GRAT_OK;
}
// A cache of either kind.
grat_status check_cache(const grat_tensor* t, const grat_tensor* scale, grat_dtype dtype, int32_t head_dim) {
    if (!scale) return check_tensor(t, dtype, head_dim);
    const grat_status st = check_eight(t, head_dim);
    return st == GRAT_OK ? check_scale(scale) : st;
}

}  // namespace
}  // namespace grat

using namespace grat;

extern "C" int64_t grat_window_attention_work(const grat_sequence* seq, int32_t window, int32_t sinks, int32_t backward) {
    ForwardPlan f;
    GradPlan g;
    if (backward) return make_gradient(seq, 1.f, window, sinks, nullptr, &g) == GRAT_OK ? g.work : 0;
    return make_forward(seq, 1.f, window, sinks, false, false, nullptr, &f) == GRAT_OK ? f.work : 0;
}

extern "C" grat_status grat_window_attention_fwd(const grat_sequence* seq, const grat_tensor* Q, const grat_tensor* K, const grat_tensor* V,
                                                 const grat_tensor* O, float* d_lse, float scale, int32_t window, int32_t sinks, void* d_work,
                                                 void* hip_stream) {
    ForwardPlan plan;
    grat_status st = make_forward(seq, scale, window, sinks, false, false, d_work, &plan);
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
    return launch_forward(plan, seq, false, hip_stream);
}

extern "C" grat_status grat_window_attention_bwd(const grat_sequence* seq, const grat_tensor* dO, const grat_tensor* Q, const grat_tensor* K,
                                                 const grat_tensor* V, const grat_tensor* O, const float* d_lse, const grat_tensor* dQ,
                                                 const grat_tensor* dK, const grat_tensor* dV, float scale, int32_t window, int32_t sinks,
                                                 void* d_work, void* hip_stream) {
    if (!d_lse) return GRAT_ERR_NULL;
    GradPlan plan;
    grat_status st = make_gradient(seq, scale, window, sinks, d_work, &plan);
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
    GradParams& g = plan.g;
    g.dO = of(dO);
    g.dQ = of(dQ);
    g.dK = of(dK);
    g.dV = of(dV);
    const bool f16 = seq->dtype == GRAT_F16, wide = seq->head_dim == 128;
    const auto launch = f16 ? (wide ? launch_window_bwd_f16_d128 : launch_window_bwd_f16_d64)
                            : (wide ? launch_window_bwd_bf16_d128 : launch_window_bwd_bf16_d64);
    return status_of(launch(p, g, plan.tile_rows, (hipStream_t)hip_stream));
}

extern "C" grat_status grat_cache_append(const grat_rotary_args* args, const grat_tensor* Q, const grat_tensor* Q_out, const grat_tensor* K,
                                         const grat_tensor* V, const grat_tensor* K_cache, const grat_tensor* V_cache, const grat_tensor* K_scale,
                                         const grat_tensor* V_scale, int32_t n_cache, void* hip_stream) {
    if (!args) return GRAT_ERR_NULL;
    grat_rotary_args r = *args;
    const bool with_q = Q || Q_out, eight = K_scale || V_scale;
    if (!with_q) r.q_heads = 1;   // (what is not read)
    if (!r.d_table) {
        r.rot = 16;
        r.axes = 1;
        r.axis_pairs[0] = 8;
        r.n_pos = 1;
        r.d_positions = nullptr;
        r.d_table = (const float*)16;
    }
    AppendParams a{};
    RotaryParams& p = a.p;
    grat_status st = make_rotary(&r, true, &p);
    if (st != GRAT_OK) return st;
    if (!args->d_table) {
        p.rot = 0;
        p.table = nullptr;
    }
    if (r.head_dim != 64 && r.head_dim != 128) return GRAT_ERR_UNSUPPORTED;
    if (!r.d_start) return GRAT_ERR_NULL;
    if (n_cache < 1 || r.inverse) return GRAT_ERR_BAD_DIMS;
    if (n_cache >= kMaxRows) return GRAT_ERR_UNSUPPORTED;
    if ((int64_t)r.batch * r.n_tokens * (r.q_heads + 2 * (int64_t)r.kv_heads) >= (int64_t)1 << 35) return GRAT_ERR_UNSUPPORTED;
    if (with_q) {
        st = check_tensor(Q, r.dtype, r.head_dim);
        if (st == GRAT_OK) st = check_output(Q_out, r.dtype, r.head_dim, r.batch, r.q_heads);
    }
    for (const grat_tensor* t : {K, V})
        if (st == GRAT_OK) st = check_tensor(t, r.dtype, r.head_dim);
    const grat_tensor *const caches[2] = {K_cache, V_cache}, *const scales[2] = {K_scale, V_scale};
    for (int i = 0; i < 2 && st == GRAT_OK; ++i) {
        if (eight && !scales[i]) return GRAT_ERR_NULL;
        st = check_cache(caches[i], scales[i], r.dtype, r.head_dim);
        if (st == GRAT_OK) st = not_repeated(caches[i], r.batch, r.kv_heads);
        if (st == GRAT_OK && eight) st = not_repeated(scales[i], r.batch, r.kv_heads);
    }
    if (st != GRAT_OK) return st;
    if (with_q) {
        p.in[0] = of(Q);
        p.out[0] = of(Q_out);
    } else {
        p.heads[0] = 0;
    }
    p.in[1] = of(K);
    p.in[2] = of(V);
    p.out[1] = of(K_cache);
    p.out[2] = of(V_cache);
    p.heads[2] = p.heads[1];
    p.n_cache = n_cache;
    if (eight) {
        a.k_scale = of(K_scale);
        a.v_scale = of(V_scale);
    }
    return status_of(launch_cache_append(a, r.dtype, eight, (hipStream_t)hip_stream));
}

extern "C" grat_status grat_cache_read(grat_dtype dtype, int32_t batch, int32_t heads, int32_t n_rows, int32_t head_dim, const grat_tensor* cache,
                                       const grat_tensor* scale, const int32_t* d_k_len, const grat_tensor* out, void* hip_stream) {
    if (batch < 1 || heads < 1 || n_rows < 1) return GRAT_ERR_BAD_DIMS;
    if (!known(dtype) || (head_dim != 64 && head_dim != 128)) return GRAT_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)batch * heads * n_rows;
    if ((int64_t)batch * heads > 65535 || n_rows >= kMaxRows || rows >= kMaxRows / 4) return GRAT_ERR_UNSUPPORTED;
    if (!scale) return GRAT_ERR_NULL;
    grat_status st = check_cache(cache, scale, dtype, head_dim);
    if (st == GRAT_OK) st = check_output(out, dtype, head_dim, batch, heads);
    if (st != GRAT_OK) return st;
    const ReadParams p{of(cache), of(scale), of(out), d_k_len, rows * (head_dim / 16), make_fastdiv((uint32_t)head_dim / 16), make_fastdiv((uint32_t)n_rows),
                       make_fastdiv((uint32_t)heads)};
    return status_of(launch_cache_read(p, dtype, (hipStream_t)hip_stream));
}

extern "C" int64_t grat_cache_attention_work(const grat_sequence* seq, int32_t window, int32_t sinks, int32_t eight) {
    if (!seq) return 0;
    const grat_sequence q = newest(*seq);
    ForwardPlan chain, tree;   // (a tree of more tokens than there may be is refused by the call itself)
    if (make_forward(&q, 1.f, window, sinks, eight != 0, false, nullptr, &chain) != GRAT_OK) return 0;
    return make_forward(&q, 1.f, window, sinks, eight != 0, true, nullptr, &tree) == GRAT_OK ? std::max(chain.work, tree.work) : chain.work;
}

extern "C" grat_status grat_cache_attention_fwd(const grat_sequence* seq, const grat_tensor* Q, const grat_tensor* K_cache, const grat_tensor* V_cache,
                                                const grat_tensor* K_scale, const grat_tensor* V_scale, const grat_tensor* O, float* d_lse, float scale,
                                                int32_t window, int32_t sinks, const int32_t* d_parent, int64_t parent_stride_b, void* d_work,
                                                void* hip_stream) {
    if (!seq) return GRAT_ERR_NULL;
    const grat_sequence q = newest(*seq);
    const bool eight = K_scale || V_scale;
    ForwardPlan plan;
    grat_status st = make_forward(&q, scale, window, sinks, eight, d_parent != nullptr, d_work, &plan);
    if (st == GRAT_OK) st = check_tensor(Q, seq->dtype, seq->head_dim);
    if (st == GRAT_OK && eight && (!K_scale || !V_scale)) st = GRAT_ERR_NULL;
    if (st == GRAT_OK) st = check_cache(K_cache, K_scale, seq->dtype, seq->head_dim);
    if (st == GRAT_OK) st = check_cache(V_cache, V_scale, seq->dtype, seq->head_dim);
    if (st == GRAT_OK) st = check_output(O, seq->dtype, seq->head_dim, seq->batch, seq->q_heads);
    if (st == GRAT_OK && d_parent && parent_stride_b < 0) st = GRAT_ERR_BAD_DIMS;
    if (st != GRAT_OK) return st;
    if (plan.work > 0 && !d_work) return GRAT_ERR_NULL;
    if (!aligned16(d_work)) return GRAT_ERR_UNSUPPORTED;
    SelParams& p = plan.p;
    p.Q = of(Q);
    p.K = of(K_cache);
    p.V = of(V_cache);
    p.O = of(O);
    p.lse = d_lse;
    if (eight) {
        p.k_scale = of(K_scale);
        p.v_scale = of(V_scale);
    }
    p.parent = d_parent;
    p.parent_stride_b = parent_stride_b;
    return launch_forward(plan, seq, eight, hip_stream);
}
