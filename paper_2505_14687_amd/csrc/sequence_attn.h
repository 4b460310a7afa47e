// Attention over lists of key blocks, within a window and over caches, on the matrix cores of gfx950: what the forward and the gradient kernels share.
//
// The rows of a query group - q_group queries of each of the heads that share a K/V head, head by head - all walk the group's list, so every
// (row tile, key unit) product is a dense one; only the newest keys and the end of a sequence need a mask.  The products are the
// "transposed" ones of attn_mfma.h: with X the operand that streams through LDS and Y the one whose rows a wave owns (its 32
// columns of the instruction, in registers as B fragments), T = X Y^T leaves lane (c = lane % 32, half = lane / 32) with the 16 streamed
// rows 8 (r / 4) + 4 half + r % 4 of its own row c per 32, and that layout, packed to 16 bits, is the B operand of
// Z^T += X'^T T if the contraction index is enumerated in the same order.  X'^T fragments come out of row-major tiles
// through the LDS transpose read.
//
// A window needs no list: what the rows of a group see together is two runs of keys, the first ones and those near (KeyRange), and the
// walk's units of 32 keys follow from their number (WindowUnits).  Rows of a group are neighbours, so a mask is needed at the ends of the runs only.  Drafted tokens
// see the committed ones as a window's rows do, and of their own number a line, kept as bits (Tree).
#pragma once
#include "mfma_elem.h"
#include "sequence_common.h"

namespace grat {

struct SelParams {
    SeqShape s;
    SeqTensor Q, K, V, O;
    float* lse;
    const int32_t* count;
    const int32_t* index;
    int32_t max_blocks;
    float scale, scale_log2;
    int32_t rows, row_tiles;      // rows of a group (q_group * share), workgroups they are cut into
    int32_t splits;               // workgroups that share a list
    int32_t items, per_xcd;       // workgroups with work, those of an XCD
    FastDiv fd_splits, fd_row_tiles, fd_groups, fd_kv_heads, fd_q_group, fd_units;   // fd_units: by block / 32
    float* part_o;                // splits > 1: [items][rows of a tile][D], with part_ml [items][rows of a tile][2]
    float* part_ml;
    int64_t window;               // attention within a window: no lists, q_group is the launch's own
    int32_t sinks;
    SeqTensor k_scale, v_scale;   // K and V in 8 bits: a float a row
    const int32_t* parent;        // drafted tokens, or null
    int64_t parent_stride_b;
    int32_t slots, part_keys, part_step;   // parts that the sequences share (Parts), or 0; keys of a unit; units that a workgroup takes at a time
};
constexpr int64_t kNoWindow = (int64_t)1 << 40;   // more than any two positions are apart

// The walk over keys of attention within a window: key tiles of 64 keys, the rows that see a tile cut into parts of about equal length.  Rows that see
// one of the first keys are as many as there are, of others at most a window's.
struct WindowGradParams {
    int32_t tiles, first_tiles;         // of a K/V head; those that hold first keys
    int32_t first_parts, near_parts;    // parts of either kind of tile
    int32_t items, per_xcd;             // of the launch
    int32_t head_items, head_slots;     // items and places in `slots` of a K/V head
    int32_t own_bits;                   // half: every workgroup works out its head's exponent itself
};

// What the gradient needs beside SelParams, in the caller's scratch memory.
struct GradParams {
    SeqTensor dO, dQ, dK, dV;
    float* delta;          // [batch][q_heads][n_q], and one more: D
    float* lse2;           // as many: lse in base 2
    int64_t stats;         // batch * q_heads * n_q
    uint32_t* bits;        // [blocks of all heads][words]
    int32_t* counters;     // entries of `groups` in use, long parts, slots in use, blocks of more than one part, short parts
    int32_t* groups;       // the groups that list a block, block after block
    int4* parts;           // block (of all heads), first group's place in `groups`, rows from and to
    int32_t* part_slot;    // of every part: its slot, -1: its block has no other
    int4* joins;           // blocks of more than one part: block, first slot, parts
    float* slots;          // sums of a part: [key tile of the block][dK, dV][key][D]
    int32_t* row_bits;     // half: exponents that dS is formed with, the smallest of each run of (at most 32) rows, head after head; else null
    int32_t* head_bits;    // half: the exponent of a K/V head
    int32_t heads, head_runs;   // K/V heads of the batch, runs of each
    int32_t words, blocks, most_parts, most_joins, part_rows;
    FastDiv fd_rows, fd_tiles, fd_top, fd_part;   // by rows of a group; key tiles of a block; max_blocks; part_rows
    WindowGradParams window;   // attention within a window: in the place of bits .. joins
};

// Dispatch by element type and head_dim (sequence_fwd_*.hip, sequence_bwd_*.hip).
hipError_t launch_selected_fwd_bf16_d128(const SelParams& p, int tile_rows, hipStream_t stream);
hipError_t launch_selected_fwd_bf16_d64(const SelParams& p, int tile_rows, hipStream_t stream);
hipError_t launch_selected_fwd_f16_d128(const SelParams& p, int tile_rows, hipStream_t stream);
hipError_t launch_selected_fwd_f16_d64(const SelParams& p, int tile_rows, hipStream_t stream);
hipError_t launch_selected_bwd_bf16_d128(const SelParams& p, const GradParams& g, int tile_rows, int tile_keys, hipStream_t stream);
hipError_t launch_selected_bwd_bf16_d64(const SelParams& p, const GradParams& g, int tile_rows, int tile_keys, hipStream_t stream);
hipError_t launch_selected_bwd_f16_d128(const SelParams& p, const GradParams& g, int tile_rows, int tile_keys, hipStream_t stream);
hipError_t launch_selected_bwd_f16_d64(const SelParams& p, const GradParams& g, int tile_rows, int tile_keys, hipStream_t stream);
void launch_grad_lists(const SelParams& p, const GradParams& g, hipStream_t stream);
void launch_grad_head_bits(const GradParams& g, hipStream_t stream);
// ... of attention within a window and over caches (cache_attn_*.hip, window_bwd_*.hip).  eight: K and V in 8 bits; p.parent: a tree
hipError_t launch_cache_attention_bf16_d128(const SelParams& p, bool eight, int tile_rows, hipStream_t stream);
hipError_t launch_cache_attention_bf16_d64(const SelParams& p, bool eight, int tile_rows, hipStream_t stream);
hipError_t launch_cache_attention_f16_d128(const SelParams& p, bool eight, int tile_rows, hipStream_t stream);
hipError_t launch_cache_attention_f16_d64(const SelParams& p, bool eight, int tile_rows, hipStream_t stream);
hipError_t launch_window_bwd_bf16_d128(const SelParams& p, const GradParams& g, int tile_rows, hipStream_t stream);
hipError_t launch_window_bwd_bf16_d64(const SelParams& p, const GradParams& g, int tile_rows, hipStream_t stream);
hipError_t launch_window_bwd_f16_d128(const SelParams& p, const GradParams& g, int tile_rows, hipStream_t stream);
hipError_t launch_window_bwd_f16_d64(const SelParams& p, const GradParams& g, int tile_rows, hipStream_t stream);

constexpr int kUnit = 32;         // keys that are looked up, masked and skipped together
constexpr int kNoUnit = 0x7fffff00;   // start of a unit that only fills a tile: behind every key

// ---- LDS tiles -------------------------------------------------------------------------------
// Tiles are unpadded, rows of D / 8 chunks of 16 bytes; chunk c of a row lies at c ^ swizzle(row).  One swizzle serves both
// reads.  ds_read_b128, lanes = consecutive rows (and the two halves of a wave neighbouring chunks): 8 rows x 2 chunks, and 16 rows,
// fall on the 16 chunk positions of a 256-byte line.  The transpose read takes 4 rows x 4 neighbouring chunks at a time: rows e = 0 .. 3 go to
// different groups of 4 positions.  head_dim 64 has two rows in a line.
template <int D>
__device__ __forceinline__ int tile_swizzle(int row) {
    return D == 128 ? (row & 3) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1) : ((row >> 1) & 1) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1);
}

// Where a wave's fragments lie in the current one of two neighbouring tiles.  One register a kind of read: what differs between reads is XORed
// in (chunks) or a constant offset (tiles, rows).  (Left to itself the compiler keeps an address for every chunk, 16 registers.)
template <int D>
struct TileReader {
    static constexpr int kRow = 2 * D, kTile = 64 * kRow;
    uint32_t row_at, col_at;
    // `tiles`: aligned to two tiles; block 0 of this wave is block `first` of a tile
    __device__ __forceinline__ TileReader(int lane, const uint8_t* tiles, int first) {
        const uint32_t base = (uint32_t)(uintptr_t)(LDS_PTR(const uint8_t))tiles + 32 * first * kRow;
        const int c = lane & 31, half = lane >> 5;
        row_at = base + c * kRow + ((tile_swizzle<D>(c) ^ half) << 4);
        const int e = (lane & 15) >> 2, cq = lane & 3, dsel = (lane >> 4) & 1, row = 4 * half + e;
        col_at = base + row * kRow + (((2 * dsel + (cq >> 1)) ^ tile_swizzle<D>(row)) << 4) + 8 * (cq & 1);
    }
    __device__ __forceinline__ void flip() {   // to the other tile
        row_at ^= kTile;
        col_at ^= kTile;
        asm volatile("" : "+v"(row_at), "+v"(col_at));
    }
    // A operand, rows = tile rows 32 block + c, dims 16 ks + 8 half .. + 7.  pair: tiles 2 pair and 2 pair + 1; odd: the second of
    // them, for callers that do not flip
    __device__ __forceinline__ frag8 rows(int pair, int block, int ks, int odd = 0) const {
        return *(LDS_PTR(const frag8))(uintptr_t)((row_at ^ (ks << 5)) + (2 * pair + odd) * kTile + 32 * block * kRow);
    }
    // A operand, rows = dims 32 db + c, contracted over 16 tile rows: 32 block + 16 s2 + accumulator order.  (8 rows on the swizzle
    // differs in its lowest bit.)
    __device__ __forceinline__ frag8 cols(int pair, int block, int s2, int db, int odd = 0) const {
        const uint32_t at = col_at ^ (db << 6), off = (2 * pair + odd) * kTile + (32 * block + 16 * s2) * kRow;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)(at + off));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)((at ^ 16) + off + 8 * kRow));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// 1 KiB, one 16-byte chunk a lane, from per-lane offsets against a uniform address straight into LDS (at dst + 16 lane).  Inline
// assembly on purpose: a load into LDS that the compiler can see makes it wait for all of them ahead of the next LDS
// read.  The caller waits (s_waitcnt) ahead of the barrier that publishes the tile.
__device__ __forceinline__ void load_lds(const uint8_t* base, uint32_t off, uint8_t* dst) {
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(LDS_PTR(uint8_t))dst);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
// ... from a 64-bit address of every lane's own
__device__ __forceinline__ void load_lds(const uint8_t* src, uint8_t* dst) {
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(LDS_PTR(uint8_t))dst);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(src) : "memory", "m0");
}

// ... 4 bytes a lane, at dst + 4 lane
__device__ __forceinline__ void load_lds_word(const uint8_t* src, uint8_t* dst) {
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(LDS_PTR(uint8_t))dst);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(src) : "memory", "m0");
}

// This wave's loads have landed, and what it read from LDS is in registers.
__device__ __forceinline__ void wave_wait() {
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");   // (no LDS read moves up past the wait)
}

// This wave's direct loads have landed, everyone's have, and everyone is done with the buffers that are filled next.
__device__ __forceinline__ void tile_barrier() {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
}

// ---- the list of a group -----------------------------------------------------------------------
// First keys of the units of a group's list that hold a key below `seen`, in list order, into LDS; returns their number (every
// thread of the workgroup calls it, it ends with a barrier), followed by one kNoUnit.
__device__ __forceinline__ int list_units(const SelParams& p, int64_t list, int seen, int32_t* s_units, int32_t* s_n) {
    if (threadIdx.x < 64) {
        // (the count and the first entries are asked for together)
        const int lane = threadIdx.x, per = (int)p.fd_units.d;
        const int32_t* const entries = p.index + list * p.max_blocks;
        const int listed = p.count[list], ahead = entries[min((int)fdiv((uint32_t)lane, p.fd_units), p.max_blocks - 1)];
        const int n = min(max(listed, 0), p.max_blocks) * per;
        int have = 0;
        for (int u0 = 0; u0 < n; u0 += 64) {
            const int u = u0 + lane;
            uint32_t entry, part;
            fdivmod((uint32_t)min(u, n - 1), p.fd_units, entry, part);
            const int block = u0 == 0 ? ahead : entries[entry];
            const int start = min(max(block, 0), p.s.n_blocks - 1) * p.s.block + (int)part * kUnit;
            const bool in = u < n && block >= 0 && block < p.s.n_blocks && start < seen;
            const uint64_t all = __ballot(in);
            if (in) s_units[have + __popcll(all & ((1ull << lane) - 1ull))] = start;
            have += __popcll(all);
        }
        if (lane == 0) {
            s_units[have] = kNoUnit;
            *s_n = have;
        }
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(*s_n);
}

// Which part of the launch a workgroup is: consecutive items go to one XCD, whose L2 then holds the K and V of few heads.
struct Item {
    int item, b, h, g, tile, split;
    __device__ __forceinline__ explicit Item(const SelParams& p) {
        item = ((int)blockIdx.x & 7) * p.per_xcd + ((int)blockIdx.x >> 3);
        uint32_t t, s, m, bh, gg, bb, hh;
        fdivmod((uint32_t)item, p.fd_splits, t, s);
        fdivmod(t, p.fd_row_tiles, t, m);
        fdivmod(t, p.fd_groups, bh, gg);
        fdivmod(bh, p.fd_kv_heads, bb, hh);
        b = (int)bb; h = (int)hh; g = (int)gg; tile = (int)m; split = (int)s;
    }
    __device__ __forceinline__ bool idle(const SelParams& p) const { return (int)(blockIdx.x >> 3) >= p.per_xcd || item >= p.items; }
    __device__ __forceinline__ bool share(const SelParams& p, int& units);
    __device__ __forceinline__ int64_t list(const SelParams& p) const { return ((int64_t)b * p.s.kv_heads + h) * p.s.n_groups + g; }
};

// Row r of a group: its head and query row; not there where it is behind the group's or the tensor's last.
struct GroupRow {
    int head, query;
    bool there;
    __device__ __forceinline__ GroupRow(const SelParams& p, int h, int g, int r) {
        uint32_t e, i;
        fdivmod((uint32_t)min(r, p.rows - 1), p.fd_q_group, e, i);
        head = h * p.s.share + (int)e;
        query = g * p.s.q_group + (int)i;
        there = r < p.rows && query < p.s.n_q;
        query = min(query, p.s.n_q - 1);
    }
};

__device__ __forceinline__ const uint8_t* row_address(const SeqTensor& t, int b, int head, int row) {
    return t.data + 2 * (b * t.stride_b + head * t.stride_h + row * t.stride_n);
}

// ---- windows --------------------------------------------------------------------------------------
// The query in row i, at position pos + i, sees the keys [0, first) and [lo, hi): the first keys and its window.  All three grow with i.
struct RowSpan {
    int first, lo, hi;
};
__device__ __forceinline__ int64_t window_pos(const SeqShape& s, int b, int len) { return s.q_pos ? (int64_t)s.q_pos[b] : (int64_t)len - s.n_q; }
__device__ __forceinline__ RowSpan row_span(const SelParams& p, int len, int64_t pos, int i) {
    const int64_t at = pos + i;
    RowSpan r;
    r.hi = (int)max((int64_t)0, min((int64_t)len, p.s.causal ? at + 1 : at + p.window));
    r.lo = (int)max((int64_t)0, min((int64_t)r.hi, at - p.window + 1));
    r.first = min(p.sinks, p.s.causal ? r.hi : len);
    return r;
}
// The keys that the rows [i0, i1] see, as units of 32 keys: of the first keys from key 0 on, then from the first key of row i0's window on that is
// not among these.  A unit's keys that no row sees are not read: the last one that some row sees stands for them.
struct KeyRange {
    int first_end, near, near_end;
    __device__ __forceinline__ int units(int keys) const { return (first_end + keys - 1) / keys + (max(near_end - near, 0) + keys - 1) / keys; }
};
__device__ __forceinline__ KeyRange rows_range(const SelParams& p, int len, int64_t pos, int i0, int i1) {
    const RowSpan a = row_span(p, len, pos, i0), z = row_span(p, len, pos, i1);
    return KeyRange{z.first, max(a.lo, z.first), z.hi};
}
// ... of a tree: its first token is one that goes on from a committed one, and no other sees more of these.
__device__ __forceinline__ KeyRange tree_range(const SelParams& p, int len) {
    const int base = len - p.s.n_q, committed = max(base, 0), first = min(p.sinks, committed);
    return KeyRange{first, (int)max((int64_t)first, min((int64_t)committed, base - p.window + 1)), len};
}
// (The same in all lanes, which what it is computed from does not always say.)
__device__ __forceinline__ KeyRange uniform(const KeyRange& r) {
    return KeyRange{__builtin_amdgcn_readfirstlane(r.first_end), __builtin_amdgcn_readfirstlane(r.near), __builtin_amdgcn_readfirstlane(r.near_end)};
}
struct WindowUnits : KeyRange {
    int first_units, n;
    __device__ __forceinline__ explicit WindowUnits(const KeyRange& r) : KeyRange(uniform(r)) {
        first_units = (first_end + kUnit - 1) / kUnit;
        n = units(kUnit);
    }
    __device__ __forceinline__ int start(int i) const { return i < first_units ? i * kUnit : near + (i - first_units) * kUnit; }
};

// Sequences of lengths that the host does not know, whose keys few workgroups share: the parts of all of them, p.slots for a K/V head's row tile, are
// of about equal length, and not shorter than pays.  A sequence a lane, at most 64.  (64 drafted tokens x 4 heads over 4 caches of 10 240 to 16 384 keys 83.1 -> 76.5 us.)
__device__ __forceinline__ int sum_up_to(int x) {   // of the lanes up to this one
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // lane - 1, - 2, - 4, - 8 of its row of 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // the row ahead, the two rows ahead
    return x + __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
}
struct Parts {
    int n, end, per;   // parts of this lane's sequence, and of all up to it; units of a part
    __device__ __forceinline__ explicit Parts(const SelParams& p) {   // by whole waves
        const SeqShape& s = p.s;
        const int lane = threadIdx.x & 63, b = min(lane, s.batch - 1), len = seq_len(s, b);
        const KeyRange r = p.parent ? tree_range(p, len) : rows_range(p, len, window_pos(s, b, len), 0, s.n_q - 1);
        const int units = lane < s.batch ? r.units(p.part_keys) : 0, step = p.part_step, all = __builtin_amdgcn_readlane(sum_up_to(units), 63);
        // (least: two steps of 64 keys of many rows; one of few, two where there are 24 and more)
        const int least = step < 4 || all >= 24 * step * s.batch ? 2 * step : step;
        per = (max((all + p.slots - 1) / p.slots, least) + step - 1) / step * step;
        for (;; per += (per / 16 + step) / step * step) {   // (as soon as a part holds the longest one there are no more parts than sequences)
            n = (units + per - 1) / per;
            end = sum_up_to(n);
            if (__builtin_amdgcn_readlane(end, 63) <= p.slots) break;
        }
    }
    // The sequence that part k belongs to, p.s.batch if none.
    __device__ __forceinline__ int of(int k) const { return __popcll(__builtin_amdgcn_ballot_w64(end <= k)); }
};

// Where p.slots says so, `split` is a part of all sequences': finds whose, and the units that it takes.  False: there is none.
__device__ __forceinline__ bool Item::share(const SelParams& p, int& units) {
    if (p.slots == 0) return true;
    const Parts parts(p);
    b = parts.of(split);
    if (b >= p.s.batch) return false;
    split -= __builtin_amdgcn_readlane(parts.end, b) - __builtin_amdgcn_readlane(parts.n, b);
    units = parts.per;
    return true;
}

// A tree of drafted tokens: token t goes on from token parent[t], or from the newest committed token (-1, and whatever is not a token ahead of t).  Its key
// lies in row base + t, its position is base + depth.  lines[t]: the tokens of its line, itself among them, that it sees.
constexpr int kMostDrafted = 256, kTreeWords = 10;   // tokens of a tree; words of a line, the last two 0
struct Tree {
    int32_t parent[kMostDrafted], depth[kMostDrafted];
    uint32_t lines[kMostDrafted * kTreeWords];
    int32_t deep[10];
    uint32_t shallow[kTreeWords - 2];
};
// Lines are doubled, of all tokens at once: round k knows the 2^k tokens from a token upward, and the one above these.  Within a window a line's tokens are gathered by
// the bits of its length.  Up to 64 tokens by each wave for itself, more through LDS.  (One token upward after the other a line of 256 tokens took 40 us and one of 64 ten;
// now 6 and two.)
__device__ __forceinline__ void build_small_tree(Tree& tree, const SelParams& p, int b, int base) {
    const int n = p.s.n_q, t = (int)(threadIdx.x & 63);
    const bool limited = p.window < n;
    const int window = (int)min(p.window, (int64_t)n);
    int up = -1, from = t;   // above the line so far, above `near`
    if (t < n) {
        up = p.parent[b * p.parent_stride_b + t];
        if (up < 0 || up >= t) up = -1;
    }
    int depth = up >= 0;
    uint64_t line = 1ull << t, near = 0;
    for (int k = 0;; ++k) {   // (ends at 2^k >= n at the latest: a parent lies ahead of its child)
        const bool last = __builtin_amdgcn_ballot_w64(up >= 0) == 0;
        if (limited && (last ? window >> k : window >> k & 1)) {
            const uint64_t x = __shfl(line, max(from, 0));
            const int above = __shfl(up, max(from, 0));
            near |= from >= 0 ? x : 0;
            from = from >= 0 ? above : -1;
        }
        if (last) break;
        const uint64_t x = __shfl(line, max(up, 0));
        const int d = __shfl(depth, max(up, 0)), above = __shfl(up, max(up, 0));
        line |= up >= 0 ? x : 0;
        depth += up >= 0 ? d : 0;
        up = up >= 0 ? above : -1;
    }
    if (limited) line = near | (line & __builtin_amdgcn_ballot_w64(base + depth < p.sinks));   // (tokens that stay visible for their positions)
    if (threadIdx.x < 64 && t < n) {
        uint32_t* const to = tree.lines + t * kTreeWords;
        to[0] = (uint32_t)line;
        to[1] = (uint32_t)(line >> 32);
#pragma unroll
        for (int w = 2; w < kTreeWords; ++w) to[w] = 0;
        tree.depth[t] = depth;
    }
    __syncthreads();
}
__device__ __forceinline__ void build_tree(Tree& tree, const SelParams& p, int b, int base) {   // by at least kMostDrafted threads; ends with a barrier
    if (p.s.n_q <= 64) return build_small_tree(tree, p, b, base);
    constexpr int kWords = kTreeWords - 2;
    const int n = p.s.n_q, t = (int)threadIdx.x, words = (n + 31) >> 5;
    const bool limited = p.window < n;
    const int window = (int)min(p.window, (int64_t)n);
    uint32_t line[kWords], near[kWords];
    int up = -1, from = t < n ? t : -1;   // above the line so far, above `near`
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
        line[w] = t >> 5 == w ? 1u << (t & 31) : 0;
        near[w] = 0;
    }
    if (t < 10) tree.deep[t] = 0;
    if (t < n) {
        up = p.parent[b * p.parent_stride_b + t];
        if (up < 0 || up >= t) up = -1;
        for (int w = words; w < kTreeWords; ++w) tree.lines[t * kTreeWords + w] = 0;
    }
    int depth = up >= 0;
    __syncthreads();
    for (int k = 0;; ++k) {   // (ends at 2^k >= n at the latest: a parent lies ahead of its child)
        if (t < n) {
            tree.parent[t] = up;
            tree.depth[t] = depth;
#pragma unroll
            for (int w = 0; w < kWords; ++w)
                if (w < words) tree.lines[t * kTreeWords + w] = line[w];
            if (up >= 0) tree.deep[k] = 1;
        }
        __syncthreads();
        const bool last = tree.deep[k] == 0;
        if (limited && (last ? window >> k : window >> k & 1) && from >= 0) {
#pragma unroll
            for (int w = 0; w < kWords; ++w)
                if (w < words) near[w] |= tree.lines[from * kTreeWords + w];
            from = tree.parent[from];
        }
        if (last) break;
        if (up >= 0) {
#pragma unroll
            for (int w = 0; w < kWords; ++w)
                if (w < words) line[w] |= tree.lines[up * kTreeWords + w];
            depth += tree.depth[up];
            up = tree.parent[up];
        }
        __syncthreads();
    }
    if (!limited) return;
    const uint64_t shallow = __builtin_amdgcn_ballot_w64(base + depth < p.sinks);   // tokens that stay visible for their positions
    if ((t & 63) == 0 && t < 32 * kWords) {
        tree.shallow[t >> 5] = (uint32_t)shallow;
        tree.shallow[(t >> 5) + 1] = (uint32_t)(shallow >> 32);
    }
    __syncthreads();
    if (t < n) {
#pragma unroll
        for (int w = 0; w < kWords; ++w)
            if (w < words) tree.lines[t * kTreeWords + w] = near[w] | (line[w] & tree.shallow[w]);
    }
    __syncthreads();
}
// What a drafted token sees of the committed ones, with hi their number.
__device__ __forceinline__ RowSpan tree_span(const SelParams& p, const Tree& tree, int base, int t) {
    const int committed = max(base, 0);
    const int64_t lo = (int64_t)base + tree.depth[t] - p.window + 1;
    return RowSpan{min(p.sinks, committed), (int)max((int64_t)0, min((int64_t)committed, lo)), committed};
}
// The lower n bits, n from 0 to 32 (what is beyond is taken for the nearest).
__device__ __forceinline__ uint32_t lower_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }
// Bit k: key start + k lies in [low, up).
__device__ __forceinline__ uint32_t range_bits(int start, int low, int up) { return lower_bits(up - start) & ~lower_bits(low - start); }
// ... : is the key of a drafted token that a row with this line sees; off: the token of the first of them.
__device__ __forceinline__ uint32_t line_bits(const uint32_t* line, int off) {
    if (off <= -32) return 0;
    const int w = min(max(off, 0) >> 5, kTreeWords - 2);
    const uint64_t x = line[w] | (uint64_t)line[w + 1] << 32;
    return off < 0 ? (uint32_t)x << -off : (uint32_t)(x >> (off & 31));
}

// What a lane's row does not see of a unit, of 32 rows a wave: of lists, of a window, of a tree.
enum Walk { kLists = 0, kWindow = 1, kTree = 2 };
template <int WALK>
struct RowMask;
template <>
struct RowMask<kLists> {   // keys behind the row's own
    int limit, least, most;   // keys below it are seen; of the wave's rows
    __device__ __forceinline__ RowMask(const SelParams& p, const GroupRow& row, const WindowUnits&, const Tree*, int len, int64_t pos) {
        limit = row.there ? row_seen(p.s, len, pos, row.query) : 0;
        least = row.there ? limit : 0x7fffffff;
        most = limit;
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
            least = min(least, __shfl_xor(least, m));
            most = max(most, __shfl_xor(most, m));
        }
        least = __builtin_amdgcn_readfirstlane(least);
        most = __builtin_amdgcn_readfirstlane(most);
    }
    __device__ __forceinline__ bool nothing() const { return most == 0; }
    __device__ __forceinline__ bool sees() const { return limit > 0; }   // this lane's row
    __device__ __forceinline__ bool idle(int start) const { return start >= most; }   // nobody in this wave sees the unit
    __device__ __forceinline__ bool cuts(int start) const { return start + kUnit > least; }
    __device__ __forceinline__ bool hides(int start, int k) const { return start + k >= limit; }   // key k of the unit
};
template <>
struct RowMask<kWindow> {
    RowSpan r;
    int first_end, least_first, least_hi, most_lo, least_lo, most;
    __device__ __forceinline__ RowMask() {}
    __device__ __forceinline__ RowMask(const SelParams& p, const GroupRow& row, const WindowUnits& u, const Tree*, int len, int64_t pos) {
        of(row, u, row_span(p, len, pos, row.query));
    }
    __device__ __forceinline__ void of(const GroupRow& row, const WindowUnits& u, RowSpan span) {
        r = span;
        if (!row.there) r = RowSpan{0, 0, 0};
        first_end = u.first_end;
        least_first = row.there ? r.first : 0x7fffffff;
        least_hi = row.there ? r.hi : 0x7fffffff;
        least_lo = row.there ? r.lo : 0x7fffffff;
        most_lo = r.lo;
        most = max(r.first, r.hi);
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
            least_first = min(least_first, __shfl_xor(least_first, m));
            least_hi = min(least_hi, __shfl_xor(least_hi, m));
            least_lo = min(least_lo, __shfl_xor(least_lo, m));
            most_lo = max(most_lo, __shfl_xor(most_lo, m));
            most = max(most, __shfl_xor(most, m));
        }
        least_first = __builtin_amdgcn_readfirstlane(least_first);
        least_hi = __builtin_amdgcn_readfirstlane(least_hi);
        least_lo = __builtin_amdgcn_readfirstlane(least_lo);
        most_lo = __builtin_amdgcn_readfirstlane(most_lo);
        most = __builtin_amdgcn_readfirstlane(most);
    }
    __device__ __forceinline__ bool nothing() const { return most == 0; }
    __device__ __forceinline__ bool sees() const { return r.first > 0 || r.hi > r.lo; }
    __device__ __forceinline__ bool idle(int start) const { return start >= most || (start >= first_end && start + kUnit <= least_lo); }
    __device__ __forceinline__ bool cuts(int start) const { return start < first_end ? start + kUnit > least_first : start + kUnit > least_hi || start < most_lo; }
    __device__ __forceinline__ bool hides(int start, int k) const {
        const bool first = start < first_end;
        const int low = first ? 0 : r.lo, width = first ? r.first : r.hi - r.lo;
        return (uint32_t)(start + k - low) >= (uint32_t)width;
    }
};

template <>
struct RowMask<kTree> : RowMask<kWindow> {   // the committed tokens as a window, and a line of drafted ones
    const uint32_t* line;
    int base;
    bool there;
    __device__ __forceinline__ RowMask(const SelParams& p, const GroupRow& row, const WindowUnits& u, const Tree* tree, int len, int64_t) {
        base = len - p.s.n_q;
        there = row.there;
        line = tree->lines + row.query * kTreeWords;
        of(row, u, tree_span(p, *tree, base, row.query));
    }
    __device__ __forceinline__ bool nothing() const { return __builtin_amdgcn_ballot_w64(there) == 0; }
    __device__ __forceinline__ bool idle(int) const { return false; }
    __device__ __forceinline__ uint32_t bits(int start) const {   // bit k: the row sees key k of the unit
        const bool first = start < first_end;
        const uint32_t drafted = line_bits(line, start - base);
        return range_bits(start, first ? 0 : r.lo, first ? r.first : r.hi) | (first || !there ? 0 : drafted);
    }
};

// ---- the walk over a list ------------------------------------------------------------------------
// K and V tiles of 64 keys (two units), double buffered.  NW waves fetch 1-KiB pieces; a wave's pieces lie in one unit.
template <int NW, int D, bool WINDOW = false>
struct KeyLoader {
    static constexpr int kPieces = 64 * D * 2 / 1024, LPW = kPieces / NW, kPerUnit = kPieces / 2, kRows = 1024 / (2 * D), kChunks = D / 8;
    static_assert(LPW >= 1 && kPerUnit % LPW == 0, "a wave's pieces lie in one unit");
    const uint8_t *K, *V;        // of the head
    int64_t pitch_k, pitch_v;    // bytes
    int last;                    // last key that may be read
    int first_end;               // windows: first keys are read up to here
    int my_unit, row[LPW], col[LPW];
    __device__ __forceinline__ KeyLoader(const SelParams& p, const Item& it, int seen, int wave, int lane, int first_keys = 0) {
        first_end = first_keys;
        K = row_address(p.K, it.b, it.h, 0);
        V = row_address(p.V, it.b, it.h, 0);
        pitch_k = 2 * p.K.stride_n;
        pitch_v = 2 * p.V.stride_n;
        last = seen - 1;
        my_unit = wave * LPW / kPerUnit;
#pragma unroll
        for (int k = 0; k < LPW; ++k) {
            const int r = (wave * LPW + k) * kRows + lane / kChunks;   // in the tile
            row[k] = r & (kUnit - 1);
            col[k] = ((lane % kChunks) ^ tile_swizzle<D>(r)) << 4;
        }
    }
    // start: of a listed unit, which begins with a key that some row sees.  Keys behind the last of these are not read: it stands for them, and they are
    // masked.
    __device__ __forceinline__ void issue(const uint8_t* head, int64_t pitch, int start, uint8_t* tile, int wave) const {
        const int left = (WINDOW && start < first_end ? first_end - 1 : last) - start;
        const uint8_t* const base = head + start * pitch;
#pragma unroll
        for (int k = 0; k < LPW; ++k) load_lds(base, (uint32_t)min(row[k], left) * (uint32_t)pitch + col[k], tile + (wave * LPW + k) * 1024);
    }
    __device__ __forceinline__ void issue(int start, uint8_t* k_tile, uint8_t* v_tile, int wave) const {
        issue(K, pitch_k, start, k_tile, wave);
        issue(V, pitch_v, start, v_tile, wave);
    }
};

// The same of K and V in 8 bits, by way of registers (a load into LDS cannot widen them; a tile of 256 rows walks a cache of 8 bits as fast as one of 16: 64 tokens of 4
// sequences over 8 192 keys 48 us against 51): e4m3 values times their row's scale are rounded to the element type (scales that are powers of two leave
// nothing to round; half saturates) and stored as the direct loads would have them.
template <int NW, bool F16, int D>
struct EightLoader {
    static constexpr int kOwnRows = 64 / NW, kC = kOwnRows * (D / 16) / 64;   // rows of a wave; chunks of 16 numbers a lane
    static_assert(kC >= 1, "");
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    struct Raw {
        u32x4 x[kC];
        float s[kC];
    };
    const uint8_t *K, *V, *ks, *vs;
    int64_t pitch_k, pitch_v, pitch_ks, pitch_vs;   // bytes
    int last, first_end, my_unit, first_row, chunk;
    __device__ __forceinline__ EightLoader(const SelParams& p, const Item& it, int seen, int wave, int lane, int first_keys) {
        K = p.K.data + it.b * p.K.stride_b + it.h * p.K.stride_h;
        V = p.V.data + it.b * p.V.stride_b + it.h * p.V.stride_h;
        ks = p.k_scale.data + 4 * (it.b * p.k_scale.stride_b + it.h * p.k_scale.stride_h);
        vs = p.v_scale.data + 4 * (it.b * p.v_scale.stride_b + it.h * p.v_scale.stride_h);
        pitch_k = p.K.stride_n;
        pitch_v = p.V.stride_n;
        pitch_ks = 4 * p.k_scale.stride_n;
        pitch_vs = 4 * p.v_scale.stride_n;
        last = seen - 1;
        first_end = first_keys;
        my_unit = wave * kOwnRows / kUnit;
        first_row = wave * kOwnRows + lane / (D / 16);   // in the tile
        chunk = lane % (D / 16);
    }
    __device__ __forceinline__ void issue(const uint8_t* head, int64_t pitch, const uint8_t* scales, int64_t scale_pitch, int start, Raw& raw) const {
        const int left = (start < first_end ? first_end - 1 : last) - start;
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            const int64_t row = start + min((first_row + c * (1024 / D)) & (kUnit - 1), left);
            raw.x[c] = *(const u32x4*)(head + row * pitch + 16 * chunk);
            raw.s[c] = *(const float*)(scales + row * scale_pitch);
        }
    }
    __device__ __forceinline__ void issue_k(int start, Raw& raw) const { issue(K, pitch_k, ks, pitch_ks, start, raw); }
    __device__ __forceinline__ void issue_v(int start, Raw& raw) const { issue(V, pitch_v, vs, pitch_vs, start, raw); }
    __device__ __forceinline__ void store(const Raw& raw, uint8_t* tile) const {
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            const int row = first_row + c * (1024 / D);
            uint8_t* const to = tile + row * 2 * D;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t word = raw.x[c][2 * j + (i >> 1)];
                    const f32x2 v = i & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)word, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)word, false);
                    float lo = v[0] * raw.s[c], hi = v[1] * raw.s[c];
                    if constexpr (F16) {   // (NaN stays)
                        lo = lo > 65504.f ? 65504.f : lo < -65504.f ? -65504.f : lo;
                        hi = hi > 65504.f ? 65504.f : hi < -65504.f ? -65504.f : hi;
                    }
                    w[i] = Elem<F16>::pack(lo, hi);
                }
                *(uint4*)(to + (((2 * chunk + j) ^ tile_swizzle<D>(row)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
};

// ---- groups of at most 16 rows ------------------------------------------------------------------
// Single tokens, lists of single queries: bound by fetching K and V, which no other rows share.  A workgroup is four waves that take every fourth
// unit of the list and wait for nothing but their own loads.  The 16x16x32 instruction wastes no columns: with Y the group's
// rows, T^T (32 keys x 16 rows, two instructions a step) leaves lane (row r = lane % 16, g = lane / 16) with keys 16 m + 4 g + i, and
// Z^T[16 dims, row] += X'^T T is contracted in that order: elements 0 .. 3 keys 4 g + i, 4 .. 7 keys 16 + 4 g + i.
// A wave has one unit of K and one of V in LDS, 16 KiB (head_dim 128): as soon as either has landed it is read into fragments, and the next one's
// loads go out into the same place.  So one of the two is on its way at any time.  (Straight from memory into fragments the 64 bytes
// of a row belong to lanes 16 apart, and a load takes four times the cycles.)  Measured: 5 227 queries x 8 lists of 4 rows over 512 keys 600 us, 739
// straight into fragments; 11 GB out of the L2, 18 TB/s or 30 bytes a cycle and compute unit, which no kernel here exceeds by much.  The gradient's
// walk over the same 740 us, 870 straight.  17 to 32 rows, two sets of 16, lose to 32x32 instructions: 2 047 tokens of half 74.5 us a training
// step against 67.5.
template <int D>
struct NarrowWave {
    static constexpr int kRow = 2 * D, kTile = kUnit * kRow, kChunks = D / 8, kRows = 1024 / kRow, kPieces = kTile / 1024, kN = D / 32, kM = D / 16;
    const uint8_t *K, *V;        // of the head
    int64_t pitch_k, pitch_v;    // bytes
    uint8_t* lds;                // K, V
    int last;                    // last key that may be read: it stands for those behind it, which are masked
    int lane;
    uint32_t row_at, col_at;
    __device__ __forceinline__ NarrowWave(const SelParams& p, const Item& it, uint8_t* lds_, int seen, int lane_) : lds(lds_), last(seen - 1), lane(lane_) {
        const int r = lane & 15, g = lane >> 4, cq = r & 3, row = 4 * g + (r >> 2);
        K = row_address(p.K, it.b, it.h, 0);
        V = row_address(p.V, it.b, it.h, 0);
        pitch_k = 2 * p.K.stride_n;
        pitch_v = 2 * p.V.stride_n;
        const uint32_t base = (uint32_t)(uintptr_t)(LDS_PTR(uint8_t))lds;
        row_at = base + r * kRow + ((tile_swizzle<D>(r) ^ g) << 4);
        col_at = base + row * kRow + (((cq >> 1) ^ tile_swizzle<D>(row)) << 4) + 8 * (cq & 1);
    }
    __device__ __forceinline__ void fetch(const uint8_t* head, int64_t pitch, int start, uint8_t* tile) const {
        const int first = min(start, last), left = last - first;
        const uint8_t* const base = head + first * pitch;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int row = k * kRows + lane / kChunks;
            load_lds(base, (uint32_t)min(row, left) * (uint32_t)pitch + (((lane % kChunks) ^ tile_swizzle<D>(row)) << 4), tile + k * 1024);
        }
    }
    // A operand, rows = keys 16 m + lane % 16 of K (tile 0) or V (1), dims 32 ks + 8 g .. + 7
    __device__ __forceinline__ frag8 rows(int tile, int m, int ks) const {
        return *(LDS_PTR(const frag8))(uintptr_t)((row_at ^ (ks << 6)) + tile * kTile + 16 * m * kRow);
    }
    // A operand, rows = dims 16 dt + lane % 16, contracted over the unit's keys
    __device__ __forceinline__ frag8 cols(int tile, int dt) const {   // (16 rows on the swizzle is the same)
        const uint32_t at = (col_at ^ (dt << 5)) + tile * kTile;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)at);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)(at + 16 * kRow));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    // Everything but the last tile's loads, or everything, has landed.  (Loads return in order; what was read from LDS is in registers too.)
    static __device__ __forceinline__ void wait_but_last() {
        __builtin_amdgcn_s_waitcnt(kPieces | 7 << 4);
        asm volatile("" ::: "memory");
    }
    // For every unit of this wave: take_k() and take_v() read what they need of K and V from LDS into registers; scores(first key) works
    // on the former, products(first key) on both.
    template <typename TK, typename S, typename TV, typename P>
    __device__ __forceinline__ void walk(const int32_t* units, int n_units, int wave, TK&& take_k, S&& scores, TV&& take_v, P&& products) const {
        if (wave >= n_units) return;
        int next = __builtin_amdgcn_readfirstlane(units[wave]);
        fetch(K, pitch_k, next, lds);
        fetch(V, pitch_v, next, lds + kTile);
        for (int i = wave; i < n_units; i += 4) {
            const int start = next;
            const bool more = i + 4 < n_units;
            next = __builtin_amdgcn_readfirstlane(units[min(i + 4, n_units - 1)]);
            wait_but_last();   // K has landed
            take_k();
            wait_but_last();   // and is in registers
            if (more) fetch(K, pitch_k, next, lds);
            scores(start);
            if (more) wait_but_last();   // V has landed
            else wave_wait();
            take_v();
            if (more) wait_but_last();
            else wave_wait();
            if (more) fetch(V, pitch_v, next, lds + kTile);
            products(start);
        }
    }
    // The waves' sums go through LDS: [wave][row][16-byte chunks of 4 dims, XORed with the row].  Then thread (row tid / 16) has D / 16
    // dims from (tid % 16) D / 16 on.
    static constexpr int kOwn = D / 16;
    static __device__ __forceinline__ void put(float* sums, int wave, int lane, const f32x4* acc) {
        const int r = lane & 15, g = lane >> 4;
#pragma unroll
        for (int dt = 0; dt < kM; ++dt)
            *(float4*)(sums + (wave * 16 + r) * D + 4 * ((4 * dt + g) ^ r)) = make_float4(acc[dt][0], acc[dt][1], acc[dt][2], acc[dt][3]);
    }
    static __device__ __forceinline__ void get(const float* sums, const float (&factor)[4], float (&x)[kOwn]) {
        const int r = threadIdx.x >> 4, sub = threadIdx.x & 15;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) x[i] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int u = 0; u < kOwn / 4; ++u) {
                const float4 v = *(const float4*)(sums + (w * 16 + r) * D + 4 * ((sub * (kOwn / 4) + u) ^ r));
                x[4 * u] = fmaf(factor[w], v.x, x[4 * u]);
                x[4 * u + 1] = fmaf(factor[w], v.y, x[4 * u + 1]);
                x[4 * u + 2] = fmaf(factor[w], v.z, x[4 * u + 2]);
                x[4 * u + 3] = fmaf(factor[w], v.w, x[4 * u + 3]);
            }
    }
    template <bool F16>
    static __device__ __forceinline__ void store(uint8_t* row, const float (&x)[kOwn], float factor) {
        uint8_t* const dst = row + 2 * kOwn * (threadIdx.x & 15);
#pragma unroll
        for (int u = 0; u < kOwn / 4; ++u) {
            uint2 v;
            v.x = Elem<F16>::pack(x[4 * u] * factor, x[4 * u + 1] * factor);
            v.y = Elem<F16>::pack(x[4 * u + 2] * factor, x[4 * u + 3] * factor);
            *(uint2*)(dst + 8 * u) = v;
        }
    }
};

// Rows from accumulators: a lane holds 4 consecutive dims at a time of its row (dims 32 db + 8 q + 4 half ..).  A wave turns its 32 rows
// through 4 KiB of LDS, 64 dims at a time, so that a store instruction covers 8 rows of 128 bytes.  row_of(i): address of row i of
// the 32, or null.  Only the wave itself uses `stage`.
template <bool F16, int D, typename F>
__device__ __forceinline__ void store_rows(uint8_t* stage, const f32x16* acc, float factor, int lane, F&& row_of) {
    using E = Elem<F16>;
#pragma unroll
    for (int pass = 0; pass < D / 64; ++pass) {
#pragma unroll
        for (int dbp = 0; dbp < 2; ++dbp)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x16& o = acc[2 * pass + dbp];
                uint2 v;
                v.x = E::pack(o[4 * q] * factor, o[4 * q + 1] * factor);
                v.y = E::pack(o[4 * q + 2] * factor, o[4 * q + 3] * factor);
                *(uint2*)(stage + (lane & 31) * 128 + 8 * (lane >> 5) + (((4 * dbp + q) ^ (lane & 7)) << 4)) = v;
            }
        __builtin_amdgcn_wave_barrier();   // (compiler: keep the reads below the writes above)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 8 * i + (lane >> 3);
            const uint4 x = *(const uint4*)(stage + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
            uint8_t* const to = row_of(r);
            if (to) *(uint4*)(to + pass * 128 + (lane & 7) * 16) = x;
        }
        __builtin_amdgcn_wave_barrier();   // (... and the next pass's writes below these reads)
    }
}

template <int D>
__device__ __forceinline__ void clear(f32x16 (&acc)[D / 32]) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[db][i] = 0.f;
}

}  // namespace grat
