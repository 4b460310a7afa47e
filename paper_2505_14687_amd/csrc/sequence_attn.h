// Attention over lists of key blocks, on the matrix cores of gfx950: what the forward and the gradient kernels share.
//
// The rows of a query group - q_group queries of each of the heads that share a K/V head, head by head - all walk the group's list, so every
// (row tile, key unit) product is a dense one; only the newest keys and the end of a sequence need a mask.  The products are the
// "transposed" ones of attn_mfma.h: with X the operand that streams through LDS and Y the one whose rows a wave owns (its 32
// columns of the instruction, in registers as B fragments), T = X Y^T leaves lane (c = lane % 32, half = lane / 32) with the 16 streamed
// rows 8 (r / 4) + 4 half + r % 4 of its own row c per 32, and that layout, packed to 16 bits, is the B operand of
// Z^T += X'^T T if the contraction index is enumerated in the same order.  X'^T fragments come out of row-major tiles
// through the LDS transpose read.
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

// ---- the walk over a list ------------------------------------------------------------------------
// K and V tiles of 64 keys (two units), double buffered.  NW waves fetch 1-KiB pieces; a wave's pieces lie in one unit.
template <int NW, int D>
struct KeyLoader {
    static constexpr int kPieces = 64 * D * 2 / 1024, LPW = kPieces / NW, kPerUnit = kPieces / 2, kRows = 1024 / (2 * D), kChunks = D / 8;
    static_assert(LPW >= 1 && kPerUnit % LPW == 0, "a wave's pieces lie in one unit");
    const uint8_t *K, *V;        // of the head
    int64_t pitch_k, pitch_v;    // bytes
    int last;                    // last key that may be read
    int my_unit, row[LPW], col[LPW];
    __device__ __forceinline__ KeyLoader(const SelParams& p, const Item& it, int seen, int wave, int lane) {
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
        const int left = last - start;
        const uint8_t* const base = head + start * pitch;
#pragma unroll
        for (int k = 0; k < LPW; ++k) load_lds(base, (uint32_t)min(row[k], left) * (uint32_t)pitch + col[k], tile + (wave * LPW + k) * 1024);
    }
    __device__ __forceinline__ void issue(int start, uint8_t* k_tile, uint8_t* v_tile, int wave) const {
        issue(K, pitch_k, start, k_tile, wave);
        issue(V, pitch_v, start, v_tile, wave);
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
