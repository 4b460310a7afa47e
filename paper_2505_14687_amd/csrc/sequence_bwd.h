// The gradient of attention over lists of key blocks.
//
// With P = exp(scale Q K^T - lse) on the listed keys that a row sees, D = sum dO O (row by row) and dS = P (dO V^T - D):
//   dV = P^T dO,  dQ = scale dS K,  dK = scale dS^T Q.
// dQ is the forward walk again: a group's rows against its list.  dK and dV belong to keys, so they walk the lists turned round: the
// groups that list a block.  Both form P and dS anew (7 products instead of 5, and no sum that depends on the order of
// atomics).  The lists are turned round through a bitmap [block][group], whose bits may be set in any order; a block's set bits are
// its groups in ascending order.  Blocks that many groups list (the first one: all of them) are cut into parts of about equal length,
// whose sums are added up in order.
//
// Steps: D and dQ | lists of every block, parts | dK, dV | joined parts.
//
// 16 384 tokens, 32 heads on 8, 16 blocks of 64 keys, bf16: dQ 420 us (6 d operations a pair, 950 TFLOP/s, the matrix pipe busy for 48 % of the cycles), lists 12,
// dK and dV 670 (8 d, 790 TFLOP/s, 40 %), join 28.  dQ is held back as the forward walk is; the walk over keys by its order - weights and dS of 32 rows are
// worked out while the wave issues no product - and by rows that are gathered through the L2, 3.9 GB, five of six from beyond it (with all of them in it a step
// takes 7 % less).
#pragma once
#include <type_traits>

#include "sequence_attn.h"

namespace grat {

// Half ends at 65 504, and below 2^-14 it loses bits; what is rounded to it for a product is taken times a power of two that the fp32 sum is
// divided by (bf16 has fp32's range):
//   P in dV's product   2^12, in the lse2 of the walk over keys: weights down to 2^-26 keep all bits
//   dS in dQ's          a row's own 2^row_bits, in the row's lse2, so that |dO| 2^row_bits is 2^9 to 2^10.  |dS| < |dO| |V| may still be too large
//                       where V is: an infinite dS leaves no element of the row's sums finite, and such a row is walked again with 2^kBitsBack less, which
//                       is enough for any V (|V| < 2^19.5 at head_dim 128)
//   dS in dK's          one power for all rows of a K/V head: the smallest that the rows took (a row that another one outweighs by 2^10 has weights down
//                       to 2^-14 in full), and one bit less: dS is formed there once more and may come out a little larger
constexpr int kWeightBits = 12, kRowBits = 10, kBitsBack = 16, kMostBits = 64;

// Exponent for a row whose dO has the sum of squares n2; a row of zeros (or NaN, infinities) has no say in the head's.
__device__ __forceinline__ int row_bits(float n2) { return kRowBits - ((__builtin_amdgcn_frexp_expf(n2) + 1) >> 1); }
__device__ __forceinline__ int head_say(float n2, int bits) { return n2 > 0.f && n2 < INFINITY ? bits : kMostBits; }
__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// ---- dK, dV ------------------------------------------------------------------------------------
// A workgroup owns 32 KW keys of one block, K and V of a wave's 32 keys in registers, and streams the Q and dO rows of
// the groups that list the block in tiles of 64 through LDS; two teams of KW waves take 32 rows of a tile each.
// What goes with a row - where it lies, lse, D, the keys it sees - is worked out by one wave, a tile ahead of the loads that need it, and
// passed on through LDS; lse and D go there straight from memory.
struct alignas(16) RowMeta {
    float lse2[64], delta[64];
    int32_t limit[64];
    const uint8_t* q[64];
    const uint8_t* d[64];
    int32_t masked;   // some row does not see all keys of the tile
};

template <int KW, bool F16, int D>
__global__ __launch_bounds__(KW * 128, KW) void grad_keys_kernel(SelParams p, GradParams g) {
    using E = Elem<F16>;
    constexpr int NW = 2 * KW, kTile = 64 * D * 2, kPieces = kTile / 1024, LPW = kPieces / NW, kRows = 1024 / (2 * D), kChunks = D / 8;
    __shared__ __attribute__((aligned(2 * kTile))) uint8_t lds[4][kTile];   // Q, Q, dO, dO
    __shared__ RowMeta meta[4];
    const SeqShape& s = p.s;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), half = lane >> 5;
    const int team = wave / KW, key_wave = wave % KW;

    // The XCDs walk the heads together, kChunk items at a time each: Q and dO of one or two K/V heads are in use at a time, which the memory-side
    // cache holds.
    constexpr int kChunk = 16;
    const int tiles = (int)g.fd_tiles.d, longs = g.counters[1], work = (longs + g.counters[4]) * tiles;
    const int turn = (int)blockIdx.x >> 3, item = ((turn / kChunk) * 8 + ((int)blockIdx.x & 7)) * kChunk + turn % kChunk;
    if (item >= work) return;
    uint32_t part_id, tile_in_block, b_, h_;
    fdivmod((uint32_t)item, g.fd_tiles, part_id, tile_in_block);
    if ((int)part_id >= longs) part_id = (uint32_t)(g.most_parts - 1 - ((int)part_id - longs));   // short parts: from the back
    const int4 part = g.parts[part_id];
    const uint32_t bh = (uint32_t)part.x / (uint32_t)s.n_blocks, block = (uint32_t)part.x - bh * (uint32_t)s.n_blocks;
    fdivmod(bh, p.fd_kv_heads, b_, h_);
    const int b = (int)b_, h = (int)h_;
    const int n_tiles = (part.w - part.z + 63) / 64;
    const int len = seq_len(s, b);
    const int64_t pos = seq_pos(s, b, len);

    const int tile_key0 = (int)block * s.block + (int)tile_in_block * (32 * KW), key = tile_key0 + key_wave * 32 + (lane & 31);
    f32x16 dk[D / 32], dv[D / 32];
    clear<D>(dk);
    clear<D>(dv);
    const int bits = F16 ? __builtin_amdgcn_readfirstlane(g.head_bits[bh]) : 0;
    const float grad_factor = ldexpf(1.f, bits - kWeightBits);   // (half: dS from the P that dV takes)
    if (n_tiles > 0 && tile_key0 < len) {
        frag8 kf[D / 16], vf[D / 16];
        {
            const int row = min(key, len - 1);
            const uint8_t *ks = row_address(p.K, b, h, row) + 16 * half, *vs = row_address(p.V, b, h, row) + 16 * half;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) kf[i] = *(const frag8*)(ks + 32 * i);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) vf[i] = *(const frag8*)(vs + 32 * i);
        }
        // -- rows of the walk
        const int32_t* const groups = g.groups + part.y;
        auto find_group = [&](int t) { return groups[fdiv((uint32_t)min(part.z + 64 * t + lane, part.w - 1), g.fd_rows)]; };
        auto put_rows = [&](int t, int group) {
            const int at = part.z + 64 * t + lane, in_list = min(at, part.w - 1);
            const GroupRow r(p, h, group, in_list - (int)(fdiv((uint32_t)in_list, g.fd_rows) * g.fd_rows.d));
            const bool there = r.there && at < part.w;
            RowMeta& m = meta[t & 3];
            m.q[lane] = row_address(p.Q, b, r.head, r.query);
            m.d[lane] = row_address(g.dO, b, r.head, r.query);
            const int limit = row_seen(s, len, pos, r.query);
            m.limit[lane] = limit;
            const bool cut = __builtin_amdgcn_ballot_w64(there && limit < tile_key0 + 32 * KW) != 0;
            if (lane == 0) m.masked = cut;
            // (rows that only fill a tile take the entry behind the last row's, which makes them weigh 0)
            const int64_t i = there ? ((int64_t)b * s.q_heads + r.head) * s.n_q + r.query : g.stats;
            load_lds_word((const uint8_t*)(g.lse2 + i), (uint8_t*)m.lse2);
            load_lds_word((const uint8_t*)(g.delta + i), (uint8_t*)m.delta);
        };
        const bool keeper = wave == NW - 1;
        int group_ahead = 0;
        if (keeper) {
            put_rows(0, find_group(0));
            put_rows(1, find_group(1));
            group_ahead = find_group(2);
        }
        tile_barrier();
        // A wave's pieces of a tile: rows kRows apart; the swizzle of piece k differs from that of piece 0 in bits that all lanes share.
        static_assert(kRows % 4 == 0, "");
        const int piece_row = wave * LPW * kRows + lane / kChunks, piece_col = (lane % kChunks) ^ tile_swizzle<D>(lane / kChunks);
        auto issue = [&](int t) {
            const RowMeta& m = meta[t & 3];
            uint8_t *qt = lds[t & 1], *dt = lds[2 + (t & 1)];
            int chunk = piece_col;
            asm volatile("" : "+v"(chunk));   // (columns are formed here: kept, they take two registers each)
            const uint8_t *q[LPW], *d[LPW];
#pragma unroll
            for (int k = 0; k < LPW; ++k) {   // (all read ahead of the first load: nothing moves across one)
                q[k] = m.q[piece_row + k * kRows];
                d[k] = m.d[piece_row + k * kRows];
            }
#pragma unroll
            for (int k = 0; k < LPW; ++k) {
                const int col = (chunk ^ tile_swizzle<D>((wave * LPW + k) * kRows)) << 4;
                load_lds(q[k] + col, qt + (wave * LPW + k) * 1024);
                load_lds(d[k] + col, dt + (wave * LPW + k) * 1024);
            }
        };
        TileReader<D> read(lane, lds[0], team);
        const float c = p.scale_log2;
        auto rows_block = [&](const RowMeta& m, bool masked) {
            const int row0 = 32 * team + 4 * half;   // of this lane in the tile
            // 4 products, each fragment read kAhead products ahead of its own: the sums of dK and dV, K and V leave 64 registers for
            // everything else, and the compiler, left to itself, reads further ahead than that allows.
            constexpr int kAhead = 2, kN = D / 16, kM = 2 * (D / 32);
            frag8 fr[2 * kN + 2 * kM];
            auto fetch = [&](int i) {
                if (i < kN) fr[i] = read.rows(0, 0, i);
                else if (i < 2 * kN) fr[i] = read.rows(1, 0, i - kN);
                else if (i < 2 * kN + kM) fr[i] = read.cols(1, 0, (i - 2 * kN) / (D / 32), (i - 2 * kN) % (D / 32));
                else if (i < 2 * kN + 2 * kM) fr[i] = read.cols(0, 0, (i - 2 * kN - kM) / (D / 32), (i - 2 * kN - kM) % (D / 32));
            };
            f32x16 S, T, zero;
#pragma unroll
            for (int i = 0; i < 16; ++i) zero[i] = 0.f;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) fetch(i);
#pragma unroll
            for (int i = 0; i < 2 * kN; ++i) {
                if (i + kAhead < 2 * kN) fetch(i + kAhead);
                if (i < kN) S = E::mfma(fr[i], kf[i], i == 0 ? zero : S);
                else T = E::mfma(fr[i], vf[i - kN], i == kN ? zero : T);
                __builtin_amdgcn_sched_barrier(0);
            }
            // (in place: S becomes P, T dS)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 l4 = *(const float4*)&m.lse2[row0 + 8 * q], d4 = *(const float4*)&m.delta[row0 + 8 * q];
                const float l[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    S[4 * q + i] = __builtin_amdgcn_exp2f(fmaf(S[4 * q + i], c, -l[i]));
                    T[4 * q + i] = (F16 ? S[4 * q + i] * grad_factor : S[4 * q + i]) * (T[4 * q + i] - dl[i]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key >= m.limit[row0 + 8 * (i >> 2) + (i & 3)]) S[i] = T[i] = 0.f;
            }
            uint32_t pw[8], dw[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) pw[i] = E::pack(S[2 * i], S[2 * i + 1]);
#pragma unroll
            for (int i = 0; i < 8; ++i) dw[i] = E::pack(T[2 * i], T[2 * i + 1]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) fetch(2 * kN + i);
#pragma unroll
            for (int i = 0; i < 2 * kM; ++i) {
                const int s2 = i % kM / (D / 32), db = i % (D / 32);
                const uint32_t* const x = i < kM ? pw + 4 * s2 : dw + 4 * s2;
                const frag8 w = __builtin_bit_cast(frag8, make_uint4(x[0], x[1], x[2], x[3]));
                fetch(2 * kN + i + kAhead);
                if (i < kM) dv[db] = E::mfma(fr[2 * kN + i], w, dv[db]);
                else dk[db] = E::mfma(fr[2 * kN + i], w, dk[db]);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        issue(0);
        for (int t = 0; t < n_tiles; ++t) {
            tile_barrier();
            if (t + 1 < n_tiles) issue(t + 1);
            if (keeper && t + 2 < n_tiles) {
                put_rows(t + 2, group_ahead);
                group_ahead = find_group(t + 3);   // (past the last row: the last row's again)
            }
            const RowMeta& m = meta[t & 3];
            rows_block(m, __builtin_amdgcn_readfirstlane(m.masked) != 0);
            read.flip();
        }
    }
    // Everyone is done with the tiles.  (The keeper's last loads have to land as well: LDS that is given back is somebody else's.)
    tile_barrier();

    // the second team's share, lane by lane: dK, then dV
    float* const mine = (float*)&lds[0][0] + key_wave * 64 * (D / 2) + lane;
    static_assert(KW * 64 * (D / 2) * 4 <= 2 * kTile, "one sum of the second team fits two tiles");
    auto add = [&](f32x16 (&acc)[D / 32]) {
        if (team == 1) {
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) mine[(db * 16 + i) * 64] = acc[db][i];
        }
        __syncthreads();
        if (team == 0) {
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[db][i] += mine[(db * 16 + i) * 64];
        }
        __syncthreads();
    };
    add(dk);
    add(dv);
    if (team == 1) return;
    const float dk_factor = F16 ? ldexpf(p.scale, -bits) : p.scale, dv_factor = F16 ? ldexpf(1.f, -kWeightBits) : 1.f;
    const int slot = g.part_slot[part_id];
    if (slot >= 0) {   // parts are joined by grad_join_kernel
        float* const dst = g.slots + (((int64_t)slot * tiles + tile_in_block) * 2 * (32 * KW) + key_wave * 32 + (lane & 31)) * D + 4 * half;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float* const to = dst + 32 * db + 8 * q;
                *(float4*)to = make_float4(dk[db][4 * q], dk[db][4 * q + 1], dk[db][4 * q + 2], dk[db][4 * q + 3]);
                *(float4*)(to + 32 * KW * D) = make_float4(dv[db][4 * q], dv[db][4 * q + 1], dv[db][4 * q + 2], dv[db][4 * q + 3]);
            }
        return;
    }
    uint8_t* const stage = &lds[0][0] + key_wave * 4096;
    auto row_of = [&](const SeqTensor& t, int i) -> uint8_t* {
        const int k = tile_key0 + key_wave * 32 + i;
        return k < s.n_k ? (uint8_t*)row_address(t, b, h, k) : nullptr;
    };
    store_rows<F16, D>(stage, dk, dk_factor, lane, [&](int i) { return row_of(g.dK, i); });
    store_rows<F16, D>(stage, dv, dv_factor, lane, [&](int i) { return row_of(g.dV, i); });
}

// dK and dV of the blocks that were cut into parts: a thread adds up 4 numbers, kJoinShare workgroups share a key tile.
constexpr int kJoinShare = 8;

template <bool F16, int D>
__global__ __launch_bounds__(256) void grad_join_kernel(SelParams p, GradParams g, int tile_keys) {
    const SeqShape& s = p.s;
    uint32_t at, tile;
    fdivmod(blockIdx.z * gridDim.y + blockIdx.y, g.fd_tiles, at, tile);
    if ((int)at >= g.counters[3]) return;
    const int4 join = g.joins[at];   // block, first slot, parts
    const int tiles = (int)g.fd_tiles.d;
    const uint32_t bh = (uint32_t)join.x / (uint32_t)s.n_blocks, j = (uint32_t)join.x - bh * (uint32_t)s.n_blocks;
    const int b = (int)fdiv(bh, p.fd_kv_heads), h = (int)bh - b * s.kv_heads;
    const int64_t pitch = (int64_t)tiles * 2 * tile_keys * D;   // of a slot
    const float* const src = g.slots + join.y * pitch + (int64_t)tile * 2 * tile_keys * D;
    for (int i = (int)blockIdx.x * 256 + threadIdx.x; i < 2 * tile_keys * (D / 4); i += 256 * kJoinShare) {
        const int which = i / (tile_keys * (D / 4)), row = i / (D / 4) % tile_keys, c = i % (D / 4);
        const int key = (int)j * s.block + (int)tile * tile_keys + row;
        if (key >= s.n_k) continue;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int k = 0; k < join.z; ++k) {
            const float4 v = *(const float4*)(src + k * pitch + 4 * (int64_t)i);
            sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
        }
        const float f = which == 0 ? (F16 ? ldexpf(p.scale, -g.head_bits[bh]) : p.scale) : F16 ? ldexpf(1.f, -kWeightBits) : 1.f;
        uint2 v;
        v.x = Elem<F16>::pack(sum.x * f, sum.y * f);
        v.y = Elem<F16>::pack(sum.z * f, sum.w * f);
        *(uint2*)((uint8_t*)row_address(which == 0 ? g.dK : g.dV, b, h, key) + 8 * c) = v;
    }
}

// ---- dQ ----------------------------------------------------------------------------------------
// The forward walk with dO beside Q in registers: S^T = K Q^T, dP^T = V dO^T, and dQ^T += K^T dS^T with K read both ways from its tile.
// Lists of at most this many units are walked twice, for an exact D (see below).  1 024 tokens in groups of 64 x 4 heads, bf16, head_dim 128; a training step without and
// with the first walk: 4 units 45 and 49 us, 8 53 and 60, 12 60 and 71, 16 65 and 80, 32 82 and 111.  The error of dQ without it, in plain forms' (with it 1.43
// throughout): scores of deviation 1 1.47, 4 2.5, 8 3.7 up to 12 units; 1.48, 2.3, 3.5 at 16 and 32.
// (With what is left over taken into D for the walk over keys, dK and dV are at 1.4 either way.)
constexpr int kFewUnits = 12;

// For the launches that follow: what they count, and what rows that only fill a tile take.
__device__ __forceinline__ void start_lists(const GradParams& g) {
    if (blockIdx.x == 0 && threadIdx.x < 5) {
        g.counters[threadIdx.x] = 0;
        g.delta[g.stats] = 0.f;
        g.lse2[g.stats] = INFINITY;
    }
}

template <int RW, int TEAMS, bool F16, int D>
__global__ __launch_bounds__(RW * TEAMS * 64, RW * TEAMS == 2 ? 1 : 2) void grad_queries_kernel(SelParams p, GradParams g) {
    using E = Elem<F16>;
    constexpr int NW = RW * TEAMS, kTile = 64 * D * 2;
    __shared__ __attribute__((aligned(2 * kTile))) uint8_t lds[4][kTile];   // K, K, V, V
    __shared__ int32_t s_n;
    extern __shared__ int32_t s_units[];
    const Item it(p);
    start_lists(g);
    if (it.idle(p)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int team = TEAMS == 1 ? 0 : wave / RW, row_wave = wave % RW, half = lane >> 5;
    const SeqShape& s = p.s;
    const GroupRow row(p, it.h, it.g, (it.tile * RW + row_wave) * 32 + (lane & 31));
    const uint8_t* const q_src = row_address(p.Q, it.b, row.head, row.query) + 16 * half;
    const uint8_t* const d_src = row_address(g.dO, it.b, row.head, row.query) + 16 * half;
    frag8 qf[D / 16], df[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *(const frag8*)(q_src + 32 * ks);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) df[ks] = *(const frag8*)(d_src + 32 * ks);
    // D, and lse in base 2 (a row that attends nothing weighs 0); the walk over the keys takes both from memory
    const int64_t stat = ((int64_t)it.b * s.q_heads + row.head) * s.n_q + row.query;
    const float lse = p.lse[stat];
    float lse2 = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f, delta = 0.f, n2 = 0.f;
    {
        typedef typename Vec16<std::conditional_t<F16, _Float16, __bf16>>::type vec;
        const uint8_t* const o_src = row_address(p.O, it.b, row.head, row.query) + 16 * half;
        vec o[D / 16];
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) o[ks] = *(const vec*)(o_src + 32 * ks);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            const vec d = __builtin_bit_cast(vec, df[ks]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                delta = fmaf((float)o[ks][e], (float)d[e], delta);
                if constexpr (F16) n2 = fmaf((float)d[e], (float)d[e], n2);
            }
        }
        delta = sum_across_halves(delta);
    }
    // half: the exponent of this lane's row (in lse2 as well), and what counts for the head's; kept in LDS for want of registers
    __shared__ int32_t s_bits[F16 ? 2 : 1][F16 ? NW * 64 : 1];
    int32_t &bits = s_bits[0][F16 ? threadIdx.x : 0], &say = s_bits[F16][F16 ? threadIdx.x : 0];
    if constexpr (F16) {
        n2 = sum_across_halves(n2);
        const int mine = row_bits(n2);
        lse2 -= (float)mine;
        bits = mine;
        say = head_say(n2, mine);
    }
    auto unscaled = [&](float x) { return F16 ? ldexpf(x, -bits) : x; };
    const int len = seq_len(s, it.b);
    const int64_t pos = seq_pos(s, it.b, len);
    const int seen = group_seen(s, len, pos, it.g);
    const int limit = row.there ? row_seen(s, len, pos, row.query) : 0;
    int least = row.there ? limit : 0x7fffffff, most = limit;
#pragma unroll
    for (int m = 1; m < 32; m *= 2) {
        least = min(least, __shfl_xor(least, m));
        most = max(most, __shfl_xor(most, m));
    }
    least = __builtin_amdgcn_readfirstlane(least);
    most = __builtin_amdgcn_readfirstlane(most);
    const int n_units = seen > 0 ? list_units(p, it.list(p), seen, s_units, &s_n) : 0;
    const int n_tiles = (n_units + 1) / 2;
    f32x16 dq[D / 32];
    clear<D>(dq);
    const float c = p.scale_log2;
    const KeyLoader<NW, D> load(p, it, seen, wave, lane);
    TileReader<D> read(lane, lds[0], team);
    auto unit_start = [&](int i) { return i < n_units ? __builtin_amdgcn_readfirstlane(s_units[i]) : kNoUnit; };
    auto unit_load = [&](int i) { return __builtin_amdgcn_readfirstlane(s_units[min(i, n_units - 1)]); };   // (as in the forward walk)
    float sum = 0.f;   // over this lane's keys: of P dP while D is being formed, then of dS
    auto block = [&](auto form_d, int hb, int start) {
        constexpr bool kFormD = decltype(form_d)::value;
        if (start >= most) return;
        f32x16 S, T;
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = T[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) S = E::mfma(read.rows(0, hb, ks), qf[ks], S);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) T = E::mfma(read.rows(1, hb, ks), df[ks], T);
        const bool masked = start + kUnit > least;
        uint32_t dw[8];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            float d0 = __builtin_amdgcn_exp2f(fmaf(S[i], c, -lse2)) * (T[i] - delta);
            float d1 = __builtin_amdgcn_exp2f(fmaf(S[i + 1], c, -lse2)) * (T[i + 1] - delta);
            if (masked) {
                const int key = start + 8 * (i >> 2) + 4 * half + (i & 3);
                if (key >= limit) d0 = 0.f;
                if (key + 1 >= limit) d1 = 0.f;
            }
            sum += d0 + d1;
            if constexpr (!kFormD) dw[i >> 1] = E::pack(d0, d1);
        }
        if constexpr (!kFormD) {
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2) {
                const frag8 w = __builtin_bit_cast(frag8, make_uint4(dw[4 * s2], dw[4 * s2 + 1], dw[4 * s2 + 2], dw[4 * s2 + 3]));
#pragma unroll
                for (int db = 0; db < D / 32; ++db) dq[db] = E::mfma(read.cols(0, hb, s2, db), w, dq[db]);
            }
        }
    };
    // A tile of two units as one stream of instructions.  Every product is followed by its share of the vector work: P of a unit behind its
    // dO V^T, its dS behind the next unit's scores (unit 0) or unit 0's dS K (unit 1); and by the read of the fragment for the
    // product kAhead later.  Keys that a row does not see get their -infinity as what their scores are added to.
    auto tile = [&](int start0, int start1) {
        constexpr int kAhead = 2, kN = D / 16, kM = 2 * (D / 32), kAll = 4 * kN + 2 * kM;
        if (start0 >= most && start1 >= most) return;   // nobody in this wave sees the units
        frag8 fr[kAll];
        auto fetch = [&](int i) {   // S T of unit 0, S T of unit 1, dS K of both
            if (i < 4 * kN) fr[i] = read.rows(i / kN % 2, i / (2 * kN), i % kN);
            else fr[i] = read.cols(0, (i - 4 * kN) / kM, (i - 4 * kN) % kM / (D / 32), (i - 4 * kN) % (D / 32));
        };
        f32x16 S[2], T[2], zero;
        uint32_t dw[2][8];
#pragma unroll
        for (int i = 0; i < 16; ++i) S[0][i] = S[1][i] = zero[i] = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int start = u == 0 ? start0 : start1;
            if (start + kUnit > least) {
#pragma unroll
                for (int i = 0; i < 16; ++i) S[u][i] = start + 8 * (i >> 2) + 4 * half + (i & 3) < limit ? 0.f : -INFINITY;
            }
        }
        auto weigh = [&](int u, int j) {   // pair j
            S[u][2 * j] = __builtin_amdgcn_exp2f(fmaf(S[u][2 * j], c, -lse2));
            S[u][2 * j + 1] = __builtin_amdgcn_exp2f(fmaf(S[u][2 * j + 1], c, -lse2));
        };
        auto grad = [&](int u, int j) {
            const float d0 = S[u][2 * j] * (T[u][2 * j] - delta), d1 = S[u][2 * j + 1] * (T[u][2 * j + 1] - delta);
            sum += d0 + d1;
            dw[u][j] = E::pack(d0, d1);
            asm volatile("" : "+v"(dw[u][j]));   // (keeps the conversion here: its first use is later)
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fetch(i);
        auto products = [&](auto u_c, auto what_c, auto&& work) {   // what: 0 scores, 1 dO V^T, 2 dS K; work(j): vector work of pair j
            constexpr int u = decltype(u_c)::value, what = decltype(what_c)::value;
            constexpr int first = what == 2 ? 4 * kN + u * kM : (2 * u + what) * kN, n = what == 2 ? kM : kN;
#pragma unroll
            for (int k = 0; k < n; ++k) {
                const int i = first + k;
                if (i + kAhead < kAll) fetch(i + kAhead);
                if constexpr (what == 0) {
                    S[u] = E::mfma(fr[i], qf[k], S[u]);
                } else if constexpr (what == 1) {
                    T[u] = E::mfma(fr[i], df[k], k == 0 ? zero : T[u]);
                } else {
                    const uint32_t* const x = &dw[u][4 * (k / (D / 32))];
                    dq[k % (D / 32)] = E::mfma(fr[i], __builtin_bit_cast(frag8, make_uint4(x[0], x[1], x[2], x[3])), dq[k % (D / 32)]);
                }
#pragma unroll
                for (int j = 8 * k / n; j < 8 * (k + 1) / n; ++j) work(j);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        using std::integral_constant;
        constexpr integral_constant<int, 0> c0{};
        constexpr integral_constant<int, 1> c1{};
        constexpr integral_constant<int, 2> c2{};
        products(c0, c0, [](int) {});
        products(c0, c1, [&](int j) { weigh(0, j); });
        products(c1, c0, [&](int j) { grad(0, j); });
        products(c1, c1, [&](int j) { weigh(1, j); });
        products(c0, c2, [&](int j) { grad(1, j); });
        products(c1, c2, [](int) {});
    };
    auto walk = [&](auto form_d) {
        load.issue(unit_load(load.my_unit), lds[0], lds[2], wave);
        for (int t = 0; t < n_tiles; ++t) {
            const int next = unit_load(2 * t + 2 + load.my_unit), start0 = unit_start(2 * t + (TEAMS == 1 ? 0 : team));
            const int start1 = TEAMS == 1 ? unit_start(2 * t + 1) : kNoUnit;
            tile_barrier();
            if (t + 1 < n_tiles) load.issue(next, lds[(t + 1) & 1], lds[2 + ((t + 1) & 1)], wave);
            if constexpr (TEAMS == 2) {
                block(form_d, 0, start0);
            } else if constexpr (decltype(form_d)::value) {
                block(form_d, 0, start0);
                block(form_d, 1, start1);
            } else {
                tile(start0, start1);
            }
            read.flip();
        }
        if (n_tiles & 1) read.flip();   // (a walk begins in the first tile)
        __syncthreads();                // everyone is done with the tiles
    };
    // over all keys of this lane's row
    __shared__ float s_sum[NW][32];
    auto over_row = [&](float mine) {
        float all = sum_across_halves(mine);
        if constexpr (TEAMS == 2) {
            if (half == 0) s_sum[wave][lane] = all;
            __syncthreads();
            all = s_sum[row_wave][lane & 31] + s_sum[RW + row_wave][lane & 31];
            __syncthreads();
        }
        return all;
    };
    // dS has to add up to 0 over a row's keys.  With D taken from the rounded O it does not, by sum dO (O's error), which is small
    // beside dO V^T where many keys are averaged into O, and as large as the rounding of dS where few are: short lists are walked a
    // first time for what is missing.  What is left over is added to D for the walk over the keys.
    if (n_tiles > 0) {
        if (n_units <= kFewUnits) {
            walk(std::true_type{});
            delta += unscaled(over_row(sum));
            sum = 0.f;
        }
        walk(std::false_type{});
        if constexpr (F16) {
            const bool over = over_row(finite(dq[0][0]) ? 0.f : 1.f) > 0.f;
            if (__syncthreads_or(over)) {
                if (over) {
                    bits -= kBitsBack;
                    say -= kBitsBack;
                    lse2 += (float)kBitsBack;
                }
                clear<D>(dq);
                sum = 0.f;
                walk(std::false_type{});
            }
        }
    }
    sum = unscaled(over_row(sum));
    if constexpr (F16) {
        int least = limit > 0 ? say : kMostBits;
#pragma unroll
        for (int m = 1; m < 32; m *= 2) least = min(least, __shfl_xor(least, m));
        if (team == 0 && lane == 0) g.row_bits[it.item * RW + row_wave] = least;
    }
    if constexpr (TEAMS == 2) {
        float* const mine = (float*)&lds[0][0] + row_wave * 64 * (D / 2) + lane;
        if (team == 1) {
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) mine[(db * 16 + i) * 64] = dq[db][i];
        }
        __syncthreads();
        if (team == 1) return;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) dq[db][i] += mine[(db * 16 + i) * 64];
    }
    if (half == 0 && row.there) {
        g.delta[stat] = delta + sum;
        g.lse2[stat] = F16 ? lse2 + (float)(bits - kWeightBits) : lse2;
    }
    uint8_t* const stage = &lds[0][0] + (TEAMS == 2 ? 2 * kTile : 0) + row_wave * 4096;   // (two teams: behind what team 0 still reads)
    store_rows<F16, D>(stage, dq, unscaled(p.scale), lane, [&](int i) -> uint8_t* {
        const GroupRow to(p, it.h, it.g, (it.tile * RW + row_wave) * 32 + i);
        return to.there ? (uint8_t*)row_address(g.dQ, it.b, to.head, to.query) : nullptr;
    });
}

// ... of groups of at most 16 rows.
template <bool F16, int D>
__global__ __launch_bounds__(256, 2) void grad_queries_narrow_kernel(SelParams p, GradParams g) {
    using E = Elem<F16>;
    using W = NarrowWave<D>;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[4][2 * W::kTile];   // K, V of every wave
    __shared__ float s_sum[2][4][16];
    __shared__ int32_t s_n, s_bits[16];
    extern __shared__ int32_t s_units[];
    const Item it(p);
    start_lists(g);
    if (it.idle(p)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), r = lane & 15, quad = lane >> 4;
    const SeqShape& s = p.s;
    const GroupRow row(p, it.h, it.g, it.tile * 16 + r);
    const uint8_t* const q_src = row_address(p.Q, it.b, row.head, row.query) + 16 * quad;
    const uint8_t* const d_src = row_address(g.dO, it.b, row.head, row.query) + 16 * quad;
    const uint8_t* const o_src = row_address(p.O, it.b, row.head, row.query) + 16 * quad;
    typedef typename Vec16<std::conditional_t<F16, _Float16, __bf16>>::type vec;
    frag8 qf[W::kN], df[W::kN];
    vec o[W::kN];
#pragma unroll
    for (int ks = 0; ks < W::kN; ++ks) {
        qf[ks] = *(const frag8*)(q_src + 64 * ks);
        df[ks] = *(const frag8*)(d_src + 64 * ks);
        o[ks] = *(const vec*)(o_src + 64 * ks);
    }
    const int64_t stat = ((int64_t)it.b * s.q_heads + row.head) * s.n_q + row.query;
    const float lse = p.lse[stat];
    float lse2 = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f, delta = 0.f, n2 = 0.f;
    auto over_quads = [](float x) {
        x += __shfl_xor(x, 16);
        return x + __shfl_xor(x, 32);
    };
#pragma unroll
    for (int ks = 0; ks < W::kN; ++ks) {
        const vec d = __builtin_bit_cast(vec, df[ks]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            delta = fmaf((float)o[ks][e], (float)d[e], delta);
            if constexpr (F16) n2 = fmaf((float)d[e], (float)d[e], n2);
        }
    }
    delta = over_quads(delta);
    int bits = 0;   // (as in grad_queries_kernel)
    if constexpr (F16) {
        n2 = over_quads(n2);
        bits = row_bits(n2);
        lse2 -= (float)bits;
    }
    const int len = seq_len(s, it.b);
    const int64_t pos = seq_pos(s, it.b, len);
    const int seen = group_seen(s, len, pos, it.g);
    const int limit = row.there ? row_seen(s, len, pos, row.query) : 0;
    int least = row.there ? limit : 0x7fffffff;
#pragma unroll
    for (int m = 1; m < 16; m *= 2) least = min(least, __shfl_xor(least, m));
    least = __builtin_amdgcn_readfirstlane(least);
    const int n_units = seen > 0 ? list_units(p, it.list(p), seen, s_units, &s_n) : 0;

    f32x4 dq[W::kM];
#pragma unroll
    for (int i = 0; i < W::kM; ++i) dq[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float c = p.scale_log2;
    float sum = 0.f;   // over this lane's keys: of P dP while D is being formed, then of dS
    const W w(p, it, lds[wave], seen, lane);
    frag8 kf[2][W::kN], vf[2][W::kN], kt[W::kM];   // K, V by rows, K by columns
    auto walk = [&](auto form_d) {
        constexpr bool kFormD = decltype(form_d)::value;
        f32x4 S[2];
        auto take_k = [&]() {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int ks = 0; ks < W::kN; ++ks) kf[m][ks] = w.rows(0, m, ks);
            if constexpr (!kFormD) {
#pragma unroll
                for (int dt = 0; dt < W::kM; ++dt) kt[dt] = w.cols(0, dt);
            }
        };
        auto take_v = [&]() {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int ks = 0; ks < W::kN; ++ks) vf[m][ks] = w.rows(1, m, ks);
        };
        auto scores = [&](int) {
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                S[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < W::kN; ++ks) S[m] = E::mfma16(kf[m][ks], qf[ks], S[m]);
            }
        };
        w.walk(s_units, n_units, wave, take_k, scores, take_v, [&](int start) {
            f32x4 T[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                T[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < W::kN; ++ks) T[m] = E::mfma16(vf[m][ks], df[ks], T[m]);
            }
            const bool masked = start + kUnit > least;
            uint32_t dw[4];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const f32x4 &x = S[i >> 2], &t = T[i >> 2];
                float d0 = __builtin_amdgcn_exp2f(fmaf(x[i & 3], c, -lse2)) * (t[i & 3] - delta);
                float d1 = __builtin_amdgcn_exp2f(fmaf(x[(i & 3) + 1], c, -lse2)) * (t[(i & 3) + 1] - delta);
                if (masked) {
                    const int key = start + 16 * (i >> 2) + 4 * quad + (i & 3);
                    if (key >= limit) d0 = 0.f;
                    if (key + 1 >= limit) d1 = 0.f;
                }
                sum += d0 + d1;
                if constexpr (!kFormD) dw[i >> 1] = E::pack(d0, d1);
            }
            if constexpr (!kFormD) {
                const frag8 x = __builtin_bit_cast(frag8, make_uint4(dw[0], dw[1], dw[2], dw[3]));
#pragma unroll
                for (int dt = 0; dt < W::kM; ++dt) dq[dt] = E::mfma16(kt[dt], x, dq[dt]);
            }
        });
    };
    int turn = 0;
    auto over_row = [&](float mine) {   // over all keys of row `r`
        const float all = over_quads(mine);
        turn ^= 1;   // (a barrier lies between what is read here and the next but one's writes)
        if (quad == 0) s_sum[turn][wave][r] = all;
        __syncthreads();
        return s_sum[turn][0][r] + s_sum[turn][1][r] + s_sum[turn][2][r] + s_sum[turn][3][r];
    };
    if (n_units > 0) {
        if (n_units <= kFewUnits) {   // short lists: a first walk for the exact D
            walk(std::true_type{});
            delta += ldexpf(over_row(sum), -bits);
            sum = 0.f;
        }
#pragma unroll 1
        for (bool again = false;; again = true) {
            walk(std::false_type{});
            if (!F16 || again) break;
            const bool over = over_row(finite(dq[0][0]) ? 0.f : 1.f) > 0.f;   // (the same in all four waves)
            if (__builtin_amdgcn_ballot_w64(over) == 0) break;
            if (over) {
                bits -= kBitsBack;
                lse2 += (float)kBitsBack;
            }
#pragma unroll
            for (int i = 0; i < W::kM; ++i) dq[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            sum = 0.f;
        }
    }
    const float left = ldexpf(over_row(sum), -bits);   // (its barrier: everyone is done with the tiles)
    if constexpr (F16) {
        int say = limit > 0 ? head_say(n2, bits) : kMostBits;
#pragma unroll
        for (int m = 1; m < 16; m *= 2) say = min(say, __shfl_xor(say, m));
        if (threadIdx.x == 0) g.row_bits[it.item] = say;
    }
    if (wave == 0 && quad == 0 && row.there) {
        g.delta[stat] = delta + left;
        g.lse2[stat] = F16 ? lse2 + (float)(bits - kWeightBits) : lse2;
    }
    float* const sums = (float*)&lds[0][0];
    static_assert(4 * 16 * D * 4 <= (int)sizeof(lds), "the results fit the tiles");
    W::put(sums, wave, lane, dq);
    if (threadIdx.x < 16) s_bits[threadIdx.x] = bits;
    __syncthreads();
    float x[W::kOwn];
    const float ones[4] = {1.f, 1.f, 1.f, 1.f};
    W::get(sums, ones, x);
    const GroupRow to(p, it.h, it.g, it.tile * 16 + (int)(threadIdx.x >> 4));
    const float factor = F16 ? ldexpf(p.scale, -s_bits[threadIdx.x >> 4]) : p.scale;
    if (to.there) W::template store<F16>((uint8_t*)row_address(g.dQ, it.b, to.head, to.query), x, factor);
}

template <int KW, bool F16, int D>
inline void launch_grad_keys(const SelParams& p, const GradParams& g, hipStream_t stream) {
    const int64_t items = (int64_t)g.most_parts * g.fd_tiles.d;
    hipLaunchKernelGGL((grad_keys_kernel<KW, F16, D>), dim3((unsigned)((items + 127) / 128 * 128)), dim3(KW * 128), 0, stream, p, g);
    if (g.most_joins > 0) {   // workgroups that share a key tile run beside each other (30 us for train_long's; 33 the other way round)
        const unsigned n = g.most_joins * g.fd_tiles.d, rows = n < 32768u ? n : 32768u;
        hipLaunchKernelGGL((grad_join_kernel<F16, D>), dim3(kJoinShare, rows, (n + rows - 1) / rows), dim3(256), 0, stream, p, g, 32 * KW);
    }
}
template <int RW, int TEAMS, bool F16, int D>
inline void launch_grad_queries(const SelParams& p, const GradParams& g, hipStream_t stream) {
    const size_t dyn = sizeof(int32_t) * ((size_t)p.max_blocks * p.fd_units.d + 1);
    hipLaunchKernelGGL((grad_queries_kernel<RW, TEAMS, F16, D>), dim3(8 * p.per_xcd), dim3(RW * TEAMS * 64), dyn, stream, p, g);
}

// tile_rows: 128, 64, 32 or 16; key tiles of 64 or 32 keys
template <bool F16, int D>
inline hipError_t launch_bwd(const SelParams& p, const GradParams& g, int tile_rows, int tile_keys, hipStream_t stream) {
    if (tile_rows == 128) launch_grad_queries<4, 1, F16, D>(p, g, stream);
    else if (tile_rows == 64) launch_grad_queries<2, 2, F16, D>(p, g, stream);
    else if (tile_rows == 32) launch_grad_queries<1, 2, F16, D>(p, g, stream);
    else
        hipLaunchKernelGGL((grad_queries_narrow_kernel<F16, D>), dim3(8 * p.per_xcd), dim3(256), sizeof(int32_t) * ((size_t)p.max_blocks * p.fd_units.d + 1),
                           stream, p, g);
    launch_grad_lists(p, g, stream);
    if (tile_keys == 64) launch_grad_keys<2, F16, D>(p, g, stream);
    else launch_grad_keys<1, F16, D>(p, g, stream);
    return hipGetLastError();
}

}  // namespace grat
