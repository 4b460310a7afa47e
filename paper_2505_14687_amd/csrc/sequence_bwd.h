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
// Steps: bits and D | lists of every block, parts | dK, dV | joined parts | dQ.
#pragma once
#include <type_traits>

#include "sequence_attn.h"

namespace grat {

// D of every row, and the scratch memory that has to be 0 (by a kernel: recorded into graphs like any other launch).
template <bool F16, int D>
__global__ __launch_bounds__(256) void grad_delta_kernel(SelParams p, GradParams g, int64_t rows, FastDiv fd_n, FastDiv fd_h) {
    typedef typename Vec16<std::conditional_t<F16, _Float16, __bf16>>::type vec;
    constexpr int L = D / 8;
    const int64_t zeros = (int64_t)g.blocks * g.words;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < zeros; i += (int64_t)gridDim.x * 256) g.bits[i] = 0;
    if (blockIdx.x == 0 && threadIdx.x < 3) g.counters[threadIdx.x] = 0;
    const int64_t at = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    if (at >= rows) return;
    uint32_t bh, n, b, h;
    fdivmod((uint32_t)at, fd_n, bh, n);
    fdivmod(bh, fd_h, b, h);
    const int c = threadIdx.x % L;
    const vec x = *(const vec*)(row_address(g.dO, (int)b, (int)h, (int)n) + 16 * c), y = *(const vec*)(row_address(p.O, (int)b, (int)h, (int)n) + 16 * c);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fmaf((float)x[e], (float)y[e], sum);
#pragma unroll
    for (int m = 1; m < L; m *= 2) sum += __shfl_xor(sum, m);
    if (c == 0) g.delta[at] = sum;
}

// ---- dK, dV ------------------------------------------------------------------------------------
// A workgroup owns 32 KW keys of one block, K and V of a wave's 32 keys in registers, and streams the Q and dO rows of
// the groups that list the block in tiles of 64 through LDS (TEAMS == 2: a team takes 32 rows of a tile each).
// What goes with a row - where it lies, lse, D, the keys it sees - is worked out by one wave, three tiles ahead for the loads
// that depend on each other, and passed on through LDS.
struct alignas(16) RowMeta {
    const uint8_t* q[64];
    const uint8_t* d[64];
    float lse2[64], delta[64];
    int32_t limit[64];
    int32_t least;   // of the 64 limits
};

template <int KW, int TEAMS, bool F16, int D>
__global__ __launch_bounds__(KW * TEAMS * 64, KW * TEAMS == 2 ? 1 : 2) void grad_keys_kernel(SelParams p, GradParams g) {
    using E = Elem<F16>;
    constexpr int NW = KW * TEAMS, kTile = 64 * D * 2, kPieces = kTile / 1024, LPW = kPieces / NW, kRows = 1024 / (2 * D), kChunks = D / 8;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[4][kTile];   // Q, Q, dO, dO
    __shared__ RowMeta meta[4];
    const SeqShape& s = p.s;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), half = lane >> 5;
    const int team = TEAMS == 1 ? 0 : wave / KW, key_wave = wave % KW;

    const int tiles = (int)g.fd_tiles.d, work = g.counters[1] * tiles, per_xcd = (work + 7) / 8;
    const int item = ((int)blockIdx.x & 7) * per_xcd + ((int)blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || item >= work) return;
    uint32_t part_id, tile_in_block, b_, h_;
    fdivmod((uint32_t)item, g.fd_tiles, part_id, tile_in_block);
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
        // -- rows: group of row `at` of the walk | its address, limit, lse, D | all of that in LDS
        const int32_t* const groups = g.groups + part.y;
        auto row_at = [&](int t) { return part.z + 64 * t + lane; };
        auto find_group = [&](int t) { return groups[fdiv((uint32_t)min(row_at(t), part.w - 1), g.fd_rows)]; };
        struct Row {
            const uint8_t *q, *d;
            float lse, delta;
            int limit;
        };
        auto find_row = [&](int t, int group) {
            const int at = min(row_at(t), part.w - 1);
            const GroupRow r(p, h, group, at - (int)(fdiv((uint32_t)at, g.fd_rows) * g.fd_rows.d));
            const bool there = r.there && row_at(t) < part.w;
            const int64_t i = ((int64_t)b * s.q_heads + r.head) * s.n_q + r.query;
            Row x;
            x.q = row_address(p.Q, b, r.head, r.query);
            x.d = row_address(g.dO, b, r.head, r.query);
            x.lse = p.lse[i];
            x.delta = g.delta[i];
            x.limit = there ? row_seen(s, len, pos, r.query) : -1;
            return x;
        };
        auto put_row = [&](int t, const Row& x) {
            RowMeta& m = meta[t & 3];
            m.q[lane] = x.q;
            m.d[lane] = x.d;
            // (rows that attend nothing, and rows that only fill a tile, weigh 0)
            m.lse2[lane] = x.limit < 0 || x.lse == -INFINITY ? INFINITY : x.lse * 1.4426950408889634f;
            m.delta[lane] = x.delta;
            m.limit[lane] = max(x.limit, 0);
            int least = x.limit < 0 ? 0x7fffffff : x.limit;
#pragma unroll
            for (int k = 1; k < 64; k *= 2) least = min(least, __shfl_xor(least, k));
            if (lane == 0) m.least = least;
        };
        const bool keeper = wave == NW - 1;
        Row ahead{};
        int group_ahead = 0;
        if (keeper) {
            put_row(0, find_row(0, find_group(0)));
            put_row(1, find_row(1, find_group(1)));
            ahead = find_row(2, find_group(2));
            group_ahead = find_group(3);
        }
        __syncthreads();
        int piece_row[LPW], col[LPW];
#pragma unroll
        for (int k = 0; k < LPW; ++k) {
            piece_row[k] = (wave * LPW + k) * kRows + lane / kChunks;
            col[k] = ((lane % kChunks) ^ tile_swizzle<D>(piece_row[k])) << 4;
        }
        auto issue = [&](int t) {
            const RowMeta& m = meta[t & 3];
            uint8_t *qt = lds[t & 1], *dt = lds[2 + (t & 1)];
#pragma unroll
            for (int k = 0; k < LPW; ++k) load_lds(m.q[piece_row[k]] + col[k], qt + (wave * LPW + k) * 1024);
#pragma unroll
            for (int k = 0; k < LPW; ++k) load_lds(m.d[piece_row[k]] + col[k], dt + (wave * LPW + k) * 1024);
        };
        const TileReader<D> read(lane);
        const float c = p.scale_log2;
        auto rows_block = [&](const RowMeta& m, const uint8_t* q_tile, const uint8_t* d_tile, int rb, bool masked) {
            f32x16 S, T;
#pragma unroll
            for (int i = 0; i < 16; ++i) S[i] = T[i] = 0.f;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) S = E::mfma(read.rows(q_tile, rb, ks), kf[ks], S);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) T = E::mfma(read.rows(d_tile, rb, ks), vf[ks], T);
            uint32_t pw[8], dw[8];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 l4 = *(const float4*)&m.lse2[32 * rb + 8 * q + 4 * half], d4 = *(const float4*)&m.delta[32 * rb + 8 * q + 4 * half];
                const float l[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
                float w[4], ds[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = __builtin_amdgcn_exp2f(fmaf(S[4 * q + i], c, -l[i]));
                    ds[i] = w[i] * (T[4 * q + i] - dl[i]);
                }
                if (masked) {
                    const int4 n4 = *(const int4*)&m.limit[32 * rb + 8 * q + 4 * half];
                    const int n[4] = {n4.x, n4.y, n4.z, n4.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (key >= n[i]) w[i] = ds[i] = 0.f;
                }
                pw[2 * q] = E::pack(w[0], w[1]);
                pw[2 * q + 1] = E::pack(w[2], w[3]);
                dw[2 * q] = E::pack(ds[0], ds[1]);
                dw[2 * q + 1] = E::pack(ds[2], ds[3]);
            }
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2) {
                const frag8 w = __builtin_bit_cast(frag8, make_uint4(pw[4 * s2], pw[4 * s2 + 1], pw[4 * s2 + 2], pw[4 * s2 + 3]));
#pragma unroll
                for (int db = 0; db < D / 32; ++db) dv[db] = E::mfma(read.cols(d_tile, rb, s2, db), w, dv[db]);
            }
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2) {
                const frag8 w = __builtin_bit_cast(frag8, make_uint4(dw[4 * s2], dw[4 * s2 + 1], dw[4 * s2 + 2], dw[4 * s2 + 3]));
#pragma unroll
                for (int db = 0; db < D / 32; ++db) dk[db] = E::mfma(read.cols(q_tile, rb, s2, db), w, dk[db]);
            }
        };
        issue(0);
        for (int t = 0; t < n_tiles; ++t) {
            tile_barrier();
            if (t + 1 < n_tiles) issue(t + 1);
            if (keeper) {   // (past the last tile too: the last row's again, in bounds)
                put_row(t + 2, ahead);
                ahead = find_row(t + 3, group_ahead);
                group_ahead = find_group(t + 4);
            }
            const RowMeta& m = meta[t & 3];
            const bool masked = __builtin_amdgcn_readfirstlane(m.least) < tile_key0 + 32 * KW;
            if constexpr (TEAMS == 1) {
                rows_block(m, lds[t & 1], lds[2 + (t & 1)], 0, masked);
                rows_block(m, lds[t & 1], lds[2 + (t & 1)], 1, masked);
            } else {
                rows_block(m, lds[t & 1], lds[2 + (t & 1)], team, masked);
            }
        }
    }
    __syncthreads();   // everyone is done with the tiles

    if constexpr (TEAMS == 2) {   // the second team's share, lane by lane: dK, then dV
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
    }
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
    store_rows<F16, D>(stage, dk, p.scale, lane, [&](int i) { return row_of(g.dK, i); });
    store_rows<F16, D>(stage, dv, 1.f, lane, [&](int i) { return row_of(g.dV, i); });
}

// dK and dV of the blocks that were cut into parts.
template <bool F16, int D>
__global__ __launch_bounds__(256) void grad_join_kernel(SelParams p, GradParams g, int tile_keys) {
    const SeqShape& s = p.s;
    uint32_t block, tile;
    fdivmod(blockIdx.x, g.fd_tiles, block, tile);
    const int2 join = g.joins[block];
    if (join.y <= 1) return;
    const int tiles = (int)g.fd_tiles.d;
    const uint32_t bh = block / (uint32_t)s.n_blocks, j = block - bh * (uint32_t)s.n_blocks;
    const int b = (int)fdiv(bh, p.fd_kv_heads), h = (int)bh - b * s.kv_heads;
    const int64_t pitch = (int64_t)tiles * 2 * tile_keys * D;   // of a slot
    const float* const src = g.slots + join.x * pitch + (int64_t)tile * 2 * tile_keys * D;
    for (int i = threadIdx.x; i < 2 * tile_keys * (D / 4); i += 256) {
        const int which = i / (tile_keys * (D / 4)), row = i / (D / 4) % tile_keys, c = i % (D / 4);
        const int key = (int)j * s.block + (int)tile * tile_keys + row;
        if (key >= s.n_k) continue;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k < join.y; ++k) {
            const float4 v = *(const float4*)(src + k * pitch + 4 * (int64_t)i);
            sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
        }
        const float f = which == 0 ? p.scale : 1.f;
        uint2 v;
        v.x = Elem<F16>::pack(sum.x * f, sum.y * f);
        v.y = Elem<F16>::pack(sum.z * f, sum.w * f);
        *(uint2*)((uint8_t*)row_address(which == 0 ? g.dK : g.dV, b, h, key) + 8 * c) = v;
    }
}

// ---- dQ ----------------------------------------------------------------------------------------
// The forward walk with dO beside Q in registers: S^T = K Q^T, dP^T = V dO^T, and dQ^T += K^T dS^T with K read both ways from its tile.
template <int RW, int TEAMS, bool F16, int D>
__global__ __launch_bounds__(RW * TEAMS * 64, RW * TEAMS == 2 ? 1 : 2) void grad_queries_kernel(SelParams p, GradParams g) {
    using E = Elem<F16>;
    constexpr int NW = RW * TEAMS, kTile = 64 * D * 2;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[4][kTile];   // K, K, V, V
    __shared__ int32_t s_n;
    extern __shared__ int32_t s_units[];
    const Item it(p);
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
    const int64_t stat = ((int64_t)it.b * s.q_heads + row.head) * s.n_q + row.query;
    const float lse = p.lse[stat], delta = g.delta[stat];
    const float lse2 = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f;   // (a row that attends nothing weighs 0)
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
    const TileReader<D> read(lane);
    auto unit_start = [&](int i) { return i < n_units ? __builtin_amdgcn_readfirstlane(s_units[i]) : kNoUnit; };
    auto block = [&](const uint8_t* k_tile, const uint8_t* v_tile, int hb, int start) {
        if (start >= most) return;
        f32x16 S, T;
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = T[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) S = E::mfma(read.rows(k_tile, hb, ks), qf[ks], S);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) T = E::mfma(read.rows(v_tile, hb, ks), df[ks], T);
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
            dw[i >> 1] = E::pack(d0, d1);
        }
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
            const frag8 w = __builtin_bit_cast(frag8, make_uint4(dw[4 * s2], dw[4 * s2 + 1], dw[4 * s2 + 2], dw[4 * s2 + 3]));
#pragma unroll
            for (int db = 0; db < D / 32; ++db) dq[db] = E::mfma(read.cols(k_tile, hb, s2, db), w, dq[db]);
        }
    };
    if (n_tiles > 0) {
        load.issue(unit_start(load.my_unit), lds[0], lds[2], wave);
        for (int t = 0; t < n_tiles; ++t) {
            const int next = unit_start(2 * t + 2 + load.my_unit);
            tile_barrier();
            if (t + 1 < n_tiles) load.issue(next, lds[(t + 1) & 1], lds[2 + ((t + 1) & 1)], wave);
            if constexpr (TEAMS == 1) {
                block(lds[t & 1], lds[2 + (t & 1)], 0, unit_start(2 * t));
                block(lds[t & 1], lds[2 + (t & 1)], 1, unit_start(2 * t + 1));
            } else {
                block(lds[t & 1], lds[2 + (t & 1)], team, unit_start(2 * t + team));
            }
        }
    }
    __syncthreads();   // everyone is done with the tiles
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
    uint8_t* const stage = &lds[0][0] + (TEAMS == 2 ? 2 * kTile : 0) + row_wave * 4096;   // (two teams: behind what team 0 still reads)
    store_rows<F16, D>(stage, dq, p.scale, lane, [&](int i) -> uint8_t* {
        const GroupRow to(p, it.h, it.g, (it.tile * RW + row_wave) * 32 + i);
        return to.there ? (uint8_t*)row_address(g.dQ, it.b, to.head, to.query) : nullptr;
    });
}

template <int KW, int TEAMS, bool F16, int D>
inline void launch_grad_keys(const SelParams& p, const GradParams& g, hipStream_t stream) {
    const int64_t items = (int64_t)g.most_parts * g.fd_tiles.d;
    hipLaunchKernelGGL((grad_keys_kernel<KW, TEAMS, F16, D>), dim3((unsigned)((items + 7) / 8 * 8)), dim3(KW * TEAMS * 64), 0, stream, p, g);
    hipLaunchKernelGGL((grad_join_kernel<F16, D>), dim3((unsigned)(g.blocks * g.fd_tiles.d)), dim3(256), 0, stream, p, g, 32 * KW);
}
template <int RW, int TEAMS, bool F16, int D>
inline void launch_grad_queries(const SelParams& p, const GradParams& g, hipStream_t stream) {
    const size_t dyn = sizeof(int32_t) * ((size_t)p.max_blocks * p.fd_units.d + 1);
    hipLaunchKernelGGL((grad_queries_kernel<RW, TEAMS, F16, D>), dim3(8 * p.per_xcd), dim3(RW * TEAMS * 64), dyn, stream, p, g);
}

// tile_rows: 128, 64 or 32; key tiles of 128, 64 or 32 keys
template <bool F16, int D>
inline hipError_t launch_bwd(const SelParams& p, const GradParams& g, int tile_rows, int tile_keys, hipStream_t stream) {
    const int64_t rows = (int64_t)p.s.batch * p.s.q_heads * p.s.n_q;
    hipLaunchKernelGGL((grad_delta_kernel<F16, D>), dim3((unsigned)((rows + 2048 / D - 1) / (2048 / D))), dim3(256), 0, stream, p, g, rows,
                       make_fastdiv((uint32_t)p.s.n_q), make_fastdiv((uint32_t)p.s.q_heads));
    launch_grad_lists(p, g, stream);
    if (tile_keys == 128) launch_grad_keys<4, 1, F16, D>(p, g, stream);
    else if (tile_keys == 64) launch_grad_keys<2, 2, F16, D>(p, g, stream);
    else launch_grad_keys<1, 2, F16, D>(p, g, stream);
    if (tile_rows == 128) launch_grad_queries<4, 1, F16, D>(p, g, stream);
    else if (tile_rows == 64) launch_grad_queries<2, 2, F16, D>(p, g, stream);
    else launch_grad_queries<1, 2, F16, D>(p, g, stream);
    return hipGetLastError();
}

}  // namespace grat
