// Attention over lists of key blocks, forward: O = softmax(scale Q K^T) V over the listed keys that a row sees.
//
// One pass over the keys with a running reference maximum and sum (base 2, scale * log2 e folded into one FMA a score; the reference
// is refreshed only where a block's sum leaves the safe range, as in attn_mfma.h).  A workgroup is RW waves of 32 rows of ONE group and
// TEAMS such sets that take the two units of a tile each (few rows), and walks the list, or with `splits` a share of
// it, in tiles of 64 keys through double-buffered LDS.
//
// 32 768 tokens, 32 heads on 8, 16 blocks of 64 keys, bf16: 570 to 606 us from card to card, 950 to 900 TFLOP/s (a library product of 16 384^3 reaches 1 375),
// the matrix pipe busy for 47 % of the cycles.  What holds it back: a block more takes 29 us (8 to 64 blocks: 363, 606, 1 080, 2 008), 1 185 TFLOP/s, and 140 us go
// by without the walk: 225 registers leave one workgroup of 8 waves to a compute unit, so nothing covers its start (count, list, Q, first K tile, one after the
// other) and its end (O through LDS), 9 us each time.  Few rows: bound by fetching K and V, see NarrowWave.
#pragma once
#include <type_traits>

#include "sequence_attn.h"

namespace grat {

template <int RW, int TEAMS, bool F16, int D>
__global__ __launch_bounds__(RW * TEAMS * 64, RW * TEAMS == 2 ? 1 : 2) void selected_fwd_kernel(SelParams p) {
    using E = Elem<F16>;
    constexpr int NW = RW * TEAMS, kTile = 64 * D * 2;
    __shared__ __attribute__((aligned(2 * kTile))) uint8_t lds[4][kTile];   // K, K, V, V
    __shared__ int32_t s_n;
    extern __shared__ int32_t s_units[];
    const Item it(p);
    if (it.idle(p)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int team = TEAMS == 1 ? 0 : wave / RW, row_wave = wave % RW;
    const int half = lane >> 5;
    const SeqShape& s = p.s;

    // this lane's row
    const int r = (it.tile * RW + row_wave) * 32 + (lane & 31);
    const GroupRow row(p, it.h, it.g, r);
    const uint8_t* const q_src = row_address(p.Q, it.b, row.head, row.query) + 16 * half;
    frag8 qf[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *(const frag8*)(q_src + 32 * ks);
    const int len = seq_len(s, it.b);
    const int64_t pos = seq_pos(s, it.b, len);
    const int seen = group_seen(s, len, pos, it.g);
    const int limit = row.there ? row_seen(s, len, pos, row.query) : 0;   // keys below it are seen
    int least = row.there ? limit : 0x7fffffff, most = limit;              // of the wave's rows
#pragma unroll
    for (int m = 1; m < 32; m *= 2) {
        least = min(least, __shfl_xor(least, m));
        most = max(most, __shfl_xor(most, m));
    }
    least = __builtin_amdgcn_readfirstlane(least);
    most = __builtin_amdgcn_readfirstlane(most);

    const int all_units = seen > 0 ? list_units(p, it.list(p), seen, s_units, &s_n) : 0;
    int u_first = 0, n_units = all_units;
    if (p.splits > 1) {   // an even number of units a part
        const int per = ((all_units + p.splits - 1) / p.splits + 1) & ~1;
        u_first = min(it.split * per, all_units);
        n_units = min(per, all_units - u_first);
    }
    const int n_tiles = (n_units + 1) / 2;

    f32x16 oacc[D / 32];
    clear<D>(oacc);
    const float c = p.scale_log2;
    float m_ref = -1e38f / fmaxf(c, 1.f);   // (finite, so that a block without a seen key weighs 0)
    float l_run = 0.f;

    const KeyLoader<NW, D> load(p, it, seen, wave, lane);
    TileReader<D> read(lane, lds[0], team);
    // (a list's last tile may lack its second unit; one of a part that ends inside the list does not)
    auto unit_start = [&](int i) { return i < n_units ? __builtin_amdgcn_readfirstlane(s_units[u_first + i]) : kNoUnit; };
    // (what fills a tile in its place is the list's last unit again: a key that is not listed may hold anything, and 0 * NaN is NaN)
    auto unit_load = [&](int i) { return __builtin_amdgcn_readfirstlane(s_units[u_first + max(min(i, n_units - 1), 0)]); };

    auto mask = [&](f32x16& S, int start) {
        if (start + kUnit > least) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (start + 8 * (i >> 2) + 4 * half + (i & 3) >= limit) S[i] = -INFINITY;
        }
    };
    auto weigh = [&](const f32x16& S, uint32_t (&w)[8]) {   // weights against the reference; this lane's sum of them
        const float mc = m_ref * c;
        float ls0 = 0.f, ls1 = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float a = __builtin_amdgcn_exp2f(fmaf(S[i], c, -mc)), b = __builtin_amdgcn_exp2f(fmaf(S[i + 1], c, -mc));
            w[i >> 1] = E::pack(a, b);
            ls0 += a;
            ls1 += b;
        }
        return ls0 + ls1;
    };
    // The rare path: a block's sum has left the safe range.  The true maximum, and everything against it.
    auto refresh = [&](const f32x16& S, uint32_t (&w)[8]) {
        float mx = S[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, S[i]);
        const float m_new = fmaxf(m_ref, max_across_halves(mx));
        const float alpha = __builtin_amdgcn_exp2f((m_ref - m_new) * c);
        m_ref = m_new;
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) oacc[db][i] *= alpha;
        return weigh(S, w);
    };
    auto outside = [&](float ls) { return __builtin_amdgcn_ballot_w64(!(ls < E::kSumLimit)) != 0; };

    if constexpr (TEAMS == 2) {
        // few rows: latency is what counts, a block after the other
        auto block = [&](int start) {
            if (start >= most) return;   // nobody in this wave sees the unit
            f32x16 S;
#pragma unroll
            for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) S = E::mfma(read.rows(0, 0, ks), qf[ks], S);
            mask(S, start);
            uint32_t pw[8];
            float ls = weigh(S, pw);
            if (outside(ls)) ls = refresh(S, pw);
            l_run += ls;
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2) {
                const frag8 w = __builtin_bit_cast(frag8, make_uint4(pw[4 * s2], pw[4 * s2 + 1], pw[4 * s2 + 2], pw[4 * s2 + 3]));
#pragma unroll
                for (int db = 0; db < D / 32; ++db) oacc[db] = E::mfma(read.cols(1, 0, s2, db), w, oacc[db]);
            }
        };
        if (n_tiles > 0) load.issue(unit_load(load.my_unit), lds[0], lds[2], wave);
        for (int t = 0; t < n_tiles; ++t) {
            const int next = unit_load(2 * t + 2 + load.my_unit);
            tile_barrier();
            if (t + 1 < n_tiles) load.issue(next, lds[(t + 1) & 1], lds[2 + ((t + 1) & 1)], wave);
            block(unit_start(2 * t + team));
            read.flip();
        }
    } else {
        // Between two barriers one stream of instructions, pipelined by units: while the matrix pipe forms the scores of a unit, the vector
        // ALU weighs those of the unit before, and the matrix pipe adds the one before that to O.  A step is two such halves: K of
        // tile t and V of tile t - 1.  The three do not depend on each other, so every product is followed by its share of the vector work
        // (6 vector instructions fit behind one) and by the read of the fragment for the product kAhead later.
        constexpr int kAhead = 2, kN = D / 16, kM = 2 * (D / 32);
        f32x16 S[2];
        uint32_t pw[2][8];
        int ahead = unit_load(load.my_unit), here = 0;   // first keys of this wave's pieces of tile t + 1 and t
        int late = kNoUnit;                               // ... of the second unit of tile t - 1
        auto step = [&](auto odd_c, auto first_c, auto last_c, int t) {
            constexpr int kOdd = decltype(odd_c)::value;   // t & 1
            constexpr bool kScores = !decltype(last_c)::value, kAdds = !decltype(first_c)::value;
            constexpr int kItems = (kScores ? kN : 0) + (kAdds ? kM : 0);
            const int start0 = kScores ? unit_start(2 * t) : 0, start1 = kScores ? unit_start(2 * t + 1) : 0;
            here = ahead;
            ahead = unit_load(2 * t + 2 + load.my_unit);
            tile_barrier();
            if (t + 1 < n_tiles) load.issue(load.K, load.pitch_k, ahead, lds[kOdd ^ 1], wave);
            if (kScores) load.issue(load.V, load.pitch_v, here, lds[2 + kOdd], wave);
            frag8 fr[2 * kItems];
            auto fetch = [&](int i) {
                const int h = i / kItems, j = i % kItems;
                if (kScores && j < kN) fr[i] = read.rows(0, h, j, kOdd);
                else fr[i] = read.cols(1, h, (j - (kScores ? kN : 0)) / (D / 32), (j - (kScores ? kN : 0)) % (D / 32), kOdd ^ 1);
            };
#pragma unroll
            for (int i = 0; i < kAhead; ++i) fetch(i);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool weighs = h == 0 ? kAdds : kScores;   // half 0: the second unit of tile t - 1, half 1: the first of tile t
                f32x16& W = S[h ^ 1];
                float e0[8], t1[8], ls0 = 0.f, ls1 = 0.f, mc = 0.f;
                if (weighs) {
                    mask(W, h == 0 ? late : start0);
                    mc = m_ref * c;
                }
                auto chunk = [&](int i) {   // 16 of them: a pair of scores takes two
                    const int g = i >> 1;
                    if ((i & 1) == 0) {
                        t1[g] = fmaf(W[2 * g + 1], c, -mc);
                        e0[g] = __builtin_amdgcn_exp2f(fmaf(W[2 * g], c, -mc));
                    } else {
                        const float e1 = __builtin_amdgcn_exp2f(t1[g]);
                        pw[h ^ 1][g] = E::pack(e0[g], e1);
                        asm volatile("" : "+v"(pw[h ^ 1][g]));   // (keeps the conversion here: its first use is a block later)
                        ls0 += e0[g];
                        ls1 += e1;
                    }
                };
#pragma unroll
                for (int j = 0; j < kItems; ++j) {
                    const int i = h * kItems + j;
                    if (i + kAhead < 2 * kItems) fetch(i + kAhead);
                    if (kScores && j < kN) {
                        f32x16 zero;
#pragma unroll
                        for (int r = 0; r < 16; ++r) zero[r] = 0.f;
                        S[h] = E::mfma(fr[i], qf[j], j == 0 ? zero : S[h]);
                    } else {
                        const int a = j - (kScores ? kN : 0), s2 = a / (D / 32), db = a % (D / 32);
                        const uint32_t* const x = &pw[h][4 * s2];
                        oacc[db] = E::mfma(fr[i], __builtin_bit_cast(frag8, make_uint4(x[0], x[1], x[2], x[3])), oacc[db]);
                    }
                    if (weighs) {
#pragma unroll
                        for (int k = 16 * j / kItems; k < 16 * (j + 1) / kItems; ++k) chunk(k);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (weighs) {
                    float ls = ls0 + ls1;
                    if (outside(ls)) ls = refresh(W, pw[h ^ 1]);
                    l_run += ls;
                }
            }
            late = start1;
        };
        using std::false_type;
        using std::true_type;
        using std::integral_constant;
        constexpr integral_constant<int, 0> even{};
        constexpr integral_constant<int, 1> odd{};
        if (n_tiles > 0) {
            load.issue(load.K, load.pitch_k, ahead, lds[0], wave);
            if (most == 0) {   // a wave without a row only fetches
                for (int t = 0; t <= n_tiles; ++t) {
                    here = ahead;
                    ahead = unit_load(2 * t + 2 + load.my_unit);
                    tile_barrier();
                    if (t + 1 < n_tiles) load.issue(load.K, load.pitch_k, ahead, lds[(t + 1) & 1], wave);
                    if (t < n_tiles) load.issue(load.V, load.pitch_v, here, lds[2 + (t & 1)], wave);
                }
            } else {
                step(even, true_type{}, false_type{}, 0);
                int t = 1;
                for (; t + 1 < n_tiles; t += 2) {
                    step(odd, false_type{}, false_type{}, t);
                    step(even, false_type{}, false_type{}, t + 1);
                }
                if (t < n_tiles) step(odd, false_type{}, false_type{}, t);
                if (n_tiles & 1) step(odd, false_type{}, true_type{}, n_tiles);
                else step(even, false_type{}, true_type{}, n_tiles);
            }
        }
    }
    float l = sum_across_halves(l_run);

    // ---- the second team's share, lane by lane -----------------------------------------------------
    if constexpr (TEAMS == 2) {
        __shared__ float s_m[RW][64], s_l[RW][64];
        float* const part = (float*)&lds[0][0] + row_wave * 64 * (D / 2) + lane;   // [register][lane]
        static_assert(RW * 64 * (D / 2) * 4 <= 2 * kTile && RW * 4096 <= 2 * kTile, "the partial results, and behind them the output");
        __syncthreads();
        if (team == 1) {
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) part[(db * 16 + i) * 64] = oacc[db][i];
            s_m[row_wave][lane] = m_ref;
            s_l[row_wave][lane] = l;
        }
        __syncthreads();
        if (team == 1) return;
        const float m2 = s_m[row_wave][lane], m = fmaxf(m_ref, m2);
        const float f1 = __builtin_amdgcn_exp2f((m_ref - m) * c), f2 = __builtin_amdgcn_exp2f((m2 - m) * c);
        m_ref = m;
        l = l * f1 + s_l[row_wave][lane] * f2;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) oacc[db][i] = oacc[db][i] * f1 + part[(db * 16 + i) * 64] * f2;
    } else {
        __syncthreads();   // everyone is done with the tiles: the output is turned through them
    }

    if (p.splits > 1) {   // parts are joined by selected_join_kernel
        const int64_t at = (int64_t)it.item * (RW * 32) + row_wave * 32 + (lane & 31);
        float* const dst = p.part_o + at * D + 4 * half;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(float4*)(dst + 32 * db + 8 * q) = make_float4(oacc[db][4 * q], oacc[db][4 * q + 1], oacc[db][4 * q + 2], oacc[db][4 * q + 3]);
        if (half == 0) *(float2*)(p.part_ml + 2 * at) = make_float2(m_ref, l);
        return;
    }
    const float inv = l > 0.f ? 1.f / l : l;   // (a row that attends nothing: 0; NaN stays)
    if (p.lse && half == 0 && row.there)
        p.lse[((int64_t)it.b * s.q_heads + row.head) * s.n_q + row.query] = (m_ref * c + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;

    uint8_t* const stage = &lds[0][0] + (TEAMS == 2 ? 2 * kTile : 0) + row_wave * 4096;   // (two teams: behind what team 0 still reads)
    store_rows<F16, D>(stage, oacc, inv, lane, [&](int i) -> uint8_t* {
        const GroupRow to(p, it.h, it.g, (it.tile * RW + row_wave) * 32 + i);
        return to.there ? (uint8_t*)row_address(p.O, it.b, to.head, to.query) : nullptr;
    });
}

// Groups of at most 16 rows; the four waves' results are joined through LDS.  Measured: 64 tokens of half over 2 048 keys each 26.9 us with the
// join (134 MB, 5.0 TB/s); one token over 2 048 keys 8.9 us, most of it two launches' start and one chain of dependent loads.
template <bool F16, int D>
__global__ __launch_bounds__(256, 2) void selected_fwd_narrow_kernel(SelParams p) {
    using E = Elem<F16>;
    using W = NarrowWave<D>;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[4][2 * W::kTile];   // K, V of every wave
    __shared__ float s_m[4][16], s_l[4][16];
    __shared__ int32_t s_n;
    extern __shared__ int32_t s_units[];
    const Item it(p);
    if (it.idle(p)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), r = lane & 15, g = lane >> 4;
    const SeqShape& s = p.s;
    const GroupRow row(p, it.h, it.g, it.tile * 16 + r);
    const uint8_t* const q_src = row_address(p.Q, it.b, row.head, row.query) + 16 * g;
    frag8 qf[W::kN];
#pragma unroll
    for (int ks = 0; ks < W::kN; ++ks) qf[ks] = *(const frag8*)(q_src + 64 * ks);
    const int len = seq_len(s, it.b);
    const int64_t pos = seq_pos(s, it.b, len);
    const int seen = group_seen(s, len, pos, it.g);
    const int limit = row.there ? row_seen(s, len, pos, row.query) : 0;
    int least = row.there ? limit : 0x7fffffff;
#pragma unroll
    for (int m = 1; m < 16; m *= 2) least = min(least, __shfl_xor(least, m));
    least = __builtin_amdgcn_readfirstlane(least);
    const int all_units = seen > 0 ? list_units(p, it.list(p), seen, s_units, &s_n) : 0;
    int u_first = 0, n_units = all_units;
    if (p.splits > 1) {
        const int per = (all_units + p.splits - 1) / p.splits;
        u_first = min(it.split * per, all_units);
        n_units = min(per, all_units - u_first);
    }

    f32x4 oacc[W::kM];
#pragma unroll
    for (int i = 0; i < W::kM; ++i) oacc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float c = p.scale_log2;
    float m_ref = -1e38f / fmaxf(c, 1.f), l_run = 0.f;   // (finite, so that a unit without a seen key weighs 0)
    const W w(p, it, lds[wave], seen, lane);
    frag8 kf[2][W::kN], vf[W::kM], weights;
    auto take_k = [&]() {
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int ks = 0; ks < W::kN; ++ks) kf[m][ks] = w.rows(0, m, ks);
    };
    auto take_v = [&]() {
#pragma unroll
        for (int dt = 0; dt < W::kM; ++dt) vf[dt] = w.cols(1, dt);
    };
    auto scores = [&](int start) {
        f32x4 S[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            S[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < W::kN; ++ks) S[m] = E::mfma16(kf[m][ks], qf[ks], S[m]);
        }
        if (start + kUnit > least) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (start + 16 * (i >> 2) + 4 * g + (i & 3) >= limit) S[i >> 2][i & 3] = -INFINITY;
        }
        uint32_t pw[4];
        auto weigh = [&]() {
            const float mc = m_ref * c;
            float ls = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = S[i >> 1][2 * (i & 1)], y = S[i >> 1][2 * (i & 1) + 1];
                const float a = __builtin_amdgcn_exp2f(fmaf(x, c, -mc)), b = __builtin_amdgcn_exp2f(fmaf(y, c, -mc));
                pw[i] = E::pack(a, b);
                ls += a + b;
            }
            return ls;
        };
        float ls = weigh();
        if (__builtin_amdgcn_ballot_w64(!(ls < E::kSumLimit)) != 0) {   // the rare path: the true maximum, and everything against it
            float mx = fmaxf(fmaxf(fmaxf(S[0][0], S[0][1]), fmaxf(S[0][2], S[0][3])), fmaxf(fmaxf(S[1][0], S[1][1]), fmaxf(S[1][2], S[1][3])));
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(m_ref, mx), alpha = __builtin_amdgcn_exp2f((m_ref - m_new) * c);
            m_ref = m_new;
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < W::kM; ++i) oacc[i] *= alpha;
            ls = weigh();
        }
        l_run += ls;
        weights = __builtin_bit_cast(frag8, make_uint4(pw[0], pw[1], pw[2], pw[3]));
    };
    w.walk(s_units + u_first, n_units, wave, take_k, scores, take_v, [&](int) {
#pragma unroll
        for (int dt = 0; dt < W::kM; ++dt) oacc[dt] = E::mfma16(vf[dt], weights, oacc[dt]);
    });

    float l = l_run + __shfl_xor(l_run, 16);
    l += __shfl_xor(l, 32);
    float* const sums = (float*)&lds[0][0];
    static_assert(4 * 16 * D * 4 <= (int)sizeof(lds), "the results fit the tiles");
    __syncthreads();   // everyone is done with the tiles
    W::put(sums, wave, lane, oacc);
    if (g == 0) {
        s_m[wave][r] = m_ref;
        s_l[wave][r] = l;
    }
    __syncthreads();
    const int mine = threadIdx.x >> 4, sub = threadIdx.x & 15;
    float M = s_m[0][mine], f[4], total = 0.f, x[W::kOwn];
#pragma unroll
    for (int k = 1; k < 4; ++k) M = fmaxf(M, s_m[k][mine]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        f[k] = __builtin_amdgcn_exp2f((s_m[k][mine] - M) * c);
        total = fmaf(f[k], s_l[k][mine], total);
    }
    W::get(sums, f, x);
    if (p.splits > 1) {   // parts are joined by selected_join_kernel
        const int64_t at = (int64_t)it.item * 16 + mine;
#pragma unroll
        for (int u = 0; u < W::kOwn / 4; ++u)
            *(float4*)(p.part_o + at * D + W::kOwn * sub + 4 * u) = make_float4(x[4 * u], x[4 * u + 1], x[4 * u + 2], x[4 * u + 3]);
        if (sub == 0) *(float2*)(p.part_ml + 2 * at) = make_float2(M, total);
        return;
    }
    const GroupRow to(p, it.h, it.g, it.tile * 16 + mine);
    if (!to.there) return;
    W::template store<F16>((uint8_t*)row_address(p.O, it.b, to.head, to.query), x, total > 0.f ? 1.f / total : total);   // (a row that attends nothing: 0; NaN stays)
    if (p.lse && sub == 0)
        p.lse[((int64_t)it.b * s.q_heads + to.head) * s.n_q + to.query] = (M * c + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
}

// Joins the parts of a split list, weighted by 2^(c (m - max m)).  D / 4 lanes share a row's dims; eight parts are in flight at a time.  (1 024 rows of
// two parts 4.0 us.  More lanes a row, one for every part, do not shorten it.)
template <bool F16, int D>
__global__ __launch_bounds__(256) void selected_join_kernel(SelParams p, int tile_rows, FastDiv fd_rows) {
    constexpr int L = D / 4, RPB = 256 / L;   // lanes of a row, rows of a workgroup
    const SeqShape& s = p.s;
    const int lane = threadIdx.x % L;
    const int64_t n = (int64_t)s.batch * s.kv_heads * s.n_groups * p.rows, at = min((int64_t)blockIdx.x * RPB + threadIdx.x / L, n - 1);
    uint32_t list, r, bh, g, b, h;
    fdivmod((uint32_t)at, fd_rows, list, r);
    fdivmod(list, p.fd_groups, bh, g);
    fdivmod(bh, p.fd_kv_heads, b, h);
    const GroupRow row(p, (int)h, (int)g, (int)r);
    const int64_t first = (((int64_t)list * p.row_tiles + r / tile_rows) * p.splits) * tile_rows + r % tile_rows;   // + split * tile_rows
    const float2* const ml = (const float2*)p.part_ml + first;
    const float4* const po = (const float4*)p.part_o + first * L + lane;
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < p.splits; i0 += 8) {
        float2 v[8];
        float4 x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = min(i0 + k, p.splits - 1);
            v[k] = ml[(int64_t)i * tile_rows];
            x[k] = po[(int64_t)i * tile_rows * L];
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = fmaxf(top, v[k].x);
        const float old = m == top ? 1.f : __builtin_amdgcn_exp2f((m - top) * p.scale_log2);
        l *= old;
        o = make_float4(o.x * old, o.y * old, o.z * old, o.w * old);
        m = top;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float f = i0 + k < p.splits ? __builtin_amdgcn_exp2f((v[k].x - m) * p.scale_log2) : 0.f;
            l = fmaf(f, v[k].y, l);
            o = make_float4(fmaf(f, x[k].x, o.x), fmaf(f, x[k].y, o.y), fmaf(f, x[k].z, o.z), fmaf(f, x[k].w, o.w));
        }
    }
    if ((int64_t)blockIdx.x * RPB + threadIdx.x / L >= n || !row.there) return;
    const float inv = l > 0.f ? 1.f / l : l;
    uint2 v;
    v.x = Elem<F16>::pack(o.x * inv, o.y * inv);
    v.y = Elem<F16>::pack(o.z * inv, o.w * inv);
    *(uint2*)((uint8_t*)row_address(p.O, (int)b, row.head, row.query) + 8 * lane) = v;
    if (p.lse && lane == 0)
        p.lse[((int64_t)b * s.q_heads + row.head) * s.n_q + row.query] = (m * p.scale_log2 + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <bool F16, int D>
inline void launch_join(const SelParams& p, int tile_rows, hipStream_t stream) {
    const int64_t rows = (int64_t)p.s.batch * p.s.kv_heads * p.s.n_groups * p.rows, per = 1024 / D;
    hipLaunchKernelGGL((selected_join_kernel<F16, D>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, stream, p, tile_rows,
                       make_fastdiv((uint32_t)p.rows));
}

template <int RW, int TEAMS, bool F16, int D>
inline void launch_fwd_tile(const SelParams& p, hipStream_t stream) {
    const size_t dyn = sizeof(int32_t) * ((size_t)p.max_blocks * p.fd_units.d + 1);
    hipLaunchKernelGGL((selected_fwd_kernel<RW, TEAMS, F16, D>), dim3(8 * p.per_xcd), dim3(RW * TEAMS * 64), dyn, stream, p);
}

// tile_rows: 256 (head_dim 128), 128, 64, 32 or 16
template <bool F16, int D>
inline hipError_t launch_fwd(const SelParams& p, int tile_rows, hipStream_t stream) {
    if constexpr (D == 128) {
        if (tile_rows == 256) launch_fwd_tile<8, 1, F16, D>(p, stream);
    }
    if (tile_rows == 128) launch_fwd_tile<4, 1, F16, D>(p, stream);
    else if (tile_rows == 64) launch_fwd_tile<2, 2, F16, D>(p, stream);
    else if (tile_rows == 32) launch_fwd_tile<1, 2, F16, D>(p, stream);
    else if (tile_rows == 16)
        hipLaunchKernelGGL((selected_fwd_narrow_kernel<F16, D>), dim3(8 * p.per_xcd), dim3(256), sizeof(int32_t) * ((size_t)p.max_blocks * p.fd_units.d + 1),
                           stream, p);
    if (p.splits > 1) launch_join<F16, D>(p, tile_rows, stream);
    return hipGetLastError();
}

}  // namespace grat
