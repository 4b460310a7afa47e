// Attention of a few rows over a cache of 16 or 8 bits: the newest tokens of a sequence as a chain or a tree of drafted tokens, within a window
// or over all keys.
//
// 8 bits, 32 heads on 8, head_dim 128: a token each of 64 sequences over 8 192 keys at most 157 us, 5.3 TB/s of values and scales; one token, window 4 096, 10.5 us: 6.5 to
// find its keys, fetch a unit and join four waves, 4 for the launch that joins the parts.
//
// Bound by fetching K and V, which no other rows share.  A workgroup is four waves that take every fourth unit of the keys (or of a share of
// them, `splits`) and wait for nothing but their own loads; each holds all of the workgroup's rows, 16 or 32.  The 16x16x32 instruction, with the rows as its columns:
// T^T (16 keys x 16 rows) leaves lane (row r = lane % 16, g = lane / 16) with keys 16 m + 4 g + i, and Z^T[16 dims, row] += X'^T T is contracted over
// 32 keys in that order: elements 0 .. 3 keys 4 g + i, 4 .. 7 keys 16 + 4 g + i.
// A unit is 32 keys, or 64: as soon as K's (or V's) has landed in LDS it is read into registers, and the next
// one's loads go out into the same place.
// 8 bits: e4m3 values become the 16-bit type of the product in registers, without loss.  A row's scale is taken to the score of its K in fp32, and to the weight of
// its V ahead of the weight's rounding.  Weights times scales may leave half's range, so they and V are bfloat16 there, whatever Q is; with half's Q a weight
// is two bfloat16 numbers, the second what the first leaves over, and V's product is formed with both.
#pragma once
#include "sequence_fwd.h"

namespace grat {

// Keys of a unit: 32, and 64 in 8 bits at head_dim 64, for chains (32 caches of 8 192 keys, a token each 51 us
// against 57, 8 tokens of 16 caches 34 against 38; but trees of 8 tokens 45 against 39, and at head_dim 128, where two workgroups of 32 rows then share a compute unit,
// a token each 98 against 94, trees of 8 tokens 63 against 58).
constexpr int cache_keys(bool eight, int head_dim, bool tree) { return eight && head_dim == 64 && !tree ? 64 : 32; }

// A wave's units of K and V, and its fragments in them.
template <bool EIGHT, int D, int KEYS>
struct CacheWave {
    static constexpr int kKeys = KEYS, kRow = EIGHT ? D : 2 * D, kTile = kKeys * kRow, kChunks = kRow / 16, kRows = 1024 / kRow, kPieces = kTile / 1024;
    static constexpr int kLoads = kPieces + (EIGHT ? 1 : 0);   // of a tile: its pieces and its scales
    static constexpr int kM = kKeys / 16, kN = D / 32, kDims = D / 16;
    static constexpr int kBytes = 2 * kTile + (EIGHT ? 512 : 0);   // K, V, their scales
    // Chunk c of a row lies at c ^ swizzle(row).  8 bits: ds_read_b128 of 16 consecutive rows, and the transpose read's rows 4 g + e, 16 + 4 g + e of
    // two neighbouring g, fall on the 16 chunk positions of a 256-byte line.
    static __device__ __forceinline__ int swizzle(int row) {
        if constexpr (EIGHT) return D == 128 ? ((row >> 1) & 7) ^ ((row >> 4) & 1) << 2 : ((row >> 2) & 3) ^ ((row >> 4) & 1) << 1;
        else return tile_swizzle<D>(row);
    }
    const uint8_t *K, *V;        // of the head
    const uint8_t *ks, *vs;      // their scales
    int64_t pitch_k, pitch_v, pitch_ks, pitch_vs;   // bytes
    uint8_t* lds;
    int first_end, near_end;     // keys are read below these: the first ones, the others
    int lane;
    uint32_t row_at, col_at;
    __device__ __forceinline__ CacheWave(const SelParams& p, const Item& it, uint8_t* lds_, int first_end_, int near_end_, int lane_)
        : lds(lds_), first_end(first_end_), near_end(near_end_), lane(lane_) {
        constexpr int kSize = EIGHT ? 1 : 2;
        const int r = lane & 15, g = lane >> 4;
        K = p.K.data + kSize * (it.b * p.K.stride_b + it.h * p.K.stride_h);
        V = p.V.data + kSize * (it.b * p.V.stride_b + it.h * p.V.stride_h);
        pitch_k = kSize * p.K.stride_n;
        pitch_v = kSize * p.V.stride_n;
        if constexpr (EIGHT) {
            ks = p.k_scale.data + 4 * (it.b * p.k_scale.stride_b + it.h * p.k_scale.stride_h);
            vs = p.v_scale.data + 4 * (it.b * p.v_scale.stride_b + it.h * p.v_scale.stride_h);
            pitch_ks = 4 * p.k_scale.stride_n;
            pitch_vs = 4 * p.v_scale.stride_n;
        }
        const uint32_t base = (uint32_t)(uintptr_t)(LDS_PTR(uint8_t))lds;
        row_at = base + r * kRow + ((swizzle(r) ^ g) << 4);
        if constexpr (EIGHT) {
            const int e = r >> 1, row = 4 * g + (e & 3) + 16 * (e >> 2);
            col_at = base + row * kRow + (swizzle(row) << 4) + 8 * (r & 1);
        } else {
            const int cq = r & 3, row = 4 * g + (r >> 2);
            col_at = base + row * kRow + (((cq >> 1) ^ swizzle(row)) << 4) + 8 * (cq & 1);
        }
    }
    // Keys behind the last one that may be read: it stands for them, and they are masked.
    __device__ __forceinline__ void fetch(const uint8_t* head, int64_t pitch, const uint8_t* scale, int64_t scale_pitch, int start, int which) const {
        const int left = (start < first_end ? first_end : near_end) - 1 - start;
        const uint8_t* const base = head + start * pitch;
        uint8_t* const tile = lds + which * kTile;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int row = k * kRows + lane / kChunks;
            load_lds(base, (uint32_t)min(row, left) * (uint32_t)pitch + (((lane % kChunks) ^ swizzle(row)) << 4), tile + k * 1024);
        }
        if constexpr (EIGHT) load_lds_word(scale + (start + (int64_t)min(lane, left)) * scale_pitch, lds + 2 * kTile + which * 256);
    }
    __device__ __forceinline__ void fetch_k(int start) const { fetch(K, pitch_k, ks, pitch_ks, start, 0); }
    __device__ __forceinline__ void fetch_v(int start) const { fetch(V, pitch_v, vs, pitch_vs, start, 1); }
    // Everything but the last tile's loads, or everything, has landed.  (Loads return in order; what was read from LDS is in registers too.)
    static __device__ __forceinline__ void wait_but_last() {
        __builtin_amdgcn_s_waitcnt(kLoads | 7 << 4);
        asm volatile("" ::: "memory");
    }
    __device__ __forceinline__ f32x4 scale(int which, int m) const {   // of keys 16 m + 4 g ..
        return *(const f32x4*)(lds + 2 * kTile + which * 256 + (16 * m + 4 * (lane >> 4)) * 4);
    }
};

// 8 e4m3 numbers as a fragment.
template <bool F16>
__device__ __forceinline__ frag8 widen(uint2 x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int v = (int)(i < 2 ? x.x : x.y);
        if constexpr (F16) w[i] = __builtin_bit_cast(uint32_t, i & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.f, false));
        else w[i] = __builtin_bit_cast(uint32_t, i & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.f, false));
    }
    return __builtin_bit_cast(frag8, make_uint4(w[0], w[1], w[2], w[3]));
}

template <int R, int KEYS, bool EIGHT, bool F16, int D, bool TREE>
__global__ __launch_bounds__(256, 2) void cache_attention_kernel(SelParams p) {
    using E = Elem<F16>;
    using W = CacheWave<EIGHT, D, KEYS>;
    using EV = Elem<F16 && !EIGHT>;   // of the weights and V
    using Out = NarrowWave<D>;
    constexpr int kLds = 4 * W::kBytes > 4 * 16 * D * 4 ? 4 * W::kBytes : 4 * 16 * D * 4;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kLds];
    __shared__ float s_m[4][16], s_l[4][16];
    __shared__ Tree tree[1];   // (of no size where nothing refers to it)
    Item it(p);
    if (it.idle(p)) return;
    int part_units = 0;
    if (!it.share(p, part_units)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), r = lane & 15, g = lane >> 4;
    const SeqShape& s = p.s;
    const int len = seq_len(s, it.b);
    const int64_t pos = window_pos(s, it.b, len);
    const int base = TREE ? len - s.n_q : 0;   // (trees are always the newest tokens)
    frag8 qf[R][W::kN];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const GroupRow row(p, it.h, 0, it.tile * (16 * R) + 16 * k + r);
        const uint8_t* const src = row_address(p.Q, it.b, row.head, row.query);
#pragma unroll
        for (int ks = 0; ks < W::kN; ++ks)   // 8 bits: 16 dims of K a lane and 64, as its reads have them
            qf[k][ks] = *(const frag8*)(src + (EIGHT ? 128 * (ks >> 1) + 32 * g + 16 * (ks & 1) : 64 * ks + 16 * g));
    }
    if constexpr (TREE) build_tree(tree[0], p, it.b, base);

    // what this lane's rows see, and what the workgroup's rows see together (all of the group's)
    RowSpan span[R];
    int line[TREE ? R : 1];   // trees: the row's line, in words
    const KeyRange keys = uniform(TREE ? tree_range(p, len) : rows_range(p, len, pos, 0, s.n_q - 1));
    const int first_end = keys.first_end, near = keys.near;
    int least_first = 0x7fffffff, least_hi = 0x7fffffff, most_lo = 0;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const GroupRow row(p, it.h, 0, it.tile * (16 * R) + 16 * k + r);
        if constexpr (TREE) {
            line[k] = row.query * kTreeWords;
            span[k] = tree_span(p, tree[0], base, row.query);
        } else {
            span[k] = row_span(p, len, pos, row.query);
        }
        if (row.there) {
            least_first = min(least_first, span[k].first);
            least_hi = min(least_hi, span[k].hi);
            most_lo = max(most_lo, span[k].lo);
        } else {
            span[k] = RowSpan{0, 0, 0};
        }
    }
#pragma unroll
    for (int m = 1; m < 16; m *= 2) {
        least_first = min(least_first, __shfl_xor(least_first, m));
        least_hi = min(least_hi, __shfl_xor(least_hi, m));
        most_lo = max(most_lo, __shfl_xor(most_lo, m));
    }
    least_first = __builtin_amdgcn_readfirstlane(least_first);
    least_hi = __builtin_amdgcn_readfirstlane(least_hi);
    most_lo = __builtin_amdgcn_readfirstlane(most_lo);
    const int first_units = (first_end + W::kKeys - 1) / W::kKeys, all_units = keys.units(W::kKeys);
    int u_first = 0, n_units = all_units;
    if (p.splits > 1) {
        const int per = part_units ? part_units : ((all_units + p.splits - 1) / p.splits + 3) & ~3;   // (a unit of every wave at a time)
        u_first = min(it.split * per, all_units);
        n_units = min(per, all_units - u_first);
    }
    auto unit_start = [&](int i) { return u_first + i < first_units ? (u_first + i) * W::kKeys : near + (u_first + i - first_units) * W::kKeys; };
    // Bit j: row k sees key `start` + j.
    auto sees = [&](int k, bool first, int start) {
        uint32_t bits = range_bits(start, first ? 0 : span[k].lo, first ? span[k].first : span[k].hi);
        if constexpr (TREE) {
            if (!first) bits |= line_bits(tree[0].lines + line[k], start - base);
        }
        return bits;
    };

    f32x4 oacc[R][W::kDims];
    float m_ref[R], l_run[R];
    const float cc = p.scale_log2;
#pragma unroll
    for (int k = 0; k < R; ++k) {
#pragma unroll
        for (int i = 0; i < W::kDims; ++i) oacc[k][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_ref[k] = -1e38f / fmaxf(cc, 1.f);   // (finite, so that a unit without a seen key weighs 0)
        l_run[k] = 0.f;
    }
    const W w(p, it, lds + wave * W::kBytes, first_end, keys.near_end, lane);
    frag8 kf[W::kM * (EIGHT ? W::kN / 2 : W::kN)], vf[EIGHT ? 1 : W::kDims];   // 8 bits: 16 numbers of K each
    uint2 v_raw[EIGHT ? W::kDims : 1][W::kM / 2];
    f32x4 k_scale[W::kM], v_scale[W::kM];
    constexpr bool kTwice = EIGHT && F16;   // weights of two bfloat16 numbers
    frag8 weights[R][W::kM / 2], rest[kTwice ? R : 1][W::kM / 2];
    auto take_k = [&]() {
#pragma unroll
        for (int m = 0; m < W::kM; ++m)
            if constexpr (EIGHT) {
#pragma unroll
                for (int kp = 0; kp < W::kN / 2; ++kp)
                    kf[m * (W::kN / 2) + kp] = *(LDS_PTR(const frag8))(uintptr_t)((w.row_at ^ (kp << 6) ^ ((m & 1) << (D == 128 ? 6 : 5))) + 16 * m * W::kRow);
                k_scale[m] = w.scale(0, m);
            } else {
#pragma unroll
                for (int ks = 0; ks < W::kN; ++ks) kf[m * W::kN + ks] = *(LDS_PTR(const frag8))(uintptr_t)((w.row_at ^ (ks << 6)) + 16 * m * W::kRow);
            }
    };
    auto take_v = [&]() {
        typedef __attribute__((ext_vector_type(2))) int i32x2;
#pragma unroll
        for (int dt = 0; dt < W::kDims; ++dt)
            if constexpr (EIGHT) {
                const uint32_t at = (w.col_at ^ (dt << 4)) + W::kTile;
                const i32x2 lo = __builtin_amdgcn_ds_read_tr8_b64_v2i32((LDS_PTR(i32x2))(uintptr_t)at);
                v_raw[dt][0] = make_uint2((uint32_t)lo[0], (uint32_t)lo[1]);
                if constexpr (W::kM == 4) {
                    const i32x2 hi = __builtin_amdgcn_ds_read_tr8_b64_v2i32((LDS_PTR(i32x2))(uintptr_t)(at + 32 * W::kRow));
                    v_raw[dt][W::kM / 2 - 1] = make_uint2((uint32_t)hi[0], (uint32_t)hi[1]);
                }
            } else {
                const uint32_t at = (w.col_at ^ (dt << 5)) + W::kTile;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)at);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(uintptr_t)(at + 16 * W::kRow));
                vf[dt] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            }
        if constexpr (EIGHT) {
#pragma unroll
            for (int m = 0; m < W::kM; ++m) v_scale[m] = w.scale(1, m);
        }
    };
    f32x4 S[R][W::kM];
    auto scores = [&]() {
#pragma unroll
        for (int m = 0; m < W::kM; ++m) {
#pragma unroll
            for (int k = 0; k < R; ++k) S[k][m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < W::kN; ++ks) {
                frag8 x;
                if constexpr (EIGHT) {
                    const uint4 raw = __builtin_bit_cast(uint4, kf[m * (W::kN / 2) + ks / 2]);
                    x = widen<F16>(ks & 1 ? make_uint2(raw.z, raw.w) : make_uint2(raw.x, raw.y));
                } else {
                    x = kf[m * W::kN + ks];
                }
#pragma unroll
                for (int k = 0; k < R; ++k) S[k][m] = E::mfma16(x, qf[k][ks], S[k][m]);
            }
            if constexpr (EIGHT) {
#pragma unroll
                for (int k = 0; k < R; ++k) S[k][m] *= k_scale[m];
            }
        }
    };
    auto weigh_rows = [&](int k, int start, bool cut, bool first) {
        f32x4(&X)[W::kM] = S[k];
        if (cut) {
#pragma unroll
            for (int h = 0; h < W::kM / 2; ++h) {
                const uint32_t bits = sees(k, first, start + 32 * h) >> (4 * g);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    X[2 * h][i] = bits >> i & 1 ? X[2 * h][i] : -INFINITY;
                    X[2 * h + 1][i] = bits >> (16 + i) & 1 ? X[2 * h + 1][i] : -INFINITY;
                }
            }
        }
        uint32_t pw[2 * W::kM], pr[2 * W::kM];
        auto weigh = [&]() {
            const float mc = m_ref[k] * cc;
            float ls = 0.f;
#pragma unroll
            for (int i = 0; i < 2 * W::kM; ++i) {
                const int m = i >> 1, e = 2 * (i & 1);
                const float a = __builtin_amdgcn_exp2f(fmaf(X[m][e], cc, -mc)), b = __builtin_amdgcn_exp2f(fmaf(X[m][e + 1], cc, -mc));
                const float x = EIGHT ? a * v_scale[m][e] : a, y = EIGHT ? b * v_scale[m][e + 1] : b;
                pw[i] = EV::pack(x, y);
                if constexpr (kTwice) pr[i] = EV::pack(x - __builtin_bit_cast(float, pw[i] << 16), y - __builtin_bit_cast(float, pw[i] & 0xffff0000u));
                ls += a + b;
            }
            return ls;
        };
        float ls = weigh();
        if (__builtin_amdgcn_ballot_w64(!(ls < EV::kSumLimit)) != 0) {   // the rare path: the true maximum, and everything against it
            float mx = X[0][0];
#pragma unroll
            for (int i = 1; i < 4 * W::kM; ++i) mx = fmaxf(mx, X[i >> 2][i & 3]);
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(m_ref[k], mx), alpha = __builtin_amdgcn_exp2f((m_ref[k] - m_new) * cc);
            m_ref[k] = m_new;
            l_run[k] *= alpha;
#pragma unroll
            for (int i = 0; i < W::kDims; ++i) oacc[k][i] *= alpha;
            ls = weigh();
        }
        l_run[k] += ls;
#pragma unroll
        for (int h = 0; h < W::kM / 2; ++h) {
            weights[k][h] = __builtin_bit_cast(frag8, make_uint4(pw[4 * h], pw[4 * h + 1], pw[4 * h + 2], pw[4 * h + 3]));
            if constexpr (kTwice) rest[k][h] = __builtin_bit_cast(frag8, make_uint4(pr[4 * h], pr[4 * h + 1], pr[4 * h + 2], pr[4 * h + 3]));
        }
    };
    auto products = [&]() {
#pragma unroll
        for (int dt = 0; dt < W::kDims; ++dt)
            if constexpr (EIGHT) {
#pragma unroll
                for (int h = 0; h < W::kM / 2; ++h) {
                    const frag8 x = widen<false>(v_raw[dt][h]);
#pragma unroll
                    for (int k = 0; k < R; ++k) {
                        oacc[k][dt] = EV::mfma16(x, weights[k][h], oacc[k][dt]);
                        if constexpr (kTwice) oacc[k][dt] = EV::mfma16(x, rest[k][h], oacc[k][dt]);
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < R; ++k) oacc[k][dt] = EV::mfma16(vf[dt], weights[k][0], oacc[k][dt]);
            }
    };
    if (wave < n_units) {
        int next = unit_start(wave);
        w.fetch_k(next);
        w.fetch_v(next);
        // (Q has landed: left to itself the compiler, which does not know of the loads into LDS, has its first use in the loop wait for all of them, in every step)
#pragma unroll
        for (int k = 0; k < R; ++k)
#pragma unroll
            for (int ks = 0; ks < W::kN; ++ks) asm volatile("" : "+v"(qf[k][ks]));
        for (int i = wave; i < n_units; i += 4) {
            const int start = next;
            const bool more = i + 4 < n_units, first = start < first_end;
            const bool cut = first ? start + W::kKeys > least_first : start + W::kKeys > least_hi || start < most_lo;
            next = unit_start(min(i + 4, n_units - 1));
            W::wait_but_last();   // K has landed
            take_k();
            W::wait_but_last();   // and is in registers
            if (more) w.fetch_k(next);
            scores();
            if (more) W::wait_but_last();   // V has landed
            else wave_wait();
            take_v();
            if (more) W::wait_but_last();
            else wave_wait();
            if (more) w.fetch_v(next);
#pragma unroll
            for (int k = 0; k < R; ++k) weigh_rows(k, start, cut, first);
            products();
        }
    }

    // the four waves' results, joined through LDS, 16 rows at a time
    float* const sums = (float*)lds;
    const int mine = threadIdx.x >> 4, sub = threadIdx.x & 15;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        float l = l_run[k] + __shfl_xor(l_run[k], 16);
        l += __shfl_xor(l, 32);
        __syncthreads();   // everyone is done with the tiles, or the 16 rows ahead
        Out::put(sums, wave, lane, oacc[k]);
        if (g == 0) {
            s_m[wave][r] = m_ref[k];
            s_l[wave][r] = l;
        }
        __syncthreads();
        float M = s_m[0][mine], f[4], total = 0.f, x[Out::kOwn];
#pragma unroll
        for (int i = 1; i < 4; ++i) M = fmaxf(M, s_m[i][mine]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = __builtin_amdgcn_exp2f((s_m[i][mine] - M) * cc);
            total = fmaf(f[i], s_l[i][mine], total);
        }
        Out::get(sums, f, x);
        if (p.splits > 1) {   // parts are joined by selected_join_kernel
            const int64_t at = (int64_t)it.item * (16 * R) + 16 * k + mine;
#pragma unroll
            for (int u = 0; u < Out::kOwn / 4; ++u)
                *(float4*)(p.part_o + at * D + Out::kOwn * sub + 4 * u) = make_float4(x[4 * u], x[4 * u + 1], x[4 * u + 2], x[4 * u + 3]);
            if (sub == 0) *(float2*)(p.part_ml + 2 * at) = make_float2(M, total);
            continue;
        }
        const GroupRow to(p, it.h, 0, it.tile * (16 * R) + 16 * k + mine);
        if (!to.there) continue;
        Out::template store<F16>((uint8_t*)row_address(p.O, it.b, to.head, to.query), x, total > 0.f ? 1.f / total : total);   // (a row that sees nothing: 0; NaN stays)
        if (p.lse && sub == 0)
            p.lse[((int64_t)it.b * s.q_heads + to.head) * s.n_q + to.query] = (M * cc + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
    }
}

// 16 R rows a workgroup
template <int R, bool EIGHT, bool F16, int D>
inline void launch_cache_sets(const SelParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)(8 * p.per_xcd));
    if (p.parent) hipLaunchKernelGGL((cache_attention_kernel<R, cache_keys(EIGHT, D, true), EIGHT, F16, D, true>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((cache_attention_kernel<R, cache_keys(EIGHT, D, false), EIGHT, F16, D, false>), grid, dim3(256), 0, stream, p);
}

// tile_rows: 16, 32; 64 (16 bits); 128, or 256 (head_dim 128)
template <bool F16, int D, int WALK, bool EIGHT>
inline void launch_cache_tiles(const SelParams& p, int tile_rows, hipStream_t stream) {
    if constexpr (D == 128) {
        if (tile_rows == 256) launch_fwd_tile<8, 1, F16, D, WALK, EIGHT>(p, stream);
    }
    if (tile_rows == 128) launch_fwd_tile<4, 1, F16, D, WALK, EIGHT>(p, stream);
    if constexpr (!EIGHT) {
        if (tile_rows == 64) launch_fwd_tile<2, 2, F16, D, WALK>(p, stream);
    }
    if (tile_rows == 32) launch_cache_sets<2, EIGHT, F16, D>(p, stream);
    else if (tile_rows == 16) launch_cache_sets<1, EIGHT, F16, D>(p, stream);
}

template <bool F16, int D>
inline hipError_t launch_cache_attention(const SelParams& p, bool eight, int tile_rows, hipStream_t stream) {
    if (eight && p.parent) launch_cache_tiles<F16, D, kTree, true>(p, tile_rows, stream);
    else if (eight) launch_cache_tiles<F16, D, kWindow, true>(p, tile_rows, stream);
    else if (p.parent) launch_cache_tiles<F16, D, kTree, false>(p, tile_rows, stream);
    else launch_cache_tiles<F16, D, kWindow, false>(p, tile_rows, stream);
    if (p.slots > 0) launch_join<F16, D, true>(p, tile_rows, stream);
    else if (p.splits > 1) launch_join<F16, D>(p, tile_rows, stream);
    return hipGetLastError();
}

}  // namespace grat
