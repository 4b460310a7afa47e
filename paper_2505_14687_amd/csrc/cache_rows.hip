// Rows of a cache in 8 bits: written with the new tokens' K turned by their positions, and read back.
//
// A row of head_dim numbers x is kept as e4m3 values of x / s and s, the least power of two with max |x| <= 448 s: as e4m3 is a floating format
// itself, a finer s would gain nothing, and with this one the division and the way back are exact.  Memory (for few tokens the launch) bounds both directions: 2 x 8 191 tokens of 32 + 2 x 8 heads written 82 us
// (4.5 TB/s in and out), 8 caches of 16 384 keys at most read back 74 us (5.1 TB/s), a token each of 32 sequences 5.5.  Rows of the tensors' own type, the same tokens: bf16 77 us
// (5.2 TB/s), fp32 155, K and V alone 22 and 44; a token each of 32 sequences 4.5.
#include <algorithm>
#include <type_traits>

#include "cache_rows.h"
#include "rotary_pairs.h"

namespace grat {

typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr int kOwnHeads = 2;   // of a thread, in flight at a time (a token each of 32 sequences 5.4 us; 4 heads 6.3, 8 heads 9.6; 8 192 tokens alike)

// 4 numbers as e4m3, rounded to nearest-even; |x| <= 448, NaN and infinities become NaN
__device__ __forceinline__ uint32_t narrow(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return (uint32_t)w;
}

// The power of two of a row whose largest finite |x| is `most`: 448 = 7/8 2^9.
__device__ __forceinline__ int row_power(float most) {
    if (!(most > 0.f)) return 0;
    const int e = __builtin_amdgcn_frexp_expf(most);
    return max(e - (__builtin_amdgcn_frexp_mantf(most) > 0.875f ? 8 : 9), -126);
}

// The largest number of 4, 8 or 16 neighbouring lanes.
__device__ __forceinline__ float row_max(float x, int lanes) {
    auto with = [&](float y) { return fmaxf(x, y); };
#define GRAT_DPP(x, control) __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), control, 0xf, 0xf, true))
    x = with(GRAT_DPP(x, 0xb1));    // lane ^ 1
    x = with(GRAT_DPP(x, 0x4e));    // lane ^ 2
    if (lanes > 4) x = with(GRAT_DPP(x, 0x141));    // the other four of eight, in mirror order
    if (lanes > 8) x = with(GRAT_DPP(x, 0x140));    // the other eight
#undef GRAT_DPP
    return x;
}

// Thread and piece as in rotary_kernel; the lanes of a row, `items` neighbours, find its largest number together.
template <typename T, bool AXES, bool EIGHT>
__global__ __launch_bounds__(256) void cache_append_kernel(RotaryParams p, SeqTensor k_scale, SeqTensor v_scale, FastDiv fd_inner, int32_t per_y, int32_t heads_first) {
    typedef typename Vec16<T>::type vec;
    constexpr int V = Vec16<T>::n;
    uint32_t slot, item, b, n;
    fdivmod(threadIdx.x, p.fd_items, slot, item);
    uint32_t outer, inner;
    fdivmod(blockIdx.x, fd_inner, outer, inner);
    const uint32_t at = heads_first ? outer : inner, chunk = heads_first ? inner : outer;
    const uint32_t per_block = 256u / (uint32_t)p.items, token = (blockIdx.y * (uint32_t)per_y + at) * per_block + slot;
    if (token >= (uint32_t)p.batch * (uint32_t)p.n_tokens) return;   // (items divides a wave: rows end as a whole)
    fdivmod(token, p.fd_tokens, b, n);

    const int turned = p.rot / (2 * V);
    const bool turn = (int)item < turned;
    const int lo = turn && !p.interleaved ? (int)item * V : (int)item * 2 * V;
    const int hi = turn && !p.interleaved ? lo + p.rot / 2 : lo + V;
    float cs[V], sn[V];
    if (turn) pair_angles<T, AXES>(p, (int)b, (int)n, (int)item * V, cs, sn);

    const int all = p.heads[0] + p.heads[1] + p.heads[2];
    const int64_t row = (int64_t)p.start[b] + n;
    const bool in_cache = row >= 0 && row < p.n_cache;
    for (int h0 = (int)chunk * p.head_chunk, h1 = min(all, h0 + p.head_chunk); h0 < h1; h0 += kOwnHeads) {
        vec x[kOwnHeads], y[kOwnHeads];
        uint8_t* dst[kOwnHeads];
        float* scale[kOwnHeads];   // of a row that is kept in 8 bits
        int kind[kOwnHeads];       // 0: Q, 1: K, 2: V
#pragma unroll
        for (int i = 0; i < kOwnHeads; ++i) {
            int h = min(h0 + i, h1 - 1), t = 0;
            if (h >= p.heads[0]) { h -= p.heads[0]; t = 1; if (h >= p.heads[1]) { h -= p.heads[1]; t = 2; } }
            // (uniform; an index into the parameters would put them into scratch memory)
            const SeqTensor in = t == 0 ? p.in[0] : t == 1 ? p.in[1] : p.in[2], out = t == 0 ? p.out[0] : t == 1 ? p.out[1] : p.out[2];
            const T* const src = (const T*)in.data + b * in.stride_b + h * in.stride_h + n * in.stride_n;
            const bool keep = h0 + i < h1 && (t == 0 || in_cache);
            const int64_t to = b * out.stride_b + h * out.stride_h + (t > 0 ? row : (int64_t)n) * out.stride_n;
            dst[i] = keep ? out.data + to * (EIGHT && t > 0 ? 1 : (int)sizeof(T)) : nullptr;
            kind[i] = t;
            if constexpr (EIGHT) {
                const SeqTensor sc = t == 1 ? k_scale : v_scale;
                scale[i] = (float*)sc.data + b * sc.stride_b + h * sc.stride_h + row * sc.stride_n;
            }
            x[i] = *(const vec*)(src + lo);
            y[i] = *(const vec*)(src + hi);
        }
#pragma unroll
        for (int i = 0; i < kOwnHeads; ++i) {
            const int t = kind[i];
            float u[V], v[V];   // the piece's two vectors
#pragma unroll
            for (int e = 0; e < V; ++e) {
                u[e] = (float)x[i][e];
                v[e] = (float)y[i][e];
            }
            if (turn && t < 2) {
// (each product and sum rounded, as elementary operations would: what lies next to a border of the 8 bits then falls to the same side)
#pragma clang fp contract(off)
                if (p.interleaved) {
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        const int q = e / 2, q2 = V / 2 + e / 2;
                        const float f = u[e], c = u[e + 1], f2 = v[e], c2 = v[e + 1];
                        u[e] = cs[q] * f - sn[q] * c;
                        u[e + 1] = sn[q] * f + cs[q] * c;
                        v[e] = cs[q2] * f2 - sn[q2] * c2;
                        v[e + 1] = sn[q2] * f2 + cs[q2] * c2;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float f = u[e], c = v[e];
                        u[e] = cs[e] * f - sn[e] * c;
                        v[e] = sn[e] * f + cs[e] * c;
                    }
                }
            }
            if (EIGHT && t > 0) {
                float most = 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float f = fabsf(u[e]), c = fabsf(v[e]);
                    most = fmaxf(most, fmaxf(f < INFINITY ? f : 0.f, c < INFINITY ? c : 0.f));
                }
                most = row_max(most, p.items);
                const int power = row_power(most);
                const float inv = ldexpf(1.f, -power);
                if constexpr (std::is_same_v<T, _Float16>) {   // what half holds stays finite when it is read back: 256 2^8 would not
                    if (power == 8) {
                        const float top = 240.f * 256.f;
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            u[e] = fabsf(u[e]) < 65520.f ? fminf(fmaxf(u[e], -top), top) : u[e];
                            v[e] = fabsf(v[e]) < 65520.f ? fminf(fmaxf(v[e], -top), top) : v[e];
                        }
                    }
                }
                uint32_t wu[V / 4], wv[V / 4];
#pragma unroll
                for (int k = 0; k < V / 4; ++k) {
                    wu[k] = narrow(u[4 * k] * inv, u[4 * k + 1] * inv, u[4 * k + 2] * inv, u[4 * k + 3] * inv);
                    wv[k] = narrow(v[4 * k] * inv, v[4 * k + 1] * inv, v[4 * k + 2] * inv, v[4 * k + 3] * inv);
                }
                if (dst[i]) {
                    if constexpr (V == 8) {
                        *(uint2*)(dst[i] + lo) = make_uint2(wu[0], wu[1]);
                        *(uint2*)(dst[i] + hi) = make_uint2(wv[0], wv[1]);
                    } else {
                        *(uint32_t*)(dst[i] + lo) = wu[0];
                        *(uint32_t*)(dst[i] + hi) = wv[0];
                    }
                    if (item == 0) *scale[i] = ldexpf(1.f, power);
                }
            } else if (dst[i]) {
                vec xo, yo;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    xo[e] = (T)u[e];
                    yo[e] = (T)v[e];
                }
                *(vec*)((T*)dst[i] + lo) = xo;
                *(vec*)((T*)dst[i] + hi) = yo;
            }
        }
    }
}

template <typename T>
static hipError_t launch_append_type(AppendParams a, bool eight, hipStream_t stream) {
    RotaryParams& p = a.p;
    p.items = p.items / (2 * Vec16<T>::n);   // (came as head_dim)
    p.fd_items = make_fastdiv((uint32_t)p.items);
    p.fd_tokens = make_fastdiv((uint32_t)p.n_tokens);
    const int64_t tokens = (int64_t)p.batch * p.n_tokens, per_block = 256 / p.items, blocks = (tokens + per_block - 1) / per_block;
    const int heads = p.heads[0] + p.heads[1] + p.heads[2];
    p.head_chunk = head_chunk(blocks, heads, kOwnHeads);
    const int64_t chunks = (heads + p.head_chunk - 1) / p.head_chunk, row = std::max<int64_t>(1, std::min<int64_t>(blocks, 65536 / chunks));
    const dim3 grid((unsigned)(chunks * row), (unsigned)((blocks + row - 1) / row));
    // Workgroups that run beside each other take what lies beside each other: the heads of a token, or its neighbours (2 x 8 191 tokens of 48 heads with rotated halves,
    // token by token in memory, us: heads first 82, tokens first 87; head by head: 77 and 72).
    const int32_t heads_first = p.in[1].stride_h < p.in[1].stride_n;
    const FastDiv fd_inner = make_fastdiv((uint32_t)(heads_first ? chunks : row));
    if (p.axes > 1) {
        if (eight) hipLaunchKernelGGL((cache_append_kernel<T, true, true>), grid, dim3(256), 0, stream, p, a.k_scale, a.v_scale, fd_inner, (int32_t)row, heads_first);
        else hipLaunchKernelGGL((cache_append_kernel<T, true, false>), grid, dim3(256), 0, stream, p, a.k_scale, a.v_scale, fd_inner, (int32_t)row, heads_first);
    } else {
        if (eight) hipLaunchKernelGGL((cache_append_kernel<T, false, true>), grid, dim3(256), 0, stream, p, a.k_scale, a.v_scale, fd_inner, (int32_t)row, heads_first);
        else hipLaunchKernelGGL((cache_append_kernel<T, false, false>), grid, dim3(256), 0, stream, p, a.k_scale, a.v_scale, fd_inner, (int32_t)row, heads_first);
    }
    return hipGetLastError();
}

hipError_t launch_cache_append(const AppendParams& a, grat_dtype dtype, bool eight, hipStream_t stream) {
    if (dtype == GRAT_BF16) return launch_append_type<__bf16>(a, eight, stream);
    if (dtype == GRAT_F16) return launch_append_type<_Float16>(a, eight, stream);
    return launch_append_type<float>(a, eight, stream);
}

// 16 numbers of a row a thread.
template <typename T>
__global__ __launch_bounds__(256) void cache_read_kernel(ReadParams p) {
    constexpr int V = Vec16<T>::n;
    typedef typename Vec16<T>::type vec;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= p.pieces) return;
    uint32_t row, piece, bh, n, b, h;
    fdivmod((uint32_t)at, p.fd_items, row, piece);
    fdivmod(row, p.fd_rows, bh, n);
    fdivmod(bh, p.fd_heads, b, h);
    T* const dst = (T*)p.out.data + b * p.out.stride_b + h * p.out.stride_h + n * p.out.stride_n + 16 * piece;
    float x[16];
    if (!p.k_len || (int)n < p.k_len[b]) {
        const uint4 raw = *(const uint4*)(p.cache.data + b * p.cache.stride_b + h * p.cache.stride_h + n * p.cache.stride_n + 16 * piece);
        const float s = ((const float*)p.scale.data)[b * p.scale.stride_b + h * p.scale.stride_h + n * p.scale.stride_n];
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 u = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), v = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
            x[4 * i] = u[0] * s;
            x[4 * i + 1] = u[1] * s;
            x[4 * i + 2] = v[0] * s;
            x[4 * i + 3] = v[1] * s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < 16; i += V) {
        vec o;
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = (T)x[i + e];
        *(vec*)(dst + i) = o;
    }
}

hipError_t launch_cache_read(const ReadParams& p, grat_dtype dtype, hipStream_t stream) {
    const dim3 grid((unsigned)((p.pieces + 255) / 256));
    if (dtype == GRAT_BF16) hipLaunchKernelGGL((cache_read_kernel<__bf16>), grid, dim3(256), 0, stream, p);
    else if (dtype == GRAT_F16) hipLaunchKernelGGL((cache_read_kernel<_Float16>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((cache_read_kernel<float>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace grat
