// Rotary positions: Q and K of a sequence or a grid turned pair by pair, and the new tokens of a cache appended.
//
// y = R(position) x on pairs of elements; the gradient is the rotation the other way, R^T.  Every element is read and
// written once and the table's 8 bytes a pair are shared by all heads of a token, so memory bandwidth bounds it.
// A thread owns one piece of a token's rows, two 16-byte vectors that hold whole pairs (interleaved: neighbours; half: `rot / 2`
// elements apart), reads its cos and sin once and walks a few heads with them, all their loads in flight ahead of
// the first store.  Measured (a copy reaches 5.3 TB/s at these sizes): 2 x 8 191 tokens of 40 heads in bf16, half of the head turned, 66 us,
// 5.1 TB/s; a grid of 115 200 tokens, 48 heads in half, 567 us, 5.0 TB/s; a token each of 32 sequences appended in 5.4 us a call,
// 3.8 of them the kernel's.
#include <algorithm>

#include "sequence_common.h"

namespace grat {

template <typename T, bool AXES>
__device__ __forceinline__ void pair_angles(const RotaryParams& p, int b, int n, int pair0, float* cs, float* sn) {
    constexpr int V = Vec16<T>::n;
    const float2* const table = (const float2*)p.table;
    const int pairs = p.rot / 2;
    auto row = [&](int pos) { return (int64_t)min(max(pos, 0), p.n_pos - 1) * pairs; };
    if constexpr (AXES) {
        const int32_t* at = p.positions + b * p.positions_stride_b + (int64_t)n * p.axes;
        int64_t r[3];
#pragma unroll
        for (int a = 0; a < 3; ++a) r[a] = row(at[min(a, p.axes - 1)]);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int pair = pair0 + e;
            const float2 v = table[(pair < p.axis_end[0] ? r[0] : pair < p.axis_end[1] ? r[1] : r[2]) + pair];
            cs[e] = v.x;
            sn[e] = p.inverse ? -v.y : v.y;
        }
    } else {
        // (start + n may leave 32 bits; what does is far outside the table either way)
        const int64_t pos = p.positions ? (int64_t)p.positions[b * p.positions_stride_b + n] : (int64_t)(p.start ? p.start[b] : 0) + n;
        const float4* src = (const float4*)(table + row((int)min((int64_t)p.n_pos, pos)) + pair0);   // (rows are whole 16-byte vectors)
#pragma unroll
        for (int e = 0; e < V; e += 2) {
            const float4 v = src[e / 2];
            cs[e] = v.x;
            sn[e] = p.inverse ? -v.y : v.y;
            cs[e + 1] = v.z;
            sn[e + 1] = p.inverse ? -v.w : v.w;
        }
    }
}

constexpr int kHeads = 4;   // in flight at a time

template <typename T, bool AXES>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p) {
    typedef typename Vec16<T>::type vec;
    constexpr int V = Vec16<T>::n;
    const uint32_t tid = threadIdx.x;
    uint32_t slot, item, b, n;
    fdivmod(tid, p.fd_items, slot, item);
    const uint32_t per_block = 256u / (uint32_t)p.items;
    if (slot >= per_block) return;
    const uint32_t token = blockIdx.x * per_block + slot;
    if (token >= (uint32_t)p.batch * (uint32_t)p.n_tokens) return;
    fdivmod(token, p.fd_tokens, b, n);

    // elements of the piece's two vectors; pieces behind the rotated ones are neighbours and pass through
    const int turned = p.rot / (2 * V);
    const bool turn = (int)item < turned;
    const int lo = turn && !p.interleaved ? (int)item * V : (int)item * 2 * V;
    const int hi = turn && !p.interleaved ? lo + p.rot / 2 : lo + V;
    float cs[V], sn[V];
    if (turn) pair_angles<T, AXES>(p, (int)b, (int)n, (int)item * V, cs, sn);

    const int all = p.heads[0] + p.heads[1] + p.heads[2];
    const int cache_row = p.n_cache > 0 ? p.start[b] : 0;
    for (int h0 = blockIdx.y * p.head_chunk, h1 = min(all, h0 + p.head_chunk); h0 < h1; h0 += kHeads) {
        vec x[kHeads], y[kHeads];
        T* dst[kHeads];
        bool turns[kHeads];
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            int h = min(h0 + i, h1 - 1), t = 0;
            if (h >= p.heads[0]) { h -= p.heads[0]; t = 1; if (h >= p.heads[1]) { h -= p.heads[1]; t = 2; } }
            // (uniform; an index into the parameters would put them into scratch memory)
            const SeqTensor in = t == 0 ? p.in[0] : t == 1 ? p.in[1] : p.in[2], out = t == 0 ? p.out[0] : t == 1 ? p.out[1] : p.out[2];
            const T* src = (const T*)in.data + b * in.stride_b + h * in.stride_h + n * in.stride_n;
            int64_t row = n;
            bool keep = h0 + i < h1;
            if (p.n_cache > 0 && t > 0) {
                row = (int64_t)cache_row + n;
                keep = keep && row >= 0 && row < p.n_cache;
            }
            turns[i] = turn && t < 2;
            T* const d = (T*)out.data + b * out.stride_b + h * out.stride_h + row * out.stride_n;
            if (!turns[i] && d == src) keep = false;   // in place: nothing to do
            dst[i] = keep ? d : nullptr;
            x[i] = *(const vec*)(src + lo);
            y[i] = *(const vec*)(src + hi);
        }
#pragma unroll
        for (int i = 0; i < kHeads; ++i) {
            if (turns[i]) {
                if (p.interleaved) {
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        const float a = (float)x[i][e], c = (float)x[i][e + 1], a2 = (float)y[i][e], c2 = (float)y[i][e + 1];
                        const int q = e / 2, q2 = V / 2 + e / 2;
                        x[i][e] = (T)(cs[q] * a - sn[q] * c);
                        x[i][e + 1] = (T)(sn[q] * a + cs[q] * c);
                        y[i][e] = (T)(cs[q2] * a2 - sn[q2] * c2);
                        y[i][e + 1] = (T)(sn[q2] * a2 + cs[q2] * c2);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float a = (float)x[i][e], c = (float)y[i][e];
                        x[i][e] = (T)(cs[e] * a - sn[e] * c);
                        y[i][e] = (T)(sn[e] * a + cs[e] * c);
                    }
                }
            }
            if (dst[i]) {
                *(vec*)(dst[i] + lo) = x[i];
                *(vec*)(dst[i] + hi) = y[i];
            }
        }
    }
}

template <typename T>
static hipError_t launch_rotary_type(RotaryParams p, hipStream_t stream) {
    p.items = p.items / (2 * Vec16<T>::n);   // (came as head_dim)
    p.fd_items = make_fastdiv((uint32_t)p.items);
    p.fd_tokens = make_fastdiv((uint32_t)p.n_tokens);
    const int64_t tokens = (int64_t)p.batch * p.n_tokens, per_block = 256 / p.items;
    const int64_t blocks = (tokens + per_block - 1) / per_block;
    const int heads = p.heads[0] + p.heads[1] + p.heads[2];
    // Heads of a thread, which share its cos and sin: multiples of kHeads, as many as leave the chip 4 096 workgroups.  (One head a thread: 115 200
    // tokens of 48 heads on a grid 761 us against 567; 8 191 tokens of 40 heads 66.6 against 65.8; a token each of 32 sequences 5.4 both ways.)
    const int64_t want = std::max<int64_t>(1, blocks * heads / 4096);
    p.head_chunk = (int)std::min<int64_t>(heads, (want + kHeads - 1) / kHeads * kHeads);
    const dim3 grid((unsigned)blocks, (unsigned)((heads + p.head_chunk - 1) / p.head_chunk));
    if (p.axes > 1) hipLaunchKernelGGL((rotary_kernel<T, true>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((rotary_kernel<T, false>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_rotary(const RotaryParams& p, grat_dtype dtype, hipStream_t stream) {
    if (dtype == GRAT_BF16) return launch_rotary_type<__bf16>(p, stream);
    if (dtype == GRAT_F16) return launch_rotary_type<_Float16>(p, stream);
    return launch_rotary_type<float>(p, stream);
}

struct TableParams {
    grat_rotary_spec spec;
    int32_t n_pos, pairs, axes, axis_end[3];
    float* table;
};

// Once a model: pow, sincos and a division in fp64 for every entry bound it.  131 072 positions of 64 pairs, 67 MB: 84 us a call (writing them takes 14).
__global__ __launch_bounds__(256) void rotary_table_kernel(TableParams p) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)p.n_pos * p.pairs) return;
    const int64_t n = i / p.pairs;
    const int pair = (int)(i - n * p.pairs);
    const int axis = pair < p.axis_end[0] ? 0 : pair < p.axis_end[1] ? 1 : 2;
    const int begin = axis == 0 ? 0 : p.axis_end[axis - 1], count = p.axis_end[axis] - begin;
    const grat_rotary_spec& s = p.spec;
    double base = s.base;
    if (s.scaling == GRAT_ROTARY_BASE && count > 1) base *= pow(s.factor, (double)count / (count - 1));
    double f = pow(base, -(double)(pair - begin) / count);
    if (s.scaling == GRAT_ROTARY_LINEAR) f /= s.factor;
    if (s.scaling == GRAT_ROTARY_RAMP) {
        const double turns = s.trained * f / 6.283185307179586476925286766559;
        const double w = fmin(1.0, fmax(0.0, (turns - s.low) / (s.high - s.low)));
        f *= w + (1.0 - w) / s.factor;
    }
    double sn, cs;
    sincos((double)n * f, &sn, &cs);
    ((float2*)p.table)[i] = make_float2((float)(s.magnitude * cs), (float)(s.magnitude * sn));
}

hipError_t launch_rotary_table(const grat_rotary_spec& spec, int32_t n_pos, int32_t axes, const int32_t* axis_pairs, float* d_table,
                               hipStream_t stream) {
    TableParams p{spec, n_pos, 0, axes, {}, d_table};
    for (int a = 0; a < 3; ++a) {
        if (a < axes) p.pairs += axis_pairs[a];
        p.axis_end[a] = p.pairs;
    }
    const int64_t blocks = ((int64_t)n_pos * p.pairs + 255) / 256;
    hipLaunchKernelGGL(rotary_table_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace grat
