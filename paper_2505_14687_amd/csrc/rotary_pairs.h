// What the kernels that turn pairs by their positions share.
#pragma once
#include "sequence_common.h"

namespace grat {

// cos and sin of the V pairs from pair0 on, of token n of sequence b.
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

// Heads of a thread, which share its cos and sin: multiples of `own`, as many as leave the chip 4 096 workgroups.
inline int head_chunk(int64_t blocks, int heads, int own) {
    const int64_t want = blocks * heads / 4096 > 1 ? blocks * heads / 4096 : 1, chunk = (want + own - 1) / own * own;
    return (int)(chunk < heads ? chunk : heads);
}

}  // namespace grat
