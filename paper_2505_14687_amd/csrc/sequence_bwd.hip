// The lists of a gradient turned round: for every key block the groups that list it, and the parts they are cut into (see sequence_bwd.h).
#include "sequence_attn.h"

namespace grat {

// A bit for every listed block with a key that the group sees.
__global__ __launch_bounds__(256) void grad_bits_kernel(SelParams p, GradParams g, int64_t entries, FastDiv fd_top) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= entries) return;
    uint32_t list, t, bh, group;
    fdivmod((uint32_t)at, fd_top, list, t);
    if ((int)t >= p.count[list]) return;
    const int block = p.index[at];
    if (block < 0 || block >= p.s.n_blocks) return;
    fdivmod(list, p.fd_groups, bh, group);
    const int b = (int)fdiv(bh, p.fd_kv_heads), len = seq_len(p.s, b);
    if (block * p.s.block >= group_seen(p.s, len, seq_pos(p.s, b, len), (int)group)) return;
    atomicOr(&g.bits[((int64_t)bh * p.s.n_blocks + block) * g.words + group / 32], 1u << (group % 32));
}

// A block's groups, ascending, and its parts.  One wave a block; where in `groups`, `parts` and `slots` a block's share lies depends on the
// order of the waves, what is computed from it does not.
__global__ __launch_bounds__(256) void grad_lists_kernel(SelParams p, GradParams g) {
    const int block = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (block >= g.blocks) return;
    const uint32_t* const words = g.bits + (int64_t)block * g.words;
    int n = 0;
    for (int w = lane; w < g.words; w += 64) n += __popc(words[w]);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) n += __shfl_xor(n, m);
    const int64_t rows = (int64_t)n * p.rows;
    const int parts = (int)max((int64_t)1, (rows + g.part_rows - 1) / g.part_rows);
    int first = 0, part0 = 0, slot0 = 0;
    if (lane == 0) {
        first = n > 0 ? atomicAdd(&g.counters[0], n) : 0;
        part0 = atomicAdd(&g.counters[1], parts);
        if (parts > 1) slot0 = atomicAdd(&g.counters[2], parts);
        g.joins[block] = make_int2(slot0, parts);
    }
    first = __shfl(first, 0);
    part0 = __shfl(part0, 0);
    slot0 = __shfl(slot0, 0);
    int at = first;
    for (int w0 = 0; w0 < g.words; w0 += 64) {
        uint32_t bits = w0 + lane < g.words ? words[w0 + lane] : 0;
        const int mine = __popc(bits);
        int before = mine;   // inclusive prefix sum
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const int up = __shfl_up(before, m);
            if (lane >= m) before += up;
        }
        int to = at + before - mine;
        while (bits) {
            g.groups[to++] = (w0 + lane) * 32 + __builtin_ctz(bits);
            bits &= bits - 1;
        }
        at += __shfl(before, 63);
    }
    const int64_t per = ((rows + parts - 1) / parts + 63) & ~(int64_t)63;   // whole tiles of 64 rows
    for (int i = lane; i < parts; i += 64) {
        g.parts[part0 + i] = make_int4(block, first, (int)min((int64_t)i * per, rows), (int)min((int64_t)(i + 1) * per, rows));
        g.part_slot[part0 + i] = parts > 1 ? slot0 + i : -1;
    }
}

void launch_grad_lists(const SelParams& p, const GradParams& g, hipStream_t stream) {
    const int64_t entries = (int64_t)p.s.batch * p.s.kv_heads * p.s.n_groups * p.max_blocks;
    hipLaunchKernelGGL(grad_bits_kernel, dim3((unsigned)((entries + 255) / 256)), dim3(256), 0, stream, p, g, entries,
                       make_fastdiv((uint32_t)p.max_blocks));
    hipLaunchKernelGGL(grad_lists_kernel, dim3((unsigned)((g.blocks + 3) / 4)), dim3(256), 0, stream, p, g);
}

}  // namespace grat
