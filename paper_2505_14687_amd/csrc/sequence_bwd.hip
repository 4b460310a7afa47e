// The lists of a gradient turned round: for every key block the groups that list it, and the parts they are cut into (see sequence_bwd.h).
#include "sequence_attn.h"

namespace grat {

// The scratch memory that has to be 0 (by a kernel: recorded into graphs like any other launch), and what rows that only fill a tile take.
__global__ __launch_bounds__(256) void grad_clear_kernel(GradParams g) {
    const int64_t n = (int64_t)g.blocks * g.words;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) g.bits[i] = 0;
    if (blockIdx.x > 0) return;
    if (threadIdx.x < 5) g.counters[threadIdx.x] = 0;
    if (threadIdx.x == 0) {
        g.delta[g.stats] = 0.f;
        g.lse2[g.stats] = INFINITY;
    }
}

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

// A block's groups, ascending, and its parts.  A workgroup takes up to kListBlocks blocks, a wave a block at a time; it asks for its share of `groups`,
// `parts` and `slots` once.  Where that lies depends on the order of the workgroups, what is computed from it does not.
constexpr int kListBlocks = 16;   // 4 in small launches, for which it is latency that counts

__global__ __launch_bounds__(256) void grad_lists_kernel(SelParams p, GradParams g, int per_group) {
    __shared__ int s_n[kListBlocks], s_at[5][kListBlocks], s_base[5];
    const int block0 = (int)blockIdx.x * per_group, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int here = min(per_group, g.blocks - block0);
    for (int i = wave; i < here; i += 4) {
        const uint32_t* const words = g.bits + (int64_t)(block0 + i) * g.words;
        int n = 0;
        for (int w = lane; w < g.words; w += 64) n += __popc(words[w]);
#pragma unroll
        for (int m = 1; m < 64; m *= 2) n += __shfl_xor(n, m);
        if (lane == 0) s_n[i] = n;
    }
    __syncthreads();
    auto parts_of = [&](int n) { return (int)max((int64_t)1, ((int64_t)n * p.rows + g.part_rows - 1) / g.part_rows); };
    // Long parts go to the front of `parts`, short ones to its back: the launch ends with these.
    auto is_long = [&](int n) { return (int64_t)n * p.rows * 2 >= (int64_t)g.part_rows; };
    if (threadIdx.x < 5) {   // groups, long parts, slots, blocks of several parts, short parts
        const int what = threadIdx.x;
        int sum = 0;
        for (int i = 0; i < here; ++i) {
            const int n = s_n[i], parts = parts_of(n);
            s_at[what][i] = sum;
            sum += what == 0 ? n : what == 1 ? (is_long(n) ? parts : 0) : what == 4 ? (is_long(n) ? 0 : parts) : parts == 1 ? 0 : what == 2 ? parts : 1;
        }
        s_base[what] = sum > 0 ? atomicAdd(&g.counters[what], sum) : 0;
    }
    __syncthreads();
    for (int i = wave; i < here; i += 4) {
        const int block = block0 + i, n = s_n[i], parts = parts_of(n);
        const int first = s_base[0] + s_at[0][i], slot0 = s_base[2] + s_at[2][i];
        const int part0 = is_long(n) ? s_base[1] + s_at[1][i] : g.most_parts - 1 - (s_base[4] + s_at[4][i]);   // (a short part is its block's only one)
        const uint32_t* const words = g.bits + (int64_t)block * g.words;
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
        const int64_t rows = (int64_t)n * p.rows, per = ((rows + parts - 1) / parts + 63) & ~(int64_t)63;   // whole tiles of 64 rows
        for (int k = lane; k < parts; k += 64) {
            g.parts[part0 + k] = make_int4(block, first, (int)min(k * per, rows), (int)min((k + 1) * per, rows));
            g.part_slot[part0 + k] = parts > 1 ? slot0 + k : -1;
        }
        if (parts > 1 && lane == 0) g.joins[s_base[3] + s_at[3][i]] = make_int4(block, slot0, parts, 0);
    }
}

void launch_grad_lists(const SelParams& p, const GradParams& g, hipStream_t stream) {
    const int64_t clears = ((int64_t)g.blocks * g.words + 1023) / 1024;
    hipLaunchKernelGGL(grad_clear_kernel, dim3((unsigned)(clears < 2048 ? clears : 2048)), dim3(256), 0, stream, g);
    const int64_t entries = (int64_t)p.s.batch * p.s.kv_heads * p.s.n_groups * p.max_blocks;
    hipLaunchKernelGGL(grad_bits_kernel, dim3((unsigned)((entries + 255) / 256)), dim3(256), 0, stream, p, g, entries,
                       make_fastdiv((uint32_t)p.max_blocks));
    const int per_group = g.blocks <= 2048 ? 4 : kListBlocks;
    hipLaunchKernelGGL(grad_lists_kernel, dim3((unsigned)((g.blocks + per_group - 1) / per_group)), dim3(256), 0, stream, p, g, per_group);
}

}  // namespace grat
