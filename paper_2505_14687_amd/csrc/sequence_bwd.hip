// The lists of a gradient turned round: for every key block the groups that list it, and the parts they are cut into (see sequence_bwd.h).
#include "sequence_attn.h"

namespace grat {

// Half: the exponent that dS of a K/V head is formed with (see sequence_bwd.h), by a workgroup of THREADS.
template <int THREADS>
__device__ __forceinline__ void put_head_bits(const GradParams& g, int bh) {
    __shared__ int s_least[THREADS / 64];
    const int32_t* const runs = g.row_bits + (int64_t)bh * g.head_runs;
    int least = 0x7fffffff;
#pragma unroll 8
    for (int i = threadIdx.x; i < g.head_runs; i += THREADS) least = min(least, runs[i]);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) least = min(least, __shfl_xor(least, m));
    if ((threadIdx.x & 63) == 0) s_least[threadIdx.x >> 6] = least;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < THREADS / 64; ++w) least = min(least, s_least[w]);
        g.head_bits[bh] = least - 1;
    }
    __syncthreads();
}

__global__ __launch_bounds__(256) void grad_head_bits_kernel(GradParams g) { put_head_bits<256>(g, (int)blockIdx.x); }

void launch_grad_head_bits(const GradParams& g, hipStream_t stream) {
    hipLaunchKernelGGL(grad_head_bits_kernel, dim3((unsigned)g.heads), dim3(256), 0, stream, g);
}

// The bitmap, cleared (by a kernel: recorded into graphs like any other launch), and half's exponents.
__global__ __launch_bounds__(256) void grad_clear_kernel(GradParams g) {
    if (g.row_bits)
        for (int bh = (int)blockIdx.x; bh < g.heads; bh += (int)gridDim.x) put_head_bits<256>(g, bh);
    const int64_t n = (int64_t)g.blocks * g.words;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) g.bits[i] = 0;
}

// A bit for every listed block with a key that the group sees.
__global__ __launch_bounds__(256) void grad_bits_kernel(SelParams p, GradParams g, int64_t entries) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= entries) return;
    uint32_t list, t, bh, group;
    fdivmod((uint32_t)at, g.fd_top, list, t);
    if ((int)t >= p.count[list]) return;
    const int block = p.index[at];
    if (block < 0 || block >= p.s.n_blocks) return;
    fdivmod(list, p.fd_groups, bh, group);
    const int b = (int)fdiv(bh, p.fd_kv_heads), len = seq_len(p.s, b);
    if (block * p.s.block >= group_seen(p.s, len, seq_pos(p.s, b, len), (int)group)) return;
    atomicOr(&g.bits[((int64_t)bh * p.s.n_blocks + block) * g.words + group / 32], 1u << (group % 32));
}

// Rows of a block are cut into parts of about p.part_rows.  Long ones go to the front of `parts`, short ones to its back: the launch ends with these.
__device__ __forceinline__ int parts_of(const SelParams& p, const GradParams& g, int n) {
    return max(1, (int)fdiv((uint32_t)(n * p.rows) + (uint32_t)g.part_rows - 1u, g.fd_part));   // (a block's rows and a part's are below 2^30)
}
__device__ __forceinline__ bool is_long(const SelParams& p, const GradParams& g, int n) { return 2u * (uint32_t)(n * p.rows) >= (uint32_t)g.part_rows; }
// What a block of n groups takes: groups, long parts, slots, places in `joins`, short parts.
__device__ __forceinline__ int takes(const SelParams& p, const GradParams& g, int n, int what) {
    const int parts = parts_of(p, g, n);
    return what == 0 ? n : what == 1 ? (is_long(p, g, n) ? parts : 0) : what == 4 ? (is_long(p, g, n) ? 0 : parts) : parts == 1 ? 0 : what == 2 ? parts : 1;
}
// Writes a block's groups, ascending, and its parts to the places `at` (one wave).
__device__ __forceinline__ void put_block(const SelParams& p, const GradParams& g, int block, int n, const uint32_t* words, const int (&at)[5], int lane) {
    int to = at[0];
    for (int w = 0; w < g.words; w += 2) {   // a group a lane
        const uint64_t bits = words[w] | (uint64_t)(w + 1 < g.words ? words[w + 1] : 0) << 32;
        if (bits >> lane & 1) g.groups[to + __popcll(bits & ((1ull << lane) - 1ull))] = 32 * w + lane;
        to += __popcll(bits);
    }
    const int parts = parts_of(p, g, n), part0 = is_long(p, g, n) ? at[1] : g.most_parts - 1 - at[4];   // (a short part is its block's only one)
    const uint32_t rows = (uint32_t)(n * p.rows), per = ((rows + parts - 1) / (uint32_t)parts + 63u) & ~63u;   // whole tiles of 64 rows
    for (int k = lane; k < parts; k += 64) {
        g.parts[part0 + k] = make_int4(block, at[0], (int)min((uint32_t)k * per, rows), (int)min((uint32_t)(k + 1) * per, rows));
        g.part_slot[part0 + k] = parts > 1 ? at[2] + k : -1;
    }
    if (parts > 1 && lane == 0) g.joins[at[3]] = make_int4(block, at[2], parts, 0);
}

// A workgroup takes kListBlocks blocks, a wave a block at a time; it asks for its share of `groups`, `parts`, `slots` and `joins` once.
// Where that lies depends on the order of the workgroups, what is computed from it does not.
constexpr int kListBlocks = 4;   // (a block a wave: 226 blocks of 7 223 groups in 16s step 375 us, in 4s 318; 4 096 blocks 1 600 and 1 591)

__global__ __launch_bounds__(256) void grad_lists_kernel(SelParams p, GradParams g) {
    __shared__ int s_n[kListBlocks], s_at[5][kListBlocks];
    const int block0 = (int)blockIdx.x * kListBlocks, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int here = min(kListBlocks, g.blocks - block0);
    for (int i = wave; i < here; i += 4) {
        const uint32_t* const words = g.bits + (int64_t)(block0 + i) * g.words;
        int n = 0;
        for (int w = lane; w < g.words; w += 64) n += __popc(words[w]);
#pragma unroll
        for (int m = 1; m < 64; m *= 2) n += __shfl_xor(n, m);
        if (lane == 0) s_n[i] = n;
    }
    __syncthreads();
    if (threadIdx.x < 5) {
        const int what = threadIdx.x;
        int sum = 0;
        for (int i = 0; i < here; ++i) sum += takes(p, g, s_n[i], what);
        int at = sum > 0 ? atomicAdd(&g.counters[what], sum) : 0;
        for (int i = 0; i < here; ++i) {
            s_at[what][i] = at;
            at += takes(p, g, s_n[i], what);
        }
    }
    __syncthreads();
    for (int i = wave; i < here; i += 4) {
        const int at[5] = {s_at[0][i], s_at[1][i], s_at[2][i], s_at[3][i], s_at[4][i]};
        put_block(p, g, block0 + i, s_n[i], g.bits + (int64_t)(block0 + i) * g.words, at, lane);
    }
}

// The same, bits included, where a head's lists have so few entries (8 192) that every workgroup can read all of them: one launch instead of three.  A
// workgroup takes kHeadBlocks blocks of a head, their bits in LDS.  (One against three, a training step: 2 047 tokens 67.5 and 72.3 us, 16 384 in groups
// of 64 1 406 and 1 427.  On 30 shapes of 512 to 16 384 entries, 2, 8 and 16 heads, one is 1 to 4 % ahead up to 8 192 - behind by 1 % once, 8 heads of 256
// groups x 32 - and -0.4 to 2 % at 16 384; at 28 892, 7 223 queries, 419 and 387.)
constexpr int kHeadBlocks = 64;

__global__ __launch_bounds__(1024) void grad_head_lists_kernel(SelParams p, GradParams g) {
    extern __shared__ uint32_t s_bits[];   // [kHeadBlocks][words]
    __shared__ int s_at[5][kHeadBlocks], s_n[kHeadBlocks];
    const SeqShape& s = p.s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bh = (int)blockIdx.y, block0 = (int)blockIdx.x * kHeadBlocks;
    const int blocks = min(kHeadBlocks, s.n_blocks - block0);
    if (g.row_bits && blockIdx.x == 0) put_head_bits<1024>(g, bh);
    for (int i = threadIdx.x; i < blocks * g.words; i += 1024) s_bits[i] = 0;
    const int b = (int)fdiv((uint32_t)bh, p.fd_kv_heads), len = seq_len(s, b);
    const int64_t pos = seq_pos(s, b, len);
    __syncthreads();
    const int64_t list0 = (int64_t)bh * s.n_groups;
    for (int i = threadIdx.x; i < s.n_groups * p.max_blocks; i += 1024) {
        uint32_t group, t;
        fdivmod((uint32_t)i, g.fd_top, group, t);
        const int block = p.index[list0 * p.max_blocks + i], at = block - block0;
        if ((int)t < p.count[list0 + group] && block >= block0 && at < blocks && block * s.block < group_seen(s, len, pos, (int)group))
            atomicOr(&s_bits[at * g.words + group / 32], 1u << (group % 32));
    }
    __syncthreads();
    for (int i = wave; i < blocks; i += 16) {
        int n = 0;
        for (int w = lane; w < g.words; w += 64) n += __popc(s_bits[i * g.words + w]);
#pragma unroll
        for (int m = 1; m < 64; m *= 2) n += __shfl_xor(n, m);
        if (lane == 0) s_n[i] = n;
    }
    __syncthreads();
    if (wave < 5) {   // places: within the workgroup, then the workgroup's
        static_assert(kHeadBlocks == 64, "a block a lane");
        const int mine = lane < blocks ? takes(p, g, s_n[lane], wave) : 0;
        int before = mine;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const int up = __shfl_up(before, m);
            if (lane >= m) before += up;
        }
        const int sum = __shfl(before, 63);
        int base = 0;
        if (lane == 0 && sum > 0) base = atomicAdd(&g.counters[wave], sum);
        s_at[wave][lane] = __shfl(base, 0) + before - mine;
    }
    __syncthreads();
    for (int i = wave; i < blocks; i += 16) {
        const int at[5] = {s_at[0][i], s_at[1][i], s_at[2][i], s_at[3][i], s_at[4][i]};
        put_block(p, g, bh * s.n_blocks + block0 + i, s_n[i], s_bits + i * g.words, at, lane);
    }
}

void launch_grad_lists(const SelParams& p, const GradParams& g, hipStream_t stream) {
    const int64_t lds = 4 * (int64_t)kHeadBlocks * g.words;
    if (lds <= 64 * 1024 && (int64_t)p.s.n_groups * p.max_blocks <= 8192) {
        hipLaunchKernelGGL(grad_head_lists_kernel, dim3((unsigned)((p.s.n_blocks + kHeadBlocks - 1) / kHeadBlocks), (unsigned)(p.s.batch * p.s.kv_heads)),
                           dim3(1024), (size_t)lds, stream, p, g);
        return;
    }
    const int64_t clears = ((int64_t)g.blocks * g.words + 1023) / 1024;
    hipLaunchKernelGGL(grad_clear_kernel, dim3((unsigned)(clears < 2048 ? clears : 2048)), dim3(256), 0, stream, g);
    const int64_t entries = (int64_t)p.s.batch * p.s.kv_heads * p.s.n_groups * p.max_blocks;
    hipLaunchKernelGGL(grad_bits_kernel, dim3((unsigned)((entries + 255) / 256)), dim3(256), 0, stream, p, g, entries);
    hipLaunchKernelGGL(grad_lists_kernel, dim3((unsigned)((g.blocks + kListBlocks - 1) / kListBlocks)), dim3(256), 0, stream, p, g);
}

}  // namespace grat
