// What a list of key blocks comes from: mean keys, scores of query groups for blocks, and the selection.
#include <algorithm>

#include "sequence_common.h"

namespace grat {

// ---- means -----------------------------------------------------------------------------------
// Means of runs of rows: key blocks (one head, rows of the tensor up to the sequence's valid keys) and query groups (the heads
// that share a K/V head, rows up to n_q).  Bound by reading the rows once.  A workgroup per run: a thread owns a 16-byte
// column and every RL-th row, sums in fp32, and the row lanes are added up through LDS in a fixed order.  Measured: Q of 32 768 tokens, 32 heads,
// bf16, in groups of 64: 268 MB in 50 us, 5.4 TB/s.
struct MeanParams {
    SeqShape s;
    SeqTensor x;
    int32_t runs, share, run_rows;   // runs per head of the result, heads and rows of a run
    int32_t of_keys;                 // rows end at the sequence's valid keys, else at n_q
    int32_t n_new;                   // keys: only runs with one of the last n_new valid keys, 0: all
    float* out;
};

template <typename T, int D>
__global__ __launch_bounds__(256) void run_means_kernel(MeanParams p) {
    typedef typename Vec16<T>::type vec;
    constexpr int V = Vec16<T>::n, C = D / V, RL = 256 / C;
    __shared__ float part[RL][D + 4];
    const int tid = threadIdx.x, col = tid % C, rl = tid / C;
    const int bh = blockIdx.y, b = bh / p.s.kv_heads, h = bh - b * p.s.kv_heads;
    const int rows = p.of_keys ? seq_len(p.s, b) : p.s.n_q;
    int run = blockIdx.x;
    if (p.n_new > 0) {
        if (rows == 0) return;
        run += max(0, rows - p.n_new) / p.run_rows;
        if ((int64_t)run * p.run_rows >= rows) return;
    }
    const int row0 = run * p.run_rows, n = max(0, min(p.run_rows, rows - row0));
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.f;
    for (int i = 0; i < p.share; ++i) {
        const T* src = (const T*)p.x.data + b * p.x.stride_b + (int64_t)(h * p.share + i) * p.x.stride_h + col * V;
#pragma unroll 4
        for (int r = rl; r < n; r += RL) {
            const vec v = *(const vec*)(src + (int64_t)(row0 + r) * p.x.stride_n);
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += (float)v[e];
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) part[rl][col * V + e] = sum[e];
    __syncthreads();
    if (tid < D) {
        float total = 0.f;
#pragma unroll
        for (int r = 0; r < RL; ++r) total += part[r][tid];
        p.out[((int64_t)bh * p.runs + run) * D + tid] = n > 0 ? total / (float)(n * p.share) : 0.f;
    }
}

// Groups of few queries: C lanes a run, each all of its rows, so that a workgroup takes 256 / C runs and nothing is joined.  (Key blocks stay with the
// other kernel, also short ones: means of some blocks have the bits that all blocks' have.)
constexpr int kShortRun = 16;   // rows; 4: 8 192 lists x 8 heads 118 -> 59 us with the scores (118 MB: 18), 16: 73 -> 27 (x 2 heads), 32: 20 -> 22

template <typename T, int D>
__global__ __launch_bounds__(256) void short_run_means_kernel(MeanParams p) {
    typedef typename Vec16<T>::type vec;
    constexpr int V = Vec16<T>::n, C = D / V;
    const int col = threadIdx.x % C, run = (int)blockIdx.x * (256 / C) + threadIdx.x / C;
    if (run >= p.runs) return;
    const int bh = blockIdx.y, b = bh / p.s.kv_heads, h = bh - b * p.s.kv_heads;
    const int row0 = run * p.run_rows, n = min(p.run_rows, p.s.n_q - row0);
    const T* const src = (const T*)p.x.data + b * p.x.stride_b + (int64_t)h * p.share * p.x.stride_h + (int64_t)row0 * p.x.stride_n + col * V;
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.f;
    int i = 0, r = 0;   // head and row
    for (int left = n * p.share; left > 0; left -= 8) {
        vec v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {   // (behind the last row: it again, and not added)
            v[k] = *(const vec*)(src + (int64_t)i * p.x.stride_h + (int64_t)r * p.x.stride_n);
            if (k + 1 < left && ++r == n) {
                r = 0;
                ++i;
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += k < left ? (float)v[k][e] : 0.f;
    }
    float* const out = p.out + ((int64_t)bh * p.runs + run) * D + col * V;
    const float all = (float)(n * p.share);
#pragma unroll
    for (int e = 0; e < V; e += 4) *(float4*)(out + e) = make_float4(sum[e] / all, sum[e + 1] / all, sum[e + 2] / all, sum[e + 3] / all);
}

template <typename T>
static hipError_t launch_means_type(const MeanParams& p, int head_dim, int runs, hipStream_t stream) {
    const int heads = p.s.batch * p.s.kv_heads;
    if (!p.of_keys && (int64_t)p.run_rows * p.share <= kShortRun) {
        const int per = 256 * Vec16<T>::n / head_dim;
        const dim3 grid((unsigned)((runs + per - 1) / per), (unsigned)heads);
        if (head_dim == 128) hipLaunchKernelGGL((short_run_means_kernel<T, 128>), grid, dim3(256), 0, stream, p);
        else hipLaunchKernelGGL((short_run_means_kernel<T, 64>), grid, dim3(256), 0, stream, p);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)runs, (unsigned)heads);
    if (head_dim == 128) hipLaunchKernelGGL((run_means_kernel<T, 128>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((run_means_kernel<T, 64>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}
static hipError_t launch_means(const MeanParams& p, grat_dtype dtype, int head_dim, int runs, hipStream_t stream) {
    if (dtype == GRAT_BF16) return launch_means_type<__bf16>(p, head_dim, runs, stream);
    if (dtype == GRAT_F16) return launch_means_type<_Float16>(p, head_dim, runs, stream);
    return launch_means_type<float>(p, head_dim, runs, stream);
}

hipError_t launch_block_means(const SeqShape& s, const SeqTensor& K, grat_dtype dtype, int32_t head_dim, int32_t n_new, float* d_means,
                              hipStream_t stream) {
    const MeanParams p{s, K, s.n_blocks, 1, s.block, 1, n_new, d_means};
    const int64_t touched = n_new > 0 ? std::min<int64_t>(s.n_blocks, ((int64_t)n_new + s.block - 2) / s.block + 1) : s.n_blocks;
    return launch_means(p, dtype, head_dim, (int)touched, stream);
}

// ---- scores ----------------------------------------------------------------------------------
struct ScoreParams {
    SeqShape s;
    SeqTensor q;
    const float* q_means;   // [batch * kv_heads][n_groups][D] (large launches)
    const float* means;
    float* scores;
    float scale;
};

// Few queries: a matrix-vector product, bound by reading the means once.  A workgroup takes 64 blocks of one K/V head; it forms the
// groups' mean queries itself, from few rows, and D / 4 lanes share a block.  Measured: 16 sequences of 1 024 blocks, 8 heads: 68 MB in
// 16 us, 4.2 TB/s.  (As a matrix product, with a launch for the mean queries, the call takes 38 us against 19.)
constexpr int kThinRows = 64;     // query rows of a K/V head up to which launches are thin
constexpr int kThinBlocks = 64;

template <typename T, int D>
__global__ __launch_bounds__(256) void thin_scores_kernel(ScoreParams p) {
    constexpr int L = D / 4, SLOTS = 256 / L;
    __shared__ float qm[kThinRows][D];
    const SeqShape& s = p.s;
    const int tid = threadIdx.x, bh = blockIdx.y, b = bh / s.kv_heads, h = bh - b * s.kv_heads;
    const int lane = tid % L, slot = tid / L;
    const float4* const M = (const float4*)p.means + (int64_t)bh * s.n_blocks * L + lane;
    const int j0 = blockIdx.x * kThinBlocks;
    constexpr int PER = kThinBlocks / SLOTS;
    float4 m[PER];   // (asked for ahead of the queries: they are what takes long)
#pragma unroll
    for (int i = 0; i < PER; ++i) m[i] = M[(int64_t)min(j0 + slot + i * SLOTS, s.n_blocks - 1) * L];
    const int len = seq_len(s, b);
    const int64_t pos = seq_pos(s, b, len);
    for (int i = tid; i < s.n_groups * D; i += 256) {
        const int g = i / D, c = i % D;
        const int r0 = g * s.q_group, n = min(s.q_group, s.n_q - r0);
        float sum = 0.f;
        for (int e = 0; e < s.share; ++e) {
            const T* src = (const T*)p.q.data + b * p.q.stride_b + (int64_t)(h * s.share + e) * p.q.stride_h + c;
            for (int r = 0; r < n; ++r) sum += (float)src[(int64_t)(r0 + r) * p.q.stride_n];
        }
        qm[g][c] = sum / (float)(n * s.share) * p.scale;
    }
    __syncthreads();
    for (int g = 0; g < s.n_groups; ++g) {
        const float4 q = *(const float4*)&qm[g][lane * 4];
        const int seen = group_seen(s, len, pos, g);
        float* const out = p.scores + ((int64_t)bh * s.n_groups + g) * s.n_blocks;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int j = j0 + slot + i * SLOTS;
            float dot = fmaf(m[i].x, q.x, fmaf(m[i].y, q.y, fmaf(m[i].z, q.z, m[i].w * q.w)));
#pragma unroll
            for (int w = 1; w < L; w *= 2) dot += __shfl_xor(dot, w);
            if (lane == 0 && j < s.n_blocks) out[j] = (int64_t)j * s.block < seen ? dot : -INFINITY;
        }
    }
}

// Many queries: a matrix product in fp32 on the fp32 matrix instruction (32x32x2), 64 groups x 64 blocks a workgroup, each of its
// four waves a quarter.  Both operands lie in LDS as rows of D floats whose 16-byte chunks are XORed with the row, so that a wave's
// b128 reads (lane = row, half of the lanes each of two chunks) spread over the banks; which k an instruction takes is free as
// long as both operands agree: element e of chunk 2 i + half.  Measured: 8 heads of 512 groups x 512 blocks 13 us, 41 TFLOP/s of the 154 that
// a large fp32 product reaches: two workgroups a compute unit, each of which waits for its tiles once.  The means before it take three times as long.
typedef __attribute__((ext_vector_type(16))) float score16;

template <int D>
__global__ __launch_bounds__(256) void scores_kernel(ScoreParams p) {
    constexpr int CH = D / 4;   // 16-byte chunks of a row
    __shared__ float4 sq[64 * CH], sm[64 * CH];
    const SeqShape& s = p.s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int bh = blockIdx.z, b = bh / s.kv_heads;
    const int g0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
    const int len = seq_len(s, b);
    const int64_t pos = seq_pos(s, b, len);
    const int most = group_seen(s, len, pos, min(g0 + 63, s.n_groups - 1));   // (later groups see more)
    score16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
    const bool any = (int64_t)j0 * s.block < most;
    if (any) {
        const float4* const Q = (const float4*)p.q_means + (int64_t)bh * s.n_groups * CH;
        const float4* const M = (const float4*)p.means + (int64_t)bh * s.n_blocks * CH;
        for (int i = tid; i < 64 * CH; i += 256) {
            const int row = i / CH, c = i % CH, to = row * CH + (c ^ (row % CH));
            sq[to] = Q[(int64_t)min(g0 + row, s.n_groups - 1) * CH + c];
            sm[to] = M[(int64_t)min(j0 + row, s.n_blocks - 1) * CH + c];
        }
        __syncthreads();
        const int qr = (wave >> 1) * 32 + (lane & 31), mr = (wave & 1) * 32 + (lane & 31), half = lane >> 5;
#pragma unroll 4
        for (int i = 0; i < CH / 2; ++i) {
            const float4 a = sq[qr * CH + ((2 * i + half) ^ (qr % CH))], m = sm[mr * CH + ((2 * i + half) ^ (mr % CH))];
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, m.x, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, m.y, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, m.z, acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, m.w, acc, 0, 0, 0);
        }
    }
    const int j = j0 + (wave & 1) * 32 + (lane & 31);
    if (j >= s.n_blocks) return;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int g = g0 + (wave >> 1) * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
        if (g < s.n_groups)
            p.scores[((int64_t)bh * s.n_groups + g) * s.n_blocks + j] =
                (int64_t)j * s.block < group_seen(s, len, pos, g) ? acc[r] * p.scale : -INFINITY;
    }
}

static bool thin(const SeqShape& s) { return (int64_t)s.n_q * s.share <= kThinRows; }

int64_t block_scores_work(const SeqShape& s, int32_t head_dim) {
    return thin(s) ? 0 : (int64_t)s.batch * s.kv_heads * s.n_groups * head_dim * (int64_t)sizeof(float);
}

template <typename T>
static void launch_thin(const ScoreParams& p, int head_dim, hipStream_t stream) {
    const dim3 grid((unsigned)((p.s.n_blocks + kThinBlocks - 1) / kThinBlocks), (unsigned)(p.s.batch * p.s.kv_heads));
    if (head_dim == 128) hipLaunchKernelGGL((thin_scores_kernel<T, 128>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((thin_scores_kernel<T, 64>), grid, dim3(256), 0, stream, p);
}

hipError_t launch_block_scores(const SeqShape& s, const SeqTensor& Q, grat_dtype dtype, int32_t head_dim, const float* d_means, float scale,
                               float* d_scores, float* d_work, hipStream_t stream) {
    const ScoreParams p{s, Q, d_work, d_means, d_scores, scale};
    if (thin(s)) {
        if (dtype == GRAT_BF16) launch_thin<__bf16>(p, head_dim, stream);
        else if (dtype == GRAT_F16) launch_thin<_Float16>(p, head_dim, stream);
        else launch_thin<float>(p, head_dim, stream);
        return hipGetLastError();
    }
    const MeanParams q{s, Q, s.n_groups, s.share, s.q_group, 0, 0, d_work};
    const hipError_t e = launch_means(q, dtype, head_dim, s.n_groups, stream);
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)((s.n_blocks + 63) / 64), (unsigned)((s.n_groups + 63) / 64), (unsigned)(s.batch * s.kv_heads));
    if (head_dim == 128) hipLaunchKernelGGL((scores_kernel<128>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((scores_kernel<64>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

// ---- selection -------------------------------------------------------------------------------
// A list is chosen by WAVES waves.  Each owns a run of 64 R consecutive blocks and holds their scores in R registers as integers that order
// like the scores; 0 is not a candidate.  The smallest selected one is found bit by bit from the highest: the largest T with at least as
// many keys >= T as are wanted; a count that is met exactly ends the search.  Keys equal to T are taken in ascending order of their
// blocks.  What is chosen is compacted by ballots, so lists ascend by construction.
//
// What bounds it is not the reading but the instructions: R ballots and R scalar counts a bit.  So where few are wanted, the common case,
// the search runs on the lanes' largest keys only and ends at the first bound that little more than `want` of them reach.  What is not
// below it (of 500 normal scores about 25 where 13 are wanted) is copied to LDS with its block, and a lane ranks one of those.  With several
// waves the best of their bounds counts, and one wave ranks.  From 4 097 blocks on (32 registers a lane and four waves, and more) the compiler keeps 132 to 482 scalar registers
// - masks of the unrolled ballots - in lanes of vector registers.  Measured: 32 768 lists of 16 from 512 blocks 28 us (46 by bits alone; reading the
// scores takes 14), 128 lists of 32 from 2 048 blocks 8.9 us a call.
struct SelectParams {
    SeqShape s;
    const float* scores;
    int32_t top, first, local;
    int32_t* count;
    int32_t* index;
    int64_t lists;
    FastDiv fd_groups, fd_kv_heads, fd_block;
};

constexpr int kFewWanted = 56;   // longest lists that are ranked

template <int WAVES, int R>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void select_blocks_kernel(SelectParams p) {
    __shared__ int s_count[2][WAVES];
    constexpr int kTwo = WAVES > 1 ? 2 : 1, kFew = 64 * kTwo;   // candidates that a lane ranks, and all of them
    __shared__ uint2 s_few[WAVES == 1 ? 4 : 1][kFew];            // key, block
    __shared__ uint32_t s_bound[2][WAVES];
    const SeqShape& s = p.s;
    const int lane = threadIdx.x & 63;
    const int wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    // (one wave a list: four lists a workgroup, which then has no barrier)
    const int64_t list = WAVES == 1 ? (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) : blockIdx.x;
    if (list >= p.lists) return;
    const float* const row = p.scores + list * s.n_blocks;
    const int j0 = wave * R * 64 + lane;   // this lane's blocks: j0 + 64 r
    float score[R];   // (asked for ahead of everything that says which of them count)
#pragma unroll
    for (int r = 0; r < R; ++r) score[r] = row[min(j0 + 64 * r, s.n_blocks - 1)];
    uint32_t bh, g;
    fdivmod((uint32_t)list, p.fd_groups, bh, g);
    const int b = (int)fdiv(bh, p.fd_kv_heads);
    const int len = seq_len(s, b);
    const int seen = group_seen(s, len, seq_pos(s, b, len), (int)g);
    const int vis = (int)fdiv((uint32_t)(seen + s.block - 1), p.fd_block);
    const int head_end = min(p.first, vis), tail = max(head_end, vis - p.local);   // [0, head_end) and [tail, vis) are in
    const int want = min(p.top - head_end - (vis - tail), tail - head_end);        // others, at most
    auto key_of = [&](int r, float x) -> uint32_t {
        const int j = j0 + 64 * r;
        x = x == 0.f ? 0.f : x;   // (-0 and 0 are equal)
        const uint32_t u = __builtin_bit_cast(uint32_t, x), order = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
        return j >= head_end && j < tail && x > -INFINITY ? order : 0;   // (false for NaN)
    };
    uint32_t held[R];
#pragma unroll
    for (int r = 0; r < R; ++r) held[r] = key_of(r, score[r]);
    int parity = 0;
    // (sum over the waves; of the waves ahead of this one)
    auto everyone = [&](int mine, int& before) {
        before = 0;
        if constexpr (WAVES == 1) {
            return mine;
        } else {
            if (lane == 0) s_count[parity][wave] = mine;
            __syncthreads();
            int all = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                if (w == wave) before = all;
                all += s_count[parity][w];
            }
            parity ^= 1;
            before = __builtin_amdgcn_readfirstlane(before);   // (the same in all lanes, which the compiler cannot know of what comes out of LDS)
            return __builtin_amdgcn_readfirstlane(all);
        }
    };
    auto count_from = [&](uint32_t t) {
        int n = 0, before;
#pragma unroll
        for (int r = 0; r < R; ++r) n += __popcll(__ballot(held[r] >= t));
        return everyone(n, before);
    };
    const uint64_t below = (1ull << lane) - 1ull;
    int32_t* const out = p.index + list * p.top;
    if constexpr (R > 1) {
        if (want > 0 && want <= kFewWanted) {
            uint32_t best = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) best = max(best, held[r]);
            auto search = [&](int least, int most) {   // a bound that this many lanes reach, or as few more than `least` as there are
                uint32_t t = 0;
#pragma unroll 1   // (unrolled, the code is fetched more slowly than it runs)
                for (int bit = 31; bit >= 0; --bit) {
                    const int n = __popcll(__ballot(best >= (t | 1u << bit)));
                    if (n >= least) t |= 1u << bit;
                    if (n >= least && n <= most) break;
                }
                return t;
            };
            uint32_t bound = search(want, want + 8);
            if constexpr (WAVES > 1) {
                // `want` keys of one wave reach the highest of the waves' bounds, and an equal share of them in every wave whose run is seen
                // as a whole the lowest of the bounds for that
                const int whole = max(1, tail / (R * 64));
                if (lane == 0) s_bound[0][wave] = bound;
                const int share = (want + whole - 1) / whole;
                const uint32_t equal = search(share, share + 1);
                if (lane == 0) s_bound[1][wave] = equal;
                __syncthreads();
                uint32_t lowest = 0xffffffffu;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    bound = max(bound, s_bound[0][w]);
                    lowest = min(lowest, w < whole ? s_bound[1][w] : lowest);
                }
                bound = __builtin_amdgcn_readfirstlane(max(bound, lowest));
            }
            int mine = 0, at;
#pragma unroll
            for (int r = 0; r < R; ++r) mine += __popcll(__ballot(held[r] >= bound));
            const int few = everyone(mine, at);
            if (bound > 0 && few <= kFew) {   // (bound = 0: no wave has `want` lanes with a candidate)
                uint2* const keys = s_few[WAVES == 1 ? threadIdx.x >> 6 : 0];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const bool in = held[r] >= bound;
                    const uint64_t all = __ballot(in);
                    if (in) keys[at + __popcll(all & below)] = make_uint2(held[r], (uint32_t)(j0 + 64 * r));
                    at += __popcll(all);
                }
                if constexpr (WAVES > 1) {
                    __syncthreads();
                    if (wave > 0) return;
                } else {
                    __builtin_amdgcn_wave_barrier();
                }
                // a lane ranks the candidates lane (+ 64): the number of larger ones
                uint2 k[kTwo];
                int rank[kTwo];
                bool in[kTwo];
                uint64_t all[kTwo];
                int have = 0;
                auto with_each = [&](auto&& f) {   // f(candidate, its number)
#pragma unroll
                    for (int u = 0; u < kTwo; ++u)
                        for (int i = 0; i < min(few - 64 * u, 64); ++i) f((uint32_t)__builtin_amdgcn_readlane(k[u].x, i), 64 * u + i);
                };
                auto take = [&]() {
                    have = 0;
#pragma unroll
                    for (int u = 0; u < kTwo; ++u) {
                        in[u] = k[u].x > 0 && rank[u] < want;
                        all[u] = __ballot(in[u]);
                        have += __popcll(all[u]);
                    }
                };
#pragma unroll
                for (int u = 0; u < kTwo; ++u) {
                    k[u] = 64 * u + lane < few ? keys[64 * u + lane] : make_uint2(0, 0);
                    rank[u] = 0;
                }
                with_each([&](uint32_t x, int) {
#pragma unroll
                    for (int u = 0; u < kTwo; ++u) rank[u] += x > k[u].x ? 1 : 0;
                });
                take();
                if (have != want) {   // the last ones taken have equals that are not: the lower blocks
                    with_each([&](uint32_t x, int i) {
#pragma unroll
                        for (int u = 0; u < kTwo; ++u) rank[u] += x == k[u].x && i < 64 * u + lane ? 1 : 0;
                    });
                    take();
                }
                const int total = head_end + want + (vis - tail);
                int at_out = head_end;
#pragma unroll
                for (int u = 0; u < kTwo; ++u) {
                    if (in[u]) out[at_out + __popcll(all[u] & below)] = (int)k[u].y;
                    at_out += __popcll(all[u]);
                }
                for (int i = lane; i < head_end; i += 64) out[i] = i;
                for (int i = lane; i < vis - tail; i += 64) out[head_end + want + i] = tail + i;
                for (int i = total + lane; i < p.top; i += 64) out[i] = -1;
                if (lane == 0) p.count[list] = total;
                return;
            }
        }
    }
    uint32_t T = 1;   // keys >= T are taken, of those equal to T only `ties`
    int ties = 0x7fffffff;
    if (want <= 0) {
        T = 0xffffffffu;   // (no score has this key)
    } else if (count_from(1) > want) {
        bool met = false;
        T = 0;
#pragma unroll 1
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t t = T | 1u << bit;
            const int n = count_from(t);
            if (n >= want) T = t;
            if (n == want) { met = true; break; }
        }
        if (!met) ties = want - count_from(T + 1);
    }
    int n = 0, tied_before;
#pragma unroll
    for (int r = 0; r < R; ++r) n += __popcll(__ballot(held[r] == T));
    everyone(n, tied_before);
    auto taken = [&](int r, int& tied) {   // tied: keys equal to T ahead of this chunk
        const int j = j0 + 64 * r;
        const uint32_t k = held[r];
        const uint64_t same = __ballot(k == T);
        const bool in = j < vis && (j < head_end || j >= tail || k > T || (k == T && tied + __popcll(same & below) < ties));
        tied += __popcll(same);
        return in;
    };
    int base = 0;
    if constexpr (WAVES > 1) {   // where this wave's part of the list begins
        int mine = 0;
#pragma unroll
        for (int r = 0, tied = tied_before; r < R; ++r) mine += __popcll(__ballot(taken(r, tied)));
        n = everyone(mine, base);
    }
#pragma unroll
    for (int r = 0, tied = tied_before; r < R; ++r) {
        const bool in = taken(r, tied);
        const uint64_t all = __ballot(in);
        if (in) out[base + __popcll(all & below)] = j0 + 64 * r;
        base += __popcll(all);
    }
    const int total = WAVES == 1 ? base : n;
    for (int i = total + (WAVES == 1 ? lane : (int)threadIdx.x); i < p.top; i += WAVES * 64) out[i] = -1;
    if (lane == 0 && wave == 0) p.count[list] = total;
}

static int64_t lists_of(const SeqShape& s) { return (int64_t)s.batch * s.kv_heads * s.n_groups; }

template <int WAVES, int R>
static void launch_select(const SelectParams& p, hipStream_t stream) {
    const int64_t blocks = WAVES == 1 ? (p.lists + 3) / 4 : p.lists;
    hipLaunchKernelGGL((select_blocks_kernel<WAVES, R>), dim3((unsigned)blocks), dim3(WAVES == 1 ? 256 : WAVES * 64), 0, stream, p);
}

// Waves that share a list: as few as hold its scores.  Waves that share one wait for each other, which costs more than the longer code of one that has more registers
// to go through (8 192 lists of 1 024 blocks: one wave 12 us, four 44; of 4 096: four 45, sixteen 247; 512 lists of 16 384: four 15, sixteen 27).  1 025 to 2 048
// blocks are the exception: two waves where there are few lists, and where a list is long enough that one wave mostly ends in the search by bits and two do
// not, unless the chip is full many times over.  2 048 blocks, us of one and of two waves: 1 024 lists of 16 8.2 and 7.7, 2 048 8.7 and 9.4, 16 384 31 and 43; lists of
// 32: 1 024 17.9 and 9.7, 2 048 18.4 and 11.7, 4 096 23 and 19, 16 384 43 and 52; lists of 48: 1 024 23 and 17, 2 048 23 and 24, 4 096 32 and 39.
static int select_waves(int n_blocks, int64_t lists, int top) {
    if (n_blocks <= 1024) return 1;
    if (n_blocks <= 2048) return lists >= 2048 && (top < 30 || top > 40 || lists >= 16384) ? 1 : 2;
    return n_blocks <= 16384 ? 4 : 8;
}
int64_t select_blocks_threads(const SeqShape& s, int32_t top) {
    const int64_t lists = lists_of(s);
    const int waves = select_waves(s.n_blocks, lists, top);
    return waves == 1 ? (lists + 3) / 4 * 256 : lists * waves * 64;
}

hipError_t launch_select_blocks(const SeqShape& s, const float* d_scores, int32_t top, int32_t first, int32_t local, int32_t* d_count,
                                int32_t* d_index, hipStream_t stream) {
    const SelectParams p{s, d_scores, top, first, local, d_count, d_index, lists_of(s),
                         make_fastdiv((uint32_t)s.n_groups), make_fastdiv((uint32_t)s.kv_heads), make_fastdiv((uint32_t)s.block)};
    const int n = s.n_blocks, waves = select_waves(n, p.lists, top);
    if (waves == 1) {
        if (n <= 64) launch_select<1, 1>(p, stream);
        else if (n <= 128) launch_select<1, 2>(p, stream);
        else if (n <= 256) launch_select<1, 4>(p, stream);
        else if (n <= 512) launch_select<1, 8>(p, stream);
        else if (n <= 1024) launch_select<1, 16>(p, stream);
        else launch_select<1, 32>(p, stream);
    } else if (waves == 2) {
        launch_select<2, 16>(p, stream);
    } else if (waves == 4) {
        if (n <= 4096) launch_select<4, 16>(p, stream);
        else if (n <= 8192) launch_select<4, 32>(p, stream);
        else launch_select<4, 64>(p, stream);
    } else {
        launch_select<8, 64>(p, stream);
    }
    return hipGetLastError();
}

}  // namespace grat
