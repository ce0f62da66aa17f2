// The k best experts of each token, and the sort of the (token, choice) pairs
// by expert: routing with k experts a token.
//
// Pair p = t k + j is choice j of token t. perm lists the pairs expert after
// expert, in ascending order within one (a stable sort); slots is its inverse:
// pair p stands in row slots[p]. Pairs without an expert (index out of [0, E))
// come after all others as -1. With k = 1 and an expert for every token this is
// the sort vector of Fig. 2's caption.
//
//   topk_count_kernel  the choices of a block's tokens, and how many of its pairs
//                      each expert has
//   pair_count_kernel  the same counts for choices that are given
//   pair_scan_kernel   per expert, the pairs in earlier blocks
//   pair_place_kernel  offsets, perm and slots
#include "common.hpp"
#include "internal.hpp"

namespace base {
namespace {

constexpr int kBlocks = 512;     // blocks of tokens, at most
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// Tokens per block, the same for every kernel of a call.
int64_t block_tokens(int64_t T) { return (T + kBlocks - 1) / kBlocks; }

// Scores in an order of unsigned integers: 0 for those that are never chosen
// (-inf and NaN), and equal for the two zeros.
__device__ inline uint32_t score_key(float x) {
    if (!(x > -INFINITY)) return 0;
    return f32_ord(x == 0.0f ? 0.0f : x);
}

// G lanes hold the E <= 4 G C scores of a token, four consecutive experts per
// lane and step of 4 G. Each of k rounds takes the largest (score, lowest expert)
// of the lanes' own largest and removes it.
template <int G, int C>
__global__ __launch_bounds__(kThreads) void topk_count_kernel(
    const float *__restrict__ S, int T, int E, int k, int tokens, int32_t *__restrict__ assign,
    float *__restrict__ scores, int32_t *__restrict__ counts) {
    extern __shared__ int32_t hist[];   // [E + 1]
    constexpr int V = 4 * C;
    for (int e = threadIdx.x; e <= E; e += kThreads) hist[e] = 0;
    __syncthreads();
    const int g = threadIdx.x % G;
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int64_t t1 = t0 + tokens < T ? t0 + tokens : T;
    for (int64_t tb = t0; tb < t1; tb += kThreads / G) {
        const int64_t t = tb + threadIdx.x / G;
        const bool live = t < t1;
        const float *row = S + (live ? t : t0) * E;
        uint32_t key[V];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int e = 4 * (g + G * c);
            if (E % 4 == 0) {
                float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                if (e < E) v = *reinterpret_cast<const float4 *>(row + e);
                key[4 * c] = score_key(v.x);
                key[4 * c + 1] = score_key(v.y);
                key[4 * c + 2] = score_key(v.z);
                key[4 * c + 3] = score_key(v.w);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    key[4 * c + i] = e + i < E ? score_key(row[e + i]) : 0;
            }
        }
        for (int j = 0; j < k; ++j) {
            uint32_t best = 0;
            int bi = 0;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (key[i] > best) {
                    best = key[i];
                    bi = i;
                }
            int be = 4 * (g + G * (bi >> 2)) + (bi & 3);
#pragma unroll
            for (int off = G / 2; off > 0; off >>= 1) {
                const uint32_t ob = __shfl_xor(best, off);
                const int oe = __shfl_xor(be, off);
                if (ob > best || (ob == best && oe < be)) {
                    best = ob;
                    be = oe;
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (4 * (g + G * (i >> 2)) + (i & 3) == be) key[i] = 0;
            if (g == 0 && live) {
                const bool has = best != 0;
                assign[t * k + j] = has ? be : -1;
                if (scores != nullptr) scores[t * k + j] = has ? f32_unord(best) : -INFINITY;
                atomicAdd(&hist[has ? be : E], 1);
            }
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += kThreads)
        counts[(int64_t)e * gridDim.x + blockIdx.x] = hist[e];
}

__device__ inline int pair_expert(const int32_t *assign, int64_t p, int E) {
    const int a = assign[p];
    return a >= 0 && a < E ? a : E;
}

__global__ __launch_bounds__(kThreads) void pair_count_kernel(const int32_t *__restrict__ assign,
                                                              int64_t N, int E, int64_t pairs,
                                                              int32_t *__restrict__ counts) {
    extern __shared__ int32_t hist[];
    for (int e = threadIdx.x; e <= E; e += kThreads) hist[e] = 0;
    __syncthreads();
    const int64_t p0 = blockIdx.x * pairs;
    const int64_t p1 = p0 + pairs < N ? p0 + pairs : N;
    for (int64_t p = p0 + threadIdx.x; p < p1; p += kThreads)
        atomicAdd(&hist[pair_expert(assign, p, E)], 1);
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += kThreads)
        counts[(int64_t)e * gridDim.x + blockIdx.x] = hist[e];
}

// One wave per expert (and one for the pairs without): counts become the pairs
// of earlier blocks, totals the pairs of all.
__global__ __launch_bounds__(64) void pair_scan_kernel(int32_t *__restrict__ counts,
                                                       int32_t *__restrict__ totals, int blocks) {
    int32_t *row = counts + (int64_t)blockIdx.x * blocks;
    const int lane = threadIdx.x;
    int carry = 0;
    for (int b0 = 0; b0 < blocks; b0 += 64) {
        const int b = b0 + lane;
        const int own = b < blocks ? row[b] : 0;
        int sum = own;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(sum, off);
            if (lane >= off) sum += o;
        }
        if (b < blocks) row[b] = carry + sum - own;
        carry += __shfl(sum, 63);
    }
    if (lane == 0) totals[blockIdx.x] = carry;
}

// A wave owns a run of the block's pairs. first[e] is the row of the block's
// first pair of expert e; the waves' own counts make of it the row of each
// wave's first. A wave then takes 64 pairs at a time: a lane's rank is the number
// of lower lanes with the same expert, found with one ballot per bit.
__global__ __launch_bounds__(kThreads) void pair_place_kernel(
    const int32_t *__restrict__ assign, int64_t N, int E, int64_t pairs,
    const int32_t *__restrict__ counts, const int32_t *__restrict__ totals,
    int32_t *__restrict__ perm, int32_t *__restrict__ slots, int32_t *__restrict__ offsets) {
    extern __shared__ int32_t lds[];
    __shared__ int wave_sum[kWaves];
    const int bins = E + 1;
    int32_t *next = lds;   // [kWaves][bins]
    const int lane = threadIdx.x & 63;
    const int wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < kWaves * bins; i += kThreads) next[i] = 0;
    // Exclusive scan of the totals, a run of bins per thread.
    const int per = (bins + kThreads - 1) / kThreads;
    const int e0 = threadIdx.x * per;
    const int e1 = e0 + per < bins ? e0 + per : bins;
    int sum = 0;
    for (int e = e0; e < e1; ++e) sum += totals[e];
    int scan = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(scan, off);
        if (lane >= off) scan += o;
    }
    if (lane == 63) wave_sum[wave] = scan;
    __syncthreads();
    int first = scan - sum;
    for (int w = 0; w < wave; ++w) first += wave_sum[w];
    const int64_t p0 = blockIdx.x * pairs;
    const int64_t p1 = p0 + pairs < N ? p0 + pairs : N;
    const int64_t run = ((pairs + kWaves - 1) / kWaves + 63) / 64 * 64;
    const int64_t q0 = p0 + wave * run;
    const int64_t q1 = q0 + run < p1 ? q0 + run : p1;
    int32_t *mine = next + wave * bins;
    for (int64_t p = q0 + lane; p < q1; p += 64) atomicAdd(&mine[pair_expert(assign, p, E)], 1);
    __syncthreads();
    for (int e = e0; e < e1; ++e) {
        if (blockIdx.x == 0) offsets[e] = first;
        int row = first + counts[(int64_t)e * gridDim.x + blockIdx.x];
        for (int w = 0; w < kWaves; ++w) {
            const int n = next[w * bins + e];
            next[w * bins + e] = row;
            row += n;
        }
        first += totals[e];
    }
    __syncthreads();
    const int bits = 32 - __clz(E);
    for (int64_t pb = q0; pb < q1; pb += 64) {
        const int64_t p = pb + lane;
        const bool live = p < q1;
        const int e = live ? pair_expert(assign, p, E) : E;
        uint64_t same = __ballot(live);
        for (int b = 0; b < bits; ++b) {
            const uint64_t m = __ballot((e >> b) & 1);
            same &= (e >> b) & 1 ? m : ~m;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        const int row = live ? mine[e] + rank : 0;
        __builtin_amdgcn_wave_barrier();
        if (live && rank == 0) mine[e] += __popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (live) {
            perm[row] = e < E ? (int32_t)p : -1;
            slots[p] = e < E ? row : -1;
        }
    }
}

template <int G, int C>
void run_topk(const float *S, int64_t T, int64_t E, int64_t k, int64_t tokens, int64_t blocks,
              int32_t *assign, float *scores, int32_t *counts, hipStream_t s) {
    hipLaunchKernelGGL((topk_count_kernel<G, C>), dim3((unsigned)blocks), dim3(kThreads),
                       (size_t)(E + 1) * 4, s, S, (int)T, (int)E, (int)k, (int)tokens, assign,
                       scores, counts);
}

}  // namespace

size_t topk_workspace_size(int64_t T, int64_t E, int64_t) {
    const int64_t tokens = block_tokens(T);
    const int64_t blocks = (T + tokens - 1) / tokens;
    return ((size_t)(E + 1) * (size_t)(blocks + 1) * 4 + 255) / 256 * 256;
}

hipError_t launch_topk(const float *S, int64_t T, int64_t E, int64_t k, int32_t *assign,
                       float *scores, int32_t *perm, int32_t *slots, int32_t *offsets,
                       void *workspace, hipStream_t s) {
    const int64_t tokens = block_tokens(T);
    const int64_t blocks = (T + tokens - 1) / tokens;
    int32_t *counts = static_cast<int32_t *>(workspace);
    int32_t *totals = counts + (E + 1) * blocks;
    if (S == nullptr) {
        hipLaunchKernelGGL(pair_count_kernel, dim3((unsigned)blocks), dim3(kThreads),
                           (size_t)(E + 1) * 4, s, assign, T * k, (int)E, tokens * k, counts);
    } else if (E <= 64) {
        run_topk<16, 1>(S, T, E, k, tokens, blocks, assign, scores, counts, s);
    } else if (E <= 128) {
        run_topk<16, 2>(S, T, E, k, tokens, blocks, assign, scores, counts, s);
    } else if (E <= 256) {
        run_topk<16, 4>(S, T, E, k, tokens, blocks, assign, scores, counts, s);
    } else if (E <= 512) {
        run_topk<64, 2>(S, T, E, k, tokens, blocks, assign, scores, counts, s);
    } else {
        run_topk<64, 8>(S, T, E, k, tokens, blocks, assign, scores, counts, s);
    }
    hipLaunchKernelGGL(pair_scan_kernel, dim3((unsigned)(E + 1)), dim3(64), 0, s, counts, totals,
                       (int)blocks);
    hipLaunchKernelGGL(pair_place_kernel, dim3((unsigned)blocks), dim3(kThreads),
                       (size_t)(E + 1) * 4 * kWaves, s, assign, T * k, (int)E, tokens * k, counts,
                       totals, perm, slots, offsets);
    return hipGetLastError();
}

}  // namespace base
