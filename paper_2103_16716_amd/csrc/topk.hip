// The k best experts of each token, and the sort of the (token, choice) pairs
// by expert: routing with k experts a token.
//
// Pair p = t k + j is choice j of token t. perm lists the pairs expert after
// expert, in ascending order within one (a stable sort); slots is its inverse:
// pair p stands in row slots[p]. Pairs without an expert (index out of [0, E))
// come after all others as -1. With k = 1 and an expert for every token this is
// the sort vector of Fig. 2's caption.
//
//   route_small_kernel  everything, in one block: few tokens
//   topk_count_kernel   the choices of a block's tokens, and how many of its pairs
//                       each expert has
//   pair_count_kernel   the same counts for choices that are given
//   pair_scan_kernel    E > 512: per expert, the pairs in earlier blocks
//   pair_place_kernel   offsets, perm and slots
#include "common.hpp"
#include "internal.hpp"

namespace base {
namespace {

constexpr int kBlocks = 256;     // blocks of tokens, at most: one per compute unit
constexpr int kThreads = 1024;
constexpr int kScanFrom = 512;   // experts above which a kernel of its own scans the counts

// Tokens per block, the same for every kernel of a call.
int64_t block_tokens(int64_t T) { return (T + kBlocks - 1) / kBlocks; }

// ------------------------------------------------------------------ choice --

// A score and its expert as one number in [1, 2) of 64 bits, whose order is: higher
// score first, then the lower expert; both zeros are equal. The mantissa holds the
// order-preserving image of the score, 0 for one that is never chosen (-inf, NaN),
// and 2047 - e. As numbers, two keys are ordered by one instruction each for the
// larger and the smaller.
__device__ inline double score_key(float x, int e) {
    const uint32_t ord = x > -INFINITY ? f32_ord(x == 0.0f ? 0.0f : x) : 0u;
    const uint64_t bits = 0x3ff0000000000000ull | (uint64_t)ord << 20 | (uint64_t)(2047 - e);
    return __builtin_bit_cast(double, bits);
}
__device__ inline uint32_t key_ord(double k) {
    return (uint32_t)(__builtin_bit_cast(uint64_t, k) >> 20);
}
__device__ inline int key_expert(double k) {
    return 2047 - (int)(__builtin_bit_cast(uint64_t, k) & 2047);
}

__device__ inline void order(double &a, double &b) {   // the larger first
    const double hi = __builtin_fmax(a, b);
    b = __builtin_fmin(a, b);
    a = hi;
}

// Bitonic networks over registers, descending.
template <int L>
__device__ inline void merge_bitonic(double (&a)[L]) {
#pragma unroll
    for (int s = L / 2; s > 0; s >>= 1)
#pragma unroll
        for (int i = 0; i < L; ++i)
            if ((i & s) == 0) order(a[i], a[i | s]);
}
template <int L>
__device__ inline void sort_descending(double (&a)[L]) {
#pragma unroll
    for (int n = 2; n <= L; n <<= 1)
#pragma unroll
        for (int s = n / 2; s > 0; s >>= 1)
#pragma unroll
            for (int i = 0; i < L; ++i)
                if ((i & s) == 0) {
                    if ((i & n) == 0 || n == L) order(a[i], a[i | s]);
                    else order(a[i | s], a[i]);
                }
}
// a: the L largest of two descending lists.
template <int L>
__device__ inline void merge_lists(double (&a)[L], const double (&b)[L]) {
#pragma unroll
    for (int i = 0; i < L; ++i) a[i] = __builtin_fmax(a[i], b[L - 1 - i]);
    merge_bitonic(a);
}

template <int kControl>
__device__ inline double move_in_row(double x) {
    const uint64_t v = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, kControl, 0xf, 0xf, true);
    const uint32_t hi =
        __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), kControl, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int kControl, int L>
__device__ inline void merge_from(double (&a)[L]) {
    double b[L];
#pragma unroll
    for (int i = 0; i < L; ++i) b[i] = move_in_row<kControl>(a[i]);
    merge_lists(a, b);
}

// The L best of a lane's share of a row of E <= 4 G C scores: four consecutive experts per
// step of 4 G.
template <int G, int C, int L>
__device__ inline void best_of_lane(const float *__restrict__ row, int E, int g,
                                    double (&best)[L]) {
    constexpr int V = 4 * C;
    float v[V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int e = 4 * (g + G * c);
        float4 x = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        if (E % 4 == 0) {
            if (e < E) x = *reinterpret_cast<const float4 *>(row + e);
        } else {
            if (e < E) x.x = row[e];
            if (e + 1 < E) x.y = row[e + 1];
            if (e + 2 < E) x.z = row[e + 2];
            if (e + 3 < E) x.w = row[e + 3];
        }
        v[4 * c] = x.x, v[4 * c + 1] = x.y, v[4 * c + 2] = x.z, v[4 * c + 3] = x.w;
    }
#pragma unroll
    for (int s = 0; s < V; s += L) {
        double more[L];
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int e = 4 * (g + G * ((s + i) >> 2)) + ((s + i) & 3);
            more[i] = s + i < V ? score_key(v[s + i < V ? s + i : 0], e < E ? e : 2047) : 0.0;
        }
        sort_descending(more);
        if (s == 0) {
#pragma unroll
            for (int i = 0; i < L; ++i) best[i] = more[i];
        } else {
            merge_lists(best, more);
        }
    }
}

// The L best of a row, in every one of the G lanes (16 or 64) that share it: lists are merged
// with those of lanes further round (a row of 16 lanes turns by 8, 4, 2, 1).
template <int G, int C, int L>
__device__ inline void best_of_row(const float *__restrict__ row, int E, int g, double (&best)[L]) {
    best_of_lane<G, C, L>(row, E, g, best);
    merge_from<0x128>(best);
    merge_from<0x124>(best);
    merge_from<0x122>(best);
    merge_from<0x121>(best);
    if constexpr (G == 64) {
#pragma unroll
        for (int off = 16; off < 64; off <<= 1) {
            double b[L];
#pragma unroll
            for (int i = 0; i < L; ++i) b[i] = __shfl_xor(best[i], off);
            merge_lists(best, b);
        }
    }
}

// The same of two rows by 16 lanes, the first's in the lower eight and the second's in the
// upper: half as many merges a row, which in this order (8 round, the mirror of eight, 2, 1)
// meet all eight lanes. 131072 tokens, 8 of 64: 37.9 us one at a time, 31.6; 65536, 8 of 256:
// 38.6 and 36.1.
template <int C, int L>
__device__ inline void best_of_two_rows(const float *__restrict__ row, const float *__restrict__ row2,
                                        int E, int g, double (&best)[L]) {
    double other[L];
    best_of_lane<16, C, L>(row, E, g, best);
    best_of_lane<16, C, L>(row2, E, g, other);
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const double give = g < 8 ? other[i] : best[i];
        best[i] = g < 8 ? best[i] : other[i];
        other[i] = move_in_row<0x128>(give);
    }
    merge_lists(best, other);
    merge_from<0x141>(best);
    merge_from<0x4e>(best);
    merge_from<0xb1>(best);
}

// More choices than the lists hold: k rounds, each of which takes the best of the row and
// removes it. Bound by the rounds' chains of maxima over the lanes: 32768 tokens, 16 of 64
// 21.5 us, 16 of 256 44.4; 8192, 33 of 1000 82.9; 4096, 64 of 2048 149.
template <int G, int C, class Emit>
__device__ inline void best_in_rounds(const float *__restrict__ row, int E, int k, int g,
                                      Emit emit) {
    constexpr int V = 4 * C;
    double key[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = 4 * (g + G * (i >> 2)) + (i & 3);
        key[i] = score_key(e < E ? row[e] : -INFINITY, e < E ? e : 2047);
    }
    for (int j = 0; j < k; ++j) {
        double best = 0.0;
#pragma unroll
        for (int i = 0; i < V; ++i) best = __builtin_fmax(best, key[i]);
#pragma unroll
        for (int off = G / 2; off > 0; off >>= 1)
            best = __builtin_fmax(best, __shfl_xor(best, off));
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (key[i] == best) key[i] = 0.0;
        emit(j, best);
    }
}

// The choices of tokens [t0, t1) by a block of kT threads: assign and scores, each pair's
// expert counted in hist [E + 1] and handed to `keep`.
template <int kT, int G, int C, int L, class Keep>
__device__ inline void choose(const float *__restrict__ S, int64_t t0, int64_t t1, int E, int k,
                              int32_t *__restrict__ assign, float *__restrict__ scores,
                              int32_t *hist, Keep keep) {
    const int g = threadIdx.x % G;
    const auto emit_of = [&](int64_t t, int j, double key) {
        const uint32_t ord = key_ord(key);
        const int a = ord != 0 ? key_expert(key) : -1;
        assign[t * k + j] = a;
        if (scores != nullptr) scores[t * k + j] = ord != 0 ? f32_unord(ord) : -INFINITY;
        if (hist != nullptr) atomicAdd(&hist[a >= 0 ? a : E], 1);
        keep(t * k + j, a >= 0 ? a : E);
    };
    if constexpr (G == 16 && L == 8) {
        if (t1 - t0 > kT / G) {   // more than one round of the block: two tokens at a time
            for (int64_t tb = t0; tb < t1; tb += kT / G * 2) {
                const int64_t t = tb + threadIdx.x / G * 2;
                const int64_t mine = t + (g >> 3);
                double best[L];
                best_of_two_rows<C, L>(S + (t < t1 ? t : t0) * E, S + (t + 1 < t1 ? t + 1 : t0) * E,
                                       E, g, best);
                double key = best[0];
#pragma unroll
                for (int i = 1; i < L; ++i)
                    if ((g & 7) == i) key = best[i];
                if (mine < t1 && (g & 7) < k) emit_of(mine, g & 7, key);
            }
            return;
        }
    }
    for (int64_t tb = t0; tb < t1; tb += kT / G) {
        const int64_t t = tb + threadIdx.x / G;
        const bool live = t < t1;
        const float *row = S + (live ? t : t0) * E;
        const auto emit = [&](int j, double key) { emit_of(t, j, key); };
        if constexpr (L > 0) {
            double best[L];
            best_of_row<G, C, L>(row, E, g, best);
            double mine = best[0];   // lane j emits choice j
#pragma unroll
            for (int i = 1; i < L; ++i)
                if (g == i) mine = best[i];
            if (live && g < k) emit(g, mine);
        } else {
            best_in_rounds<G, C>(row, E, k, g, [&](int j, double key) {
                if (live && g == 0) emit(j, key);
            });
        }
    }
}

// Threads of a block: half as many where a lane's 32 scores need the registers.
template <int C>
constexpr int kChoosers = C > 4 ? kThreads / 2 : kThreads;

template <int G, int C, int L>
__global__ __launch_bounds__(kChoosers<C>) void topk_count_kernel(
    const float *__restrict__ S, int64_t T, int E, int k, int64_t tokens,
    int32_t *__restrict__ assign, float *__restrict__ scores, int32_t *__restrict__ counts) {
    extern __shared__ int32_t hist[];   // [E + 1]
    for (int e = threadIdx.x; e <= E; e += kChoosers<C>) hist[e] = 0;
    __syncthreads();
    const int64_t t0 = blockIdx.x * tokens;
    choose<kChoosers<C>, G, C, L>(S, t0, t0 + tokens < T ? t0 + tokens : T, E, k, assign, scores,
                                  hist, [](int64_t, int) {});
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += kChoosers<C>)
        counts[(int64_t)blockIdx.x * (E + 1) + e] = hist[e];
}

// ------------------------------------------------------------------- order --

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
        counts[(int64_t)blockIdx.x * (E + 1) + e] = hist[e];
}

// A thread per expert (and one for the pairs without): counts become the pairs of earlier
// blocks, totals the pairs of all. 14 us for 1024 or 2048 experts of 256 blocks: few waves, each
// with a chain of loads.
__global__ __launch_bounds__(64) void pair_scan_kernel(int32_t *__restrict__ counts,
                                                       int32_t *__restrict__ totals, int bins,
                                                       int blocks) {
    const int e = blockIdx.x * 64 + threadIdx.x;
    if (e >= bins) return;
    int sum = 0;
    for (int b0 = 0; b0 < blocks; b0 += 16) {
        int n[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
            n[i] = b0 + i < blocks ? counts[(int64_t)(b0 + i) * bins + e] : 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (b0 + i < blocks) counts[(int64_t)(b0 + i) * bins + e] = sum;
            sum += n[i];
        }
    }
    totals[e] = sum;
}

// Exclusive sum over the block's threads.
template <int kWaves>
__device__ inline int scan_threads(int own, int *wave_sum) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = own;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(sum, off);
        if (lane >= off) sum += o;
    }
    if (lane == 63) wave_sum[wave] = sum;
    __syncthreads();
    int at = sum - own;
    for (int w = 0; w < wave; ++w) at += wave_sum[w];
    return at;
}

// Places a block's pairs [p0, p1). total[e] is the pairs of expert e in all blocks, before[e]
// those in earlier ones (LDS; before null: none). A wave owns a run of the pairs: it counts
// them per expert in its row of `next` [kWaves][E + 1], which then becomes the row of its
// first pair of each expert. It then takes 64 pairs at a time: a lane's rank is the number
// of lower lanes with the same expert, found with one ballot per bit.
template <int kWaves, class Expert>
__device__ inline void place(int64_t p0, int64_t p1, int E, const int32_t *total,
                             const int32_t *before, int32_t *next, int *wave_sum, Expert expert,
                             int32_t *__restrict__ perm, int32_t *__restrict__ slots,
                             int32_t *__restrict__ offsets) {
    constexpr int kT = 64 * kWaves;
    const int bins = E + 1;
    const int lane = threadIdx.x & 63;
    for (int i = threadIdx.x; i < kWaves * bins; i += kT) next[i] = 0;
    const int per = (bins + kT - 1) / kT;
    const int e0 = threadIdx.x * per;
    const int e1 = e0 + per < bins ? e0 + per : bins;
    int sum = 0;
    for (int e = e0; e < e1; ++e) sum += total[e];
    int first = scan_threads<kWaves>(sum, wave_sum);   // (a barrier behind the clearing, too)
    const int64_t run = ((p1 - p0 + kWaves - 1) / kWaves + 63) / 64 * 64;
    const int64_t q0 = p0 + (threadIdx.x >> 6) * run;
    const int64_t q1 = q0 + run < p1 ? q0 + run : p1;
    int32_t *mine = next + (threadIdx.x >> 6) * bins;
    for (int64_t p = q0 + lane; p < q1; p += 64) atomicAdd(&mine[expert(p)], 1);
    __syncthreads();
    for (int e = e0; e < e1; ++e) {
        if (offsets != nullptr) offsets[e] = first;
        int row = first + (before == nullptr ? 0 : before[e]);
        for (int w = 0; w < kWaves; ++w) {
            const int n = next[w * bins + e];
            next[w * bins + e] = row;
            row += n;
        }
        first += total[e];
    }
    __syncthreads();
    const int bits = 32 - __clz(E);
    for (int64_t pb = q0; pb < q1; pb += 64) {
        const int64_t p = pb + lane;
        const bool live = p < q1;
        const int e = live ? expert(p) : E;
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

// totals null: every block adds up the counts of all blocks, [blocks][E + 1], for itself
// (up to 512 experts and 256 blocks that is less than a launch); else they have been scanned.
template <int kWaves>
__global__ __launch_bounds__(64 * kWaves) void pair_place_kernel(
    const int32_t *__restrict__ assign, int64_t N, int E, int64_t pairs,
    const int32_t *__restrict__ counts, const int32_t *__restrict__ totals,
    int32_t *__restrict__ perm, int32_t *__restrict__ slots, int32_t *__restrict__ offsets) {
    extern __shared__ int32_t lds[];
    __shared__ int wave_sum[kWaves];
    constexpr int kT = 64 * kWaves;
    const int bins = E + 1;
    int32_t *total = lds, *before = lds + bins, *next = lds + 2 * bins;
    if (totals == nullptr) {
        for (int e = threadIdx.x; e < 2 * bins; e += kT) lds[e] = 0;
        __syncthreads();
        // Groups of 64-aligned threads take a part of the blocks each.
        const int wide = (bins + 63) / 64 * 64;
        const int groups = kT / wide > 0 ? kT / wide : 1;
        const int part = ((int)gridDim.x + groups - 1) / groups;
        const int g = threadIdx.x / wide;
        const int e = threadIdx.x - g * wide;
        if (g < groups && e < bins) {
            const int b0 = g * part;
            const int b1 = b0 + part < (int)gridDim.x ? b0 + part : (int)gridDim.x;
            int all = 0, early = 0;
#pragma unroll 16
            for (int b = b0; b < b1; ++b) {
                const int n = counts[(int64_t)b * bins + e];
                all += n;
                early += b < (int)blockIdx.x ? n : 0;
            }
            atomicAdd(&total[e], all);
            atomicAdd(&before[e], early);
        }
    } else {
        for (int e = threadIdx.x; e < bins; e += kT) {
            total[e] = totals[e];
            before[e] = counts[(int64_t)blockIdx.x * bins + e];
        }
    }
    __syncthreads();
    const int64_t p0 = blockIdx.x * pairs;
    const int64_t p1 = p0 + pairs < N ? p0 + pairs : N;
    place<kWaves>(p0, p1, E, total, before, next, wave_sum,
                  [&](int64_t p) { return pair_expert(assign, p, E); }, perm, slots,
                  blockIdx.x == 0 ? offsets : nullptr);
}

// Few tokens: the latency of launches is what counts, so one block does it all and keeps the
// pairs' experts in LDS. us in a graph, one block and two launches: 64 tokens, 2 of 64 experts
// 4.5 and 10; 256 tokens 7.6 and 10.1; 128 tokens, 8 of 256 11.5 and 15; 256 tokens 19.9 and
// 16.7, so by the scores as well.
constexpr int kSmallTokens = 256;
constexpr int kSmallPairs = 2048;
constexpr int kSmallScores = 32768;

template <int G, int C, int L>
__global__ __launch_bounds__(kThreads) void route_small_kernel(
    const float *__restrict__ S, int T, int E, int k, int32_t *__restrict__ assign,
    float *__restrict__ scores, int32_t *__restrict__ perm, int32_t *__restrict__ slots,
    int32_t *__restrict__ offsets) {
    extern __shared__ int32_t lds[];   // [1 + 16][E + 1]
    __shared__ int wave_sum[kThreads / 64];
    __shared__ uint16_t of_pair[kSmallPairs];
    for (int e = threadIdx.x; e <= E; e += kThreads) lds[e] = 0;
    __syncthreads();
    choose<kThreads, G, C, L>(S, 0, T, E, k, assign, scores, lds,
                              [&](int64_t p, int e) { of_pair[p] = (uint16_t)e; });
    __syncthreads();
    place<kThreads / 64>(0, (int64_t)T * k, E, lds, nullptr, lds + E + 1, wave_sum,
                         [&](int64_t p) { return (int)of_pair[p]; }, perm, slots, offsets);
}

// ---------------------------------------------------------------- launches --

struct RouteCall {
    const float *S;
    int64_t T, E, k, tokens, blocks;
    int32_t *assign;
    float *scores;
    int32_t *perm, *slots, *offsets, *counts;
};

bool is_small(int64_t T, int64_t E, int64_t k) {
    return T <= kSmallTokens && T * k <= kSmallPairs && T * E <= kSmallScores && E <= kScanFrom;
}

template <int G, int C, int L>
void choose_as(const RouteCall &c, hipStream_t s) {
    if constexpr (4 * G * C <= 1024)
        if (is_small(c.T, c.E, c.k)) {
            hipLaunchKernelGGL((route_small_kernel<G, C, L>), dim3(1), dim3(kThreads),
                               (size_t)(c.E + 1) * 4 * (1 + kThreads / 64), s, c.S, (int)c.T,
                               (int)c.E, (int)c.k, c.assign, c.scores, c.perm, c.slots,
                               c.offsets);
            return;
        }
    hipLaunchKernelGGL((topk_count_kernel<G, C, L>), dim3((unsigned)c.blocks),
                       dim3(kChoosers<C>), (size_t)(c.E + 1) * 4, s, c.S, c.T, (int)c.E, (int)c.k,
                       c.tokens, c.assign, c.scores, c.counts);
}
template <int G, int C>
void choose_for(const RouteCall &c, hipStream_t s) {
    if (c.k <= 2) choose_as<G, C, 2>(c, s);
    else if (c.k <= 8) choose_as<G, C, 8>(c, s);
    else choose_as<G, C, 0>(c, s);
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
    int32_t *totals = E > kScanFrom ? counts + (E + 1) * blocks : nullptr;
    const RouteCall c = {S, T, E, k, tokens, blocks, assign, scores, perm, slots, offsets, counts};
    if (S == nullptr)
        hipLaunchKernelGGL(pair_count_kernel, dim3((unsigned)blocks), dim3(kThreads),
                           (size_t)(E + 1) * 4, s, assign, T * k, (int)E, tokens * k, counts);
    else if (E <= 64) choose_for<16, 1>(c, s);
    else if (E <= 128) choose_for<16, 2>(c, s);
    else if (E <= 256) choose_for<16, 4>(c, s);
    else if (E <= 1024) choose_for<64, 4>(c, s);
    else choose_for<64, 8>(c, s);
    if (S != nullptr && is_small(T, E, k)) return hipGetLastError();
    if (totals != nullptr) {
        hipLaunchKernelGGL(pair_scan_kernel, dim3((unsigned)((E + 64) / 64)), dim3(64), 0, s,
                           counts, totals, (int)(E + 1), (int)blocks);
        hipLaunchKernelGGL(pair_place_kernel<4>, dim3((unsigned)blocks), dim3(256),
                           (size_t)(E + 1) * 4 * 6, s, assign, T * k, (int)E, tokens * k, counts,
                           totals, perm, slots, offsets);
    } else {
        hipLaunchKernelGGL(pair_place_kernel<16>, dim3((unsigned)blocks), dim3(kThreads),
                           (size_t)(E + 1) * 4 * 18, s, assign, T * k, (int)E, tokens * k, counts,
                           totals, perm, slots, offsets);
    }
    return hipGetLastError();
}

}  // namespace base
