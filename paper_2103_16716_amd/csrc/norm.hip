// Layer norm of routed rows with the weights of each row's expert, and its
// gradient (the norm at the head of an expert's feed-forward block).
//
//   y = (x - m) r g_e + b_e,  m = mean(x),  r = 1 / sqrt(mean((x - m)^2) + eps)
//   with xh = (x - m) r and h = g_e dy:
//   dx = r (h - mean(h) - xh mean(h xh)),  dg_e = sum dy xh,  db_e = sum dy
//
// Row r of the routed order is row src(r) of x: r itself, or perm[r] / k when the
// sort vector is given, so that the routed copy of x need not be written. Rows
// outside every expert's range, and those without a source, are left alone. Both
// passes over a row (mean, then squares about it) run on registers. Bound by
// memory: each row is read once and written once.
//
//   norm_kernel           y, mean and rstd
//   norm_backward_kernel  dx, and sums of dy xh and dy over runs of rows
//   norm_weights_kernel   those sums added up per expert, in a fixed order
#include "common.hpp"
#include "internal.hpp"
#include "rows.hpp"

namespace base {
namespace {

// Sum over the R threads (64, or a whole block of R) that share a row.
template <int R>
__device__ inline float row_sum(float v, float *lds) {
    v = wave_sum(v);
    if constexpr (R > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < R / 64; ++w) v += lds[w];
        __syncthreads();
    }
    return v;
}

// The routed rows' sources and experts (offsets null: one expert, every row).
struct RowMap {
    const int32_t *perm, *offsets;
    int64_t x_rows;
    int N, E, k;
    __device__ int64_t source(int64_t r) const {
        if (perm == nullptr) return r;
        const int p = perm[r];
        const int64_t s = p < 0 ? -1 : p / k;
        return s < x_rows ? s : -1;
    }
    // Expert of row r, -1 for none; called by whole waves.
    __device__ int expert(int r) const {
        if (offsets == nullptr) return 0;
        if (r < offsets[0]) return -1;
        const int e = expert_of_row(offsets, E, r);
        return e < E ? e : -1;
    }
};

// R threads and up to C chunks each hold a row; a block of 256 or R threads.
template <int R>
constexpr int kBlock = R > 256 ? R : 256;

template <bool BF16, int R, int C>
__global__ __launch_bounds__(kBlock<R>) void norm_kernel(
    const void *__restrict__ x, const void *__restrict__ g, const void *__restrict__ b,
    RowMap map, void *__restrict__ y, float *__restrict__ mean, float *__restrict__ rstd, int d,
    float eps) {
    using Ck = RowChunk<BF16>;
    __shared__ float lds[16];
    const int ncs = d / Ck::kN;
    const int l = threadIdx.x % R;
    constexpr int kRows = kBlock<R> / R;
    // (r, e and src are uniform over the threads that share a row.)
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / R; r < map.N;
         r += (int64_t)gridDim.x * kRows) {
        const int e = map.expert((int)r);
        const int64_t src = map.source(r);
        if (e < 0 || src < 0) continue;
        float v[C][Ck::kN];
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int i = l + c * R;
#pragma unroll
            for (int q = 0; q < Ck::kN; ++q) v[c][q] = 0.0f;
            if (i < ncs) Ck::widen(Ck::fetch(x, src * ncs + i), v[c]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int q = 0; q < Ck::kN; ++q) sum += v[c][q];
        const float m = row_sum<R>(sum, lds) / d;
        float sq = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (l + c * R < ncs)
#pragma unroll
                for (int q = 0; q < Ck::kN; ++q) {
                    v[c][q] -= m;
                    sq = fmaf(v[c][q], v[c][q], sq);
                }
        const float rs = 1.0f / sqrtf(row_sum<R>(sq, lds) / d + eps);
        if (l == 0) {
            mean[r] = m;
            rstd[r] = rs;
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int i = l + c * R;
            if (i >= ncs) continue;
            float w[Ck::kN], o[Ck::kN];
            Ck::widen(Ck::fetch(g, (int64_t)e * ncs + i), w);
            if (b != nullptr) {
                Ck::widen(Ck::fetch(b, (int64_t)e * ncs + i), o);
            } else {
#pragma unroll
                for (int q = 0; q < Ck::kN; ++q) o[q] = 0.0f;
            }
#pragma unroll
            for (int q = 0; q < Ck::kN; ++q) o[q] = fmaf(v[c][q] * rs, w[q], o[q]);
            Ck::store(y, r * ncs + i, o);
        }
    }
}

// A block takes runs of kRun<R> consecutive rows, R threads a row, and goes through the
// experts that have rows among them. Each thread sums dy xh and dy of its own
// columns over its rows; the groups of R threads add theirs in LDS one after
// another. The sums of run p's rows of expert e go to slot p + e of the partial
// sums: p + e grows from each (run, expert) with rows in common to the next, so
// that no two share a slot.
template <int R>
constexpr int kRun = 16 * (kBlock<R> / R);

// (Two waves a SIMD, which the compiler else misses by a few registers (bf16 rows of 1032 to 2048
// keep two in memory), and the groups' sums by four columns of a lane next to each other: 32768
// rows of 2048 in bf16 87 us; with one wave 104; with the sums in the order of columns, twice the
// LDS conflicts, 91. 12 cycles of conflicts a LDS instruction are left.)
template <bool BF16, int R, int C>
__global__ __launch_bounds__(kBlock<R>, 2) void norm_backward_kernel(
    const void *dy, const void *__restrict__ x, const void *__restrict__ g,
    const float *__restrict__ mean, const float *__restrict__ rstd, const void *residual,
    RowMap map, void *dx, float *__restrict__ part, int d) {
    using Ck = RowChunk<BF16>;
    constexpr int kN = Ck::kN;
    constexpr int kGroups = kBlock<R> / R;
    extern __shared__ float sums[];   // [2][C kN / 4][R][4], more than one group only
    __shared__ float lds[16];
    const int ncs = d / kN;
    const int l = threadIdx.x % R;
    const int group = threadIdx.x / R;
    for (int64_t run = blockIdx.x; run * kRun<R> < map.N; run += gridDim.x) {
        const int64_t r0 = run * kRun<R>;
        const int64_t r1 = r0 + kRun<R> < map.N ? r0 + kRun<R> : map.N;
        int e = 0;
        if (map.offsets != nullptr) e = expert_of_row(map.offsets, map.E, (int)r0);
        for (; e < map.E; ++e) {   // (uniform)
            int64_t a = r0, z = r1;
            if (map.offsets != nullptr) {
                const int64_t ea = row_bound(map.offsets, e, map.N);
                const int64_t ez = row_bound(map.offsets, e + 1, map.N);
                if (ea >= r1) break;
                a = ea > r0 ? ea : r0;
                z = ez < r1 ? ez : r1;
                if (a >= z) continue;
            }
            float w[C][kN], dg[C][kN], db[C][kN];
#pragma unroll
            for (int c = 0; c < C; ++c) {
#pragma unroll
                for (int q = 0; q < kN; ++q) w[c][q] = dg[c][q] = db[c][q] = 0.0f;
                if (l + c * R < ncs) Ck::widen(Ck::fetch(g, (int64_t)e * ncs + l + c * R), w[c]);
            }
            // A row's loads are issued before the sums of the one before it.
            u32x4_t raw_x[C], raw_dy[C];
            int64_t src = -1;
            float m, rs;
            auto fetch = [&](int64_t r) {
                src = r < z ? map.source(r) : -1;
                if (src < 0) return;
                m = mean[r];
                rs = rstd[r];
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (l + c * R < ncs) {
                        raw_x[c] = Ck::fetch(x, src * ncs + l + c * R);
                        raw_dy[c] = Ck::fetch(dy, r * ncs + l + c * R);
                    }
            };
            fetch(a + group);
            for (int64_t r = a + group; r < z; r += kGroups) {
                if (src < 0) {   // (uniform over the threads that share the row)
                    fetch(r + kGroups);
                    continue;
                }
                float xh[C][kN], h[C][kN];
                float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
                for (int c = 0; c < C; ++c) {
#pragma unroll
                    for (int q = 0; q < kN; ++q) xh[c][q] = h[c][q] = 0.0f;
                    if (l + c * R < ncs) {
                        Ck::widen(raw_x[c], xh[c]);
                        Ck::widen(raw_dy[c], h[c]);
#pragma unroll
                        for (int q = 0; q < kN; ++q) {
                            xh[c][q] = (xh[c][q] - m) * rs;
                            dg[c][q] = fmaf(h[c][q], xh[c][q], dg[c][q]);
                            db[c][q] += h[c][q];
                            h[c][q] *= w[c][q];
                            s1 += h[c][q];
                            s2 = fmaf(h[c][q], xh[c][q], s2);
                        }
                    }
                }
                const float scale = rs;
                fetch(r + kGroups);
                s1 = row_sum<R>(s1, lds) / d;
                s2 = row_sum<R>(s2, lds) / d;
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    if (l + c * R >= ncs) continue;
                    float o[kN];
#pragma unroll
                    for (int q = 0; q < kN; ++q) o[q] = scale * (h[c][q] - s1 - xh[c][q] * s2);
                    if (residual != nullptr) {
                        float a[kN];
                        Ck::widen(Ck::fetch(residual, r * ncs + l + c * R), a);
#pragma unroll
                        for (int q = 0; q < kN; ++q) o[q] += a[q];
                    }
                    Ck::store(dx, r * ncs + l + c * R, o);
                }
            }
            float *out = part + (run + e) * 2 * d;
            if constexpr (kGroups > 1) {
                for (int w0 = 0; w0 < kGroups; ++w0) {
                    if (group == w0)
#pragma unroll
                        for (int c = 0; c < C; ++c)
                            if (l + c * R < ncs)
#pragma unroll
                                for (int q = 0; q < kN; ++q) {
                                    const int i = ((c * kN + q) / 4 * R + l) * 4 + q % 4;
                                    if (w0 > 0) {
                                        dg[c][q] += sums[i];
                                        db[c][q] += sums[C * kN * R + i];
                                    }
                                    if (w0 < kGroups - 1) {
                                        sums[i] = dg[c][q];
                                        sums[C * kN * R + i] = db[c][q];
                                    }
                                }
                    __syncthreads();
                }
            }
            if (group == kGroups - 1)
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (l + c * R < ncs)
#pragma unroll
                        for (int q = 0; q < kN; q += 4) {
                            const int i = (l + c * R) * kN + q;
                            *reinterpret_cast<float4 *>(out + i) =
                                make_float4(dg[c][q], dg[c][q + 1], dg[c][q + 2], dg[c][q + 3]);
                            *reinterpret_cast<float4 *>(out + d + i) =
                                make_float4(db[c][q], db[c][q + 1], db[c][q + 2], db[c][q + 3]);
                        }
        }
    }
}

// dg_e and db_e: the sums of the blocks that hold rows of expert e, in their
// order. A block for 64 of the 2 d columns of an expert; its W waves take a part of
// the blocks each: 16 where experts are few (one expert, 1024 blocks, d = 4096: 62 us with
// four waves).
template <int W>
__global__ __launch_bounds__(64 * W) void norm_weights_kernel(const float *__restrict__ part,
                                                              const int32_t *__restrict__ offsets,
                                                              float *__restrict__ dg,
                                                              float *__restrict__ db, int N, int d,
                                                              int run) {
    __shared__ float lds[W][64];
    const int e = blockIdx.y;
    const int lane = threadIdx.x & 63;
    const int wave = threadIdx.x >> 6;
    const int i = blockIdx.x * 64 + lane;   // column of [2 d]
    const int a = offsets == nullptr ? 0 : row_bound(offsets, e, N);
    const int z = offsets == nullptr ? N : row_bound(offsets, e + 1, N);
    float sum = 0.0f;
    if (a < z && i < 2 * d) {
        const int p0 = a / run, p1 = (z - 1) / run + 1;
        const int per = (p1 - p0 + W - 1) / W;
        const int q0 = p0 + wave * per;
        const int q1 = q0 + per < p1 ? q0 + per : p1;
#pragma unroll 8
        for (int p = q0; p < q1; ++p) sum += part[((int64_t)p + e) * 2 * d + i];
    }
    lds[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && i < 2 * d) {
        sum = lds[0][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) sum += lds[w][lane];
        float *out = i < d ? dg : db;
        if (out != nullptr) out[(int64_t)e * d + (i < d ? i : i - d)] = sum;
    }
}

constexpr int64_t kMaxBlocks = 1 << 22;   // a launch has fewer than 2^32 threads; rows go round

struct NormCall {
    const void *x, *g, *b, *dy, *residual;
    const float *mean_in, *rstd_in;
    void *y;
    float *mean, *rstd, *part;
    RowMap map;
    int d;
    float eps;
    bool backward;
};

template <bool BF16, int R, int C>
void launch_norm_as(const NormCall &n, hipStream_t s) {
    constexpr int kGroups = kBlock<R> / R;
    const int64_t rows = n.backward ? kRun<R> : kGroups;
    int64_t blocks = ((int64_t)n.map.N + rows - 1) / rows;
    if (blocks > kMaxBlocks) blocks = kMaxBlocks;
    if (!n.backward) {
        hipLaunchKernelGGL((norm_kernel<BF16, R, C>), dim3((unsigned)blocks), dim3(kBlock<R>), 0, s,
                           n.x, n.g, n.b, n.map, n.y, n.mean, n.rstd, n.d, n.eps);
        return;
    }
    hipLaunchKernelGGL((norm_backward_kernel<BF16, R, C>), dim3((unsigned)blocks),
                       dim3(kBlock<R>), kGroups > 1 ? C * RowChunk<BF16>::kN * R * 8 : 0, s, n.dy,
                       n.x, n.g, n.mean_in, n.rstd_in, n.residual, n.map, n.y, n.part, n.d);
}

// Threads per row: a wave up to 4 chunks a lane, then a block of four waves, then of eight
// (1024 threads would leave the gradient half the registers that it needs; with 512, fp32 rows
// of more than 8192, eight chunks a thread, keep 42 in memory: 4096 rows of 16384 182 us, 8192
// of 8192, which have room, 162).
int row_threads(int64_t ncs) { return ncs <= 256 ? 64 : ncs <= 1024 ? 256 : 512; }

template <bool BF16>
void launch_norm_for(const NormCall &n, hipStream_t s) {
    const int64_t ncs = n.d / RowChunk<BF16>::kN;
    switch (row_threads(ncs)) {
        case 64:
            if (ncs <= 64) return launch_norm_as<BF16, 64, 1>(n, s);
            if (ncs <= 128) return launch_norm_as<BF16, 64, 2>(n, s);
            return launch_norm_as<BF16, 64, 4>(n, s);
        case 256:
            if (ncs <= 512) return launch_norm_as<BF16, 256, 2>(n, s);
            return launch_norm_as<BF16, 256, 4>(n, s);
        default:
            if constexpr (!BF16)
                if (ncs > 2048) return launch_norm_as<BF16, 512, 8>(n, s);
            return launch_norm_as<BF16, 512, 4>(n, s);
    }
}

int64_t rows_per_run(int64_t ncs) {
    switch (row_threads(ncs)) {
        case 64: return kRun<64>;
        case 256: return kRun<256>;
        default: return kRun<512>;
    }
}

}  // namespace

// The partial sums of whichever type has the shorter runs.
size_t norm_workspace_size(int64_t N, int64_t E, int64_t d) {
    const int64_t run = rows_per_run(d / 4) < rows_per_run(d / 8) ? rows_per_run(d / 4)
                                                                  : rows_per_run(d / 8);
    return ((size_t)((N + run - 1) / run + E) * (size_t)d * 8 + 255) / 256 * 256;
}

hipError_t launch_norm(const void *x, const int32_t *perm, int64_t x_rows, int64_t k,
                       const void *weight, const void *bias, const int32_t *offsets, void *y,
                       float *mean, float *rstd, int64_t N, int64_t E, int64_t d, double eps,
                       int bf16, hipStream_t s) {
    NormCall n{};
    n.x = x;
    n.g = weight;
    n.b = bias;
    n.y = y;
    n.mean = mean;
    n.rstd = rstd;
    n.map = RowMap{perm, offsets, x_rows, (int)N, (int)E, (int)k};
    n.d = (int)d;
    n.eps = (float)eps;
    if (bf16) launch_norm_for<true>(n, s);
    else launch_norm_for<false>(n, s);
    return hipGetLastError();
}

hipError_t launch_norm_backward(const void *dy, const void *x, const int32_t *perm, int64_t x_rows,
                                int64_t k, const void *weight, const float *mean,
                                const float *rstd, const int32_t *offsets, const void *residual,
                                void *dx, float *dweight, float *dbias, int64_t N, int64_t E,
                                int64_t d, int bf16, void *workspace, hipStream_t s) {
    NormCall n{};
    n.x = x;
    n.g = weight;
    n.dy = dy;
    n.residual = residual;
    n.mean_in = mean;
    n.rstd_in = rstd;
    n.y = dx;
    n.part = static_cast<float *>(workspace);
    n.map = RowMap{perm, offsets, x_rows, (int)N, (int)E, (int)k};
    n.d = (int)d;
    n.backward = true;
    if (bf16) launch_norm_for<true>(n, s);
    else launch_norm_for<false>(n, s);
    const int64_t run = rows_per_run(d / (bf16 ? 8 : 4));
    const dim3 grid((unsigned)((2 * d + 63) / 64), (unsigned)E);
    if (N / run >= 32 * E)
        hipLaunchKernelGGL(norm_weights_kernel<16>, grid, dim3(1024), 0, s, n.part, offsets, dweight,
                           dbias, (int)N, (int)d, (int)run);
    else
        hipLaunchKernelGGL(norm_weights_kernel<4>, grid, dim3(256), 0, s, n.part, offsets, dweight,
                           dbias, (int)N, (int)d, (int)run);
    return hipGetLastError();
}

}  // namespace base
