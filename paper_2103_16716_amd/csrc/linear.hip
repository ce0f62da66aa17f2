// The experts' products: rows of the routed order times the matrix of each row's
// expert, and the gradients.
//
//   y[r]  = act(x[r] W_e^T + b_e) + residual[r]      W [E, O, K], e the row's expert
//   dx[r] = (dy[r] W_e) where relu_of[r] > 0, else 0
//   dW_e  = sum over its rows of dy[r] x[r]^T,  db_e = sum of dy[r]
//
// Products are summed in fp32. Rows in no expert's range are left alone; an expert
// without rows has zero dW and db.
#include "common.hpp"
#include "internal.hpp"
#include "rows.hpp"

namespace base {
namespace {

// Tile `tile` of the experts' rows in tiles of BM, expert after expert: its
// expert, its first row and the end of the expert's rows. Asked by whole waves.
struct RowTile {
    int e, r0, r1;
};
__device__ inline bool find_row_tile(const int32_t *__restrict__ offsets, int E, int N, int BM,
                                     int tile, RowTile &out) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        const int e = e0 + lane;
        const int a = e < E ? row_bound(offsets, e, N) : 0;
        const int z = e < E ? row_bound(offsets, e + 1, N) : 0;
        const int n = z > a ? (z - a + BM - 1) / BM : 0;
        int sum = n;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(sum, off);
            if (lane >= off) sum += o;
        }
        const uint64_t past = __ballot(before + sum > tile);
        if (past != 0) {
            const int f = __ffsll((unsigned long long)past) - 1;
            out.e = e0 + f;
            out.r1 = __shfl(z, f);
            out.r0 = __shfl(a, f) + (tile - before - __shfl(sum - n, f)) * BM;
            return true;
        }
        before += __shfl(sum, 63);
    }
    return false;
}

template <bool BF16>
__device__ inline float element(const void *p, int64_t i) {
    if constexpr (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[i] << 16);
    else return static_cast<const float *>(p)[i];
}
template <bool BF16>
__device__ inline void put(void *p, int64_t i, float v) {
    if constexpr (BF16) static_cast<__bf16 *>(p)[i] = (__bf16)v;
    else static_cast<float *>(p)[i] = v;
}

// Tiles of 64 x 64 outputs and steps of 16 of the contraction on the vector units.
// kNT: y; kNN: dx; kTN: dW (and, in the tiles of the first 64 inputs, db).
enum { kNT, kNN, kTN };
constexpr int kT = 64, kS = 16;

template <bool BF16, int kForm>
__global__ __launch_bounds__(256) void linear_kernel(
    const void *__restrict__ A, const void *__restrict__ B, const void *__restrict__ bias,
    const void *extra, const int32_t *__restrict__ offsets, void *out, float *__restrict__ db,
    int N, int E, int K, int O, int relu) {
    __shared__ float a_lds[kS][kT + 1], b_lds[kS][kT + 1];
    RowTile rt;
    const int n0 = blockIdx.x * kT;
    if constexpr (kForm == kTN) {
        rt.e = blockIdx.z;
        rt.r0 = row_bound(offsets, rt.e, N);
        rt.r1 = row_bound(offsets, rt.e + 1, N);
    } else {
        if (!find_row_tile(offsets, E, N, kT, blockIdx.y, rt)) return;
    }
    // Output [m0.., n0..] of [m_end, cols]; contraction over [s0, s1).
    const int m0 = kForm == kTN ? blockIdx.y * kT : rt.r0;
    const int m_end = kForm == kTN ? O : rt.r1;
    const int cols = kForm == kNT ? O : K;
    const int s0 = kForm == kTN ? rt.r0 : 0;
    const int s1 = kForm == kTN ? rt.r1 : kForm == kNT ? K : O;
    const int64_t we = (int64_t)rt.e * O * K;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    float sum[4] = {};
    for (int s = s0; s < s1; s += kS) {
        for (int i = threadIdx.x; i < kS * kT; i += 256) {
            const int q = kForm == kTN ? i / kT : i % kS, m = kForm == kTN ? i % kT : i / kS;
            const bool in = s + q < s1 && m0 + m < m_end;
            const int64_t at = kForm == kTN ? (int64_t)(s + q) * O + m0 + m
                                            : (int64_t)(m0 + m) * (kForm == kNT ? K : O) + s + q;
            a_lds[q][m] = in ? element<BF16>(A, at) : 0.0f;
        }
        for (int i = threadIdx.x; i < kS * kT; i += 256) {
            const int q = kForm == kNT ? i % kS : i / kT, n = kForm == kNT ? i / kS : i % kT;
            const bool in = s + q < s1 && n0 + n < cols;
            const int64_t at = kForm == kTN   ? (int64_t)(s + q) * K + n0 + n
                               : kForm == kNN ? we + (int64_t)(s + q) * K + n0 + n
                                              : we + (int64_t)(n0 + n) * K + s + q;
            b_lds[q][n] = in ? element<BF16>(B, at) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kS; ++q) {
            float a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[i] = a_lds[q][ty + 16 * i];
                b[i] = b_lds[q][tx + 16 * i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[i] += a[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(a[i], b[j], acc[i][j]);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = m0 + ty + 16 * i;
        if (m >= m_end) continue;
        if (kForm == kTN && db != nullptr && n0 == 0 && tx == 0) db[(int64_t)rt.e * O + m] = sum[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = n0 + tx + 16 * j;
            if (n >= cols) continue;
            float v = acc[i][j];
            const int64_t at = (int64_t)m * cols + n;
            if constexpr (kForm == kTN) {
                static_cast<float *>(out)[we + at] = v;
            } else {
                if (kForm == kNT) {
                    if (bias != nullptr) v += element<BF16>(bias, (int64_t)rt.e * O + n);
                    if (relu) v = v < 0.0f ? 0.0f : v;
                    if (extra != nullptr) v += element<BF16>(extra, at);
                } else if (extra != nullptr && !(element<BF16>(extra, at) > 0.0f)) {
                    v = 0.0f;
                }
                put<BF16>(out, at, v);
            }
        }
    }
}

template <int kForm>
hipError_t launch_as(const void *A, const void *B, const void *bias, const void *extra,
                     const int32_t *offsets, void *out, float *db, int64_t N, int64_t E, int64_t K,
                     int64_t O, int relu, int bf16, hipStream_t s) {
    const int64_t cols = kForm == kNT ? O : K;
    const int64_t rows = kForm == kTN ? (O + kT - 1) / kT : N / kT + (E < N ? E : N);
    const dim3 grid((unsigned)((cols + kT - 1) / kT), (unsigned)rows, kForm == kTN ? (unsigned)E : 1);
    if (bf16)
        hipLaunchKernelGGL((linear_kernel<true, kForm>), grid, dim3(256), 0, s, A, B, bias, extra,
                           offsets, out, db, (int)N, (int)E, (int)K, (int)O, relu);
    else
        hipLaunchKernelGGL((linear_kernel<false, kForm>), grid, dim3(256), 0, s, A, B, bias, extra,
                           offsets, out, db, (int)N, (int)E, (int)K, (int)O, relu);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear(const void *x, const void *w, const void *bias, const void *residual,
                         const int32_t *offsets, void *y, int64_t N, int64_t E, int64_t K,
                         int64_t O, int relu, int bf16, hipStream_t s) {
    return launch_as<kNT>(x, w, bias, residual, offsets, y, nullptr, N, E, K, O, relu, bf16, s);
}

hipError_t launch_linear_dx(const void *dy, const void *w, const void *relu_of,
                            const int32_t *offsets, void *dx, int64_t N, int64_t E, int64_t K,
                            int64_t O, int bf16, hipStream_t s) {
    return launch_as<kNN>(dy, w, nullptr, relu_of, offsets, dx, nullptr, N, E, K, O, 0, bf16, s);
}

hipError_t launch_linear_dw(const void *dy, const void *x, const int32_t *offsets, float *dw,
                            float *db, int64_t N, int64_t E, int64_t K, int64_t O, int bf16,
                            hipStream_t s) {
    return launch_as<kTN>(dy, x, nullptr, nullptr, offsets, dw, db, N, E, K, O, 0, bf16, s);
}

}  // namespace base
