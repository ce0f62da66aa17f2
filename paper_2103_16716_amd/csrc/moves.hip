// Token rows to their experts and back with k experts a token, and the gradient.
// slots[t k + j] is the routed row of choice j of token t (-1: none), N = T k
// routed rows. All three kernels go token by token, and sums over choices run in
// their order, without atomics. dispatch and combine read a token's row once for
// its k choices. combine_backward goes choice by choice and reads dY[t] again for
// each: 32768 tokens, two choices, rows of 2048 in bf16 540 MB where 403 would do,
// 132 us (6.1 TB/s); 8192 tokens of eight 130 us. An entry of slots outside [0, N)
// is no row.
#include "common.hpp"
#include "internal.hpp"
#include "rows.hpp"

namespace base {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int64_t kMaxBlocks = 1 << 22;   // a launch has fewer than 2^32 threads; blocks go round

// out[slots[t, j]] = w[t, j] x[t]: a thread per 16-byte chunk of a token's row.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void dispatch_kernel(
    const void *__restrict__ x, const float *__restrict__ w, const int32_t *__restrict__ slots,
    void *__restrict__ out, int64_t N, int64_t total, int k, int ncs) {
    using Ck = RowChunk<BF16>;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total;
         i += (int64_t)gridDim.x * kThreads) {
        const int64_t t = i / ncs;
        const int c = (int)(i - t * ncs);
        const u32x4_t raw = Ck::fetch_once(x, i);
        float v[Ck::kN];
        Ck::widen(raw, v);
        for (int j = 0; j < k; ++j) {
            const int64_t r = slots[t * k + j];
            if (r < 0 || r >= N) continue;
            u32x4_t o = raw;
            if (w != nullptr) {
                const float g = w[t * k + j];
                float y[Ck::kN];
#pragma unroll
                for (int q = 0; q < Ck::kN; ++q) y[q] = g * v[q];
                o = Ck::narrow(y);
            }
            reinterpret_cast<u32x4_t *>(out)[r * ncs + c] = o;
        }
    }
}

// out[t] = residual[t] + sum_j w[t, j] F[slots[t, j]].
template <bool BF16>
__global__ __launch_bounds__(kThreads) void combine_kernel(
    const void *__restrict__ F, const float *__restrict__ w, const int32_t *__restrict__ slots,
    const void *residual, void *out, int64_t N, int64_t total, int k, int ncs) {
    using Ck = RowChunk<BF16>;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total;
         i += (int64_t)gridDim.x * kThreads) {
        const int64_t t = i / ncs;
        const int c = (int)(i - t * ncs);
        float y[Ck::kN];
#pragma unroll
        for (int q = 0; q < Ck::kN; ++q) y[q] = 0.0f;
        if (residual != nullptr) Ck::widen(Ck::fetch(residual, i), y);
        for (int j = 0; j < k; ++j) {
            const int64_t r = slots[t * k + j];
            if (r < 0 || r >= N) continue;
            const float g = w == nullptr ? 1.0f : w[t * k + j];
            float f[Ck::kN];
            Ck::widen(Ck::fetch(F, r * ncs + c), f);
#pragma unroll
            for (int q = 0; q < Ck::kN; ++q) y[q] = fmaf(g, f[q], y[q]);
        }
        Ck::store(out, i, y);
    }
}

// A wave per token, one choice after another: dF[r] = w[t, j] dY[t] and dw[t, j] = dY[t] . F[r],
// r = slots[t, j].
template <bool BF16>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(
    const void *__restrict__ dY, const void *__restrict__ F, const float *__restrict__ w,
    const int32_t *__restrict__ slots, void *__restrict__ dF, float *__restrict__ dw, int64_t T,
    int64_t N, int k, int ncs) {
    using Ck = RowChunk<BF16>;
    const int lane = threadIdx.x & 63;
    for (int64_t t = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); t < T;
         t += (int64_t)gridDim.x * kWaves) {
        for (int j = 0; j < k; ++j) {
            const int64_t r = slots[t * k + j];
            float dot = 0.0f;
            if (r >= 0 && r < N) {
                const float g = w[t * k + j];
                for (int c = lane; c < ncs; c += 64) {
                    float y[Ck::kN], f[Ck::kN];
                    Ck::widen(Ck::fetch(dY, t * ncs + c), y);
                    Ck::widen(Ck::fetch(F, r * ncs + c), f);
#pragma unroll
                    for (int q = 0; q < Ck::kN; ++q) {
                        dot = fmaf(y[q], f[q], dot);
                        y[q] *= g;
                    }
                    Ck::store(dF, r * ncs + c, y);
                }
            }
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) dot += __shfl_xor(dot, off);
            if (lane == 0) dw[t * k + j] = dot;
        }
    }
}

dim3 blocks_for(int64_t n, int64_t per) {
    const int64_t b = (n + per - 1) / per;
    return dim3((unsigned)(b < kMaxBlocks ? b : kMaxBlocks));
}

}  // namespace

hipError_t launch_dispatch(const void *x, const float *w, const int32_t *slots, void *out,
                           int64_t T, int64_t k, int64_t d, int bf16, hipStream_t s) {
    const int ncs = (int)(d / (bf16 ? 8 : 4));
    const int64_t total = T * ncs;
    const dim3 grid = blocks_for(total, kThreads);
    if (bf16)
        hipLaunchKernelGGL(dispatch_kernel<true>, grid, dim3(kThreads), 0, s, x, w, slots, out,
                           T * k, total, (int)k, ncs);
    else
        hipLaunchKernelGGL(dispatch_kernel<false>, grid, dim3(kThreads), 0, s, x, w, slots, out,
                           T * k, total, (int)k, ncs);
    return hipGetLastError();
}

hipError_t launch_combine(const void *F, const float *w, const int32_t *slots,
                          const void *residual, void *out, int64_t T, int64_t k, int64_t d,
                          int bf16, hipStream_t s) {
    const int ncs = (int)(d / (bf16 ? 8 : 4));
    const int64_t total = T * ncs;
    const dim3 grid = blocks_for(total, kThreads);
    if (bf16)
        hipLaunchKernelGGL(combine_kernel<true>, grid, dim3(kThreads), 0, s, F, w, slots, residual,
                           out, T * k, total, (int)k, ncs);
    else
        hipLaunchKernelGGL(combine_kernel<false>, grid, dim3(kThreads), 0, s, F, w, slots,
                           residual, out, T * k, total, (int)k, ncs);
    return hipGetLastError();
}

hipError_t launch_combine_backward(const void *dY, const void *F, const float *w,
                                   const int32_t *slots, void *dF, float *dw, int64_t T, int64_t k,
                                   int64_t d, int bf16, hipStream_t s) {
    const int ncs = (int)(d / (bf16 ? 8 : 4));
    const dim3 grid = blocks_for(T, kWaves);
    if (bf16)
        hipLaunchKernelGGL(combine_backward_kernel<true>, grid, dim3(kThreads), 0, s, dY, F, w,
                           slots, dF, dw, T, T * k, (int)k, ncs);
    else
        hipLaunchKernelGGL(combine_backward_kernel<false>, grid, dim3(kThreads), 0, s, dY, F, w,
                           slots, dF, dw, T, T * k, (int)k, ncs);
    return hipGetLastError();
}

}  // namespace base
