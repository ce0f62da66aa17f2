// Rows of matrices in 16-byte chunks, widened to fp32, and lookups in the row
// ranges of the experts. Shared by the kernels of the expert layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace base {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// One 16-byte chunk of a row: 8 bf16 (widened exactly; rounded to nearest even
// on the way back) or 4 fp32 values.
template <bool BF16>
struct RowChunk {
    static constexpr int kN = BF16 ? 8 : 4;
    __device__ static u32x4_t fetch(const void *base, int64_t chunk) {
        return reinterpret_cast<const u32x4_t *>(base)[chunk];
    }
    __device__ static u32x4_t fetch_once(const void *base, int64_t chunk) {
        return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(base) + chunk);
    }
    __device__ static void widen(u32x4_t x, float (&v)[kN]) {
        if constexpr (BF16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(x[i] << 16);
                v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(x[i]);
        }
    }
    __device__ static u32x4_t narrow(const float (&v)[kN]) {
        u32x4_t x;
        if constexpr (BF16) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = __builtin_bit_cast(
                    uint32_t,
                    __builtin_convertvector((f32x2_t{v[2 * i], v[2 * i + 1]}), bf16x2_t));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __float_as_uint(v[i]);
        }
        return x;
    }
    __device__ static void store(void *base, int64_t chunk, const float (&v)[kN]) {
        reinterpret_cast<u32x4_t *>(base)[chunk] = narrow(v);
    }
};

// Sum over the 64 lanes, in every lane: rows of 16 lanes turn by 8, 4, 2 and 1, then rows and
// half waves are exchanged. The order is fixed. No memory is involved (a shuffle through the
// LDS takes an order of magnitude longer).
template <int kControl>
__device__ inline float turned(float v) {
    return __uint_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_uint(v), kControl, 0xf, 0xf, true));
}
__device__ inline float wave_sum(float v) {
    typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
    v += turned<0x128>(v);
    v += turned<0x124>(v);
    v += turned<0x122>(v);
    v += turned<0x121>(v);
    const uint32_t a = __float_as_uint(v);
    const u32x2_t r =
        __builtin_bit_cast(u32x2_t, __builtin_amdgcn_permlane16_swap(a, a, false, false));
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    const uint32_t b = __float_as_uint(v);
    const u32x2_t h =
        __builtin_bit_cast(u32x2_t, __builtin_amdgcn_permlane32_swap(b, b, false, false));
    return __uint_as_float(h[0]) + __uint_as_float(h[1]);
}

// The experts' row ranges: expert e has rows [offsets[e], offsets[e + 1]) of N.
// Values outside [0, N] are brought into it, so that no range leaves the
// matrices whatever the buffer holds.
__device__ inline int row_bound(const int32_t *__restrict__ offsets, int e, int N) {
    const int o = offsets[e];
    return o < 0 ? 0 : (o > N ? N : o);
}

// The expert of row r, asked by all 64 lanes of a wave at once: the number of
// experts whose range ends at or before it (E and more: no expert). One round
// of loads instead of a chain of them.
__device__ inline int expert_of_row(const int32_t *__restrict__ offsets, int E, int r) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        const int e = e0 + lane;
        n += __popcll(__ballot(e < E && offsets[e < E ? e + 1 : E] <= r));
    }
    return n;
}

}  // namespace base
