// What the attention kernels with a window share: 16 x 16 scores S^T = K Q^T, a lane holding keys 4c .. 4c + 3 of column n, n = lane % 16 (a query or
// query head), c = lane / 16, which is also how O^T += V^T P^T takes the weights: they never leave their lane.
#pragma once
#include "common.h"

namespace rlhf {

typedef f16_t f16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// Greatest of (sum over) the four lanes that hold a column.
__device__ __forceinline__ float column_max(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float column_sum(float x) {
    x += __shfl_xor(x, 16, kWave);
    return x + __shfl_xor(x, 32, kWave);
}

template <typename T> struct Matrix16;
template <> struct Matrix16<f16_t> {
    // Weights of up to 2^14: what half loses below its normal range is 2^-39 of the greatest.
    static constexpr float TOP = 14.f;
    static __device__ __forceinline__ f32x4_t qk(u32x4_t a, u32x4_t b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4_t pv(u32x2_t a, u32x2_t b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4_t, a), __builtin_bit_cast(f16x4_t, b), c, 0, 0, 0);
    }
};
template <> struct Matrix16<bf16_t> {
    static constexpr float TOP = 0.f;
    static __device__ __forceinline__ f32x4_t qk(u32x4_t a, u32x4_t b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4_t pv(u32x2_t a, u32x2_t b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4_t, a), __builtin_bit_cast(s16x4_t, b), c, 0, 0, 0);
    }
};

// Float: k = 4 products.  A lane has 4 dims of key n (K) and D = HD / 16 dims of its four keys (V), D n .. D n + D - 1, so that a row of V is read by 16 lanes
// side by side; sums o[d] hold dim D (4c + r) + d in element r.
template <int HD> struct FloatQuery {
    f32x4_t q[HD / 16];
    __device__ __forceinline__ void load(const float* p, int c) {
#pragma unroll
        for (int s = 0; s < HD / 16; ++s) q[s] = *(const f32x4_t*)(p + s * 16 + c * 4);
    }
};
template <int HD> struct FloatTile {
    static constexpr int D = HD / 16;
    f32x4_t k[D], v[4][D / 4];
    // Rows 0 .. last of K and V; those behind it are the last one again.
    template <bool ONCE> __device__ __forceinline__ void load(const float* pk, size_t ldk, const float* pv, size_t ldv, int last, int n, int c) {
        const auto get = [](const float* p) { return ONCE ? __builtin_nontemporal_load((const f32x4_t*)p) : *(const f32x4_t*)p; };
        pk += min(n, last) * ldk + c * 4;
#pragma unroll
        for (int s = 0; s < D; ++s) k[s] = get(pk + s * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < D / 4; ++d) v[i][d] = get(pv + min(4 * c + i, last) * ldv + n * D + d * 4);
    }
    __device__ __forceinline__ f32x4_t scores(const FloatQuery<HD>& q) const {
        f32x4_t s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i][e], q.q[i][e], s, 0, 0, 0);
        return s;
    }
    __device__ __forceinline__ void add(const f32x4_t& p, f32x4_t (&o)[D]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < D; ++d) o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i][d / 4][d % 4], p[i], o[d], 0, 0, 0);
    }
    // Four dims at a time, in order: put(dim, values).
    template <typename F> static __device__ __forceinline__ void each(const f32x4_t (&o)[D], int c, F put) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int d = 0; d < D; d += 4) put((4 * c + r) * D + d, f32x4_t{o[d][r], o[d + 1][r], o[d + 2][r], o[d + 3][r]});
    }
};

}  // namespace rlhf
