// What the attention kernels with a window share: 16 x 16 scores S^T = K Q^T, a lane holding keys 4c .. 4c + 3 of column n, n = lane % 16 (a query or
// query head), c = lane / 16, which is also how O^T += V^T P^T takes the weights: they never leave their lane.
#pragma once
#include "common.h"

namespace rlhf {

typedef f16_t f16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// log2 of a weight by a score: log2(e) / sqrt(HD).
template <int HD> constexpr float kScoreUnit = 1.44269504088896f * (HD == 64 ? 0.125f : 0.0883883476483184f);

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
    // Weights of up to 2^14, the greatest of them at least 2^6 (where a reference starts): half a step below half's normal range, 2^-25, is at most
    // 2^-31 of the greatest.
    static constexpr float TOP = 14.f;
    static constexpr uint32_t ONES = 0x3C003C00u;
    static __device__ __forceinline__ f32x4_t qk(u32x4_t a, u32x4_t b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4_t pv(u32x2_t a, u32x2_t b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4_t, a), __builtin_bit_cast(f16x4_t, b), c, 0, 0, 0);
    }
};
template <> struct Matrix16<bf16_t> {
    static constexpr float TOP = 0.f;
    static constexpr uint32_t ONES = 0x3F803F80u;
    static __device__ __forceinline__ f32x4_t qk(u32x4_t a, u32x4_t b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4_t pv(u32x2_t a, u32x2_t b, f32x4_t c) {
        return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4_t, a), __builtin_bit_cast(s16x4_t, b), c, 0, 0, 0);
    }
};

// Float: k = 4 products.  A lane has 4 dims of key n (K) and dims 64 i + 4 n .. + 3 of its four keys (V), so that 16 lanes side by side read 256 bytes of a row;
// element r of sums o[4 i + e] is dim 64 i + 4 (4c + r) + e.
template <int HD> struct FloatQuery {
    f32x4_t q[HD / 16];
    __device__ __forceinline__ void load(const float* p, int c) {
#pragma unroll
        for (int s = 0; s < HD / 16; ++s) q[s] = *(const f32x4_t*)(p + s * 16 + c * 4);
    }
};
// Four dims at a time: put(dim, values).
template <int HD, typename F> __device__ __forceinline__ void each_dims(const f32x4_t (&o)[HD / 16], int c, F put) {
#pragma unroll
    for (int i = 0; i < HD / 64; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) put(64 * i + 16 * c + 4 * r, f32x4_t{o[4 * i][r], o[4 * i + 1][r], o[4 * i + 2][r], o[4 * i + 3][r]});
}
__device__ __forceinline__ void float_scores(const f32x4_t& k, const f32x4_t& q, f32x4_t& s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], q[e], s, 0, 0, 0);
}
__device__ __forceinline__ void float_sums(const f32x4_t& v, float p, f32x4_t* o) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], p, o[e], 0, 0, 0);
}

}  // namespace rlhf
