// A few elements of a row at a time, at any alignment.
#pragma once
#include "common.h"

namespace rlhf {

// Two floats as two packed 16-bit elements, and back; rounded to nearest, a NaN stays one.
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<bf16_t>(float lo, float hi) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, pair{(__bf16)lo, (__bf16)hi});
}
template <> __device__ __forceinline__ uint32_t pack2<f16_t>(float lo, float hi) {
    typedef f16_t pair __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, pair{(f16_t)lo, (f16_t)hi});
}
// One float to T, rounded to nearest; a NaN stays one whatever its payload (f32_to_bf16 carries some of them over into -0).
template <typename T> __device__ __forceinline__ T round_to(float x) { return from_f32<T>(x); }
template <> __device__ __forceinline__ bf16_t round_to<bf16_t>(float x) { return __builtin_bit_cast(bf16_t, (__bf16)x); }

template <typename T> __device__ __forceinline__ float unpack(uint32_t w, int hi);
template <> __device__ __forceinline__ float unpack<bf16_t>(uint32_t w, int hi) { return __uint_as_float(hi ? w & 0xFFFF0000u : w << 16); }
template <> __device__ __forceinline__ float unpack<f16_t>(uint32_t w, int hi) {
    typedef f16_t pair __attribute__((ext_vector_type(2)));
    return (float)__builtin_bit_cast(pair, w)[hi];
}

// N elements of a row, 8 or 16 bytes, at any alignment of the element's, packed as they came.
template <typename T, int N = 16 / sizeof(T)> struct Vec {
    static constexpr int WORDS = N * sizeof(T) / 4;
    static_assert(N % 2 == 0 && (WORDS == 2 || WORDS == 4), "8 or 16 bytes");
    uint32_t w[WORDS];
    typedef uint32_t Words __attribute__((ext_vector_type(WORDS), aligned(2), may_alias));
    // ONCE: what nobody reads again soon, evict-first in the L2 (policy loss of 8192 x 32000 bf16 201 -> 181 us).  A store of
    // that kind has to fill its lines together with its neighbours (lanes 32 bytes apart: 97 -> 227 us for 524 MB of zeros).
    template <bool ONCE> __device__ __forceinline__ void load(const T* p) {
        const Words q = ONCE ? __builtin_nontemporal_load((const Words*)p) : *(const Words*)p;
#pragma unroll
        for (int k = 0; k < WORDS; ++k) w[k] = q[k];
    }
    template <bool ONCE> __device__ __forceinline__ void store(T* p) const {
        Words q;
#pragma unroll
        for (int k = 0; k < WORDS; ++k) q[k] = w[k];
        if (ONCE) __builtin_nontemporal_store(q, (Words*)p);
        else *(Words*)p = q;
    }
    __device__ __forceinline__ void get(float (&x)[N]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = __uint_as_float(w[e]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = unpack<T>(w[e / 2], e & 1);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[N]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] = __float_as_uint(x[e]);
        } else {
#pragma unroll
            for (int k = 0; k < WORDS; ++k) w[k] = pack2<T>(x[2 * k], x[2 * k + 1]);
        }
    }
    __device__ __forceinline__ void fill(float v) {
        float x[N];
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = v;
        set(x);
    }
    // What get() gave before is not kept for get() after it: the packed form is the one that stays in registers.
    __device__ __forceinline__ void forget() {
#pragma unroll
        for (int k = 0; k < WORDS; ++k) asm volatile("" : "+v"(w[k]));
    }
};

}  // namespace rlhf
