// 16 bytes of a row at a time, at any alignment of its elements.
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
template <typename T> __device__ __forceinline__ float unpack(uint32_t w, int hi);
template <> __device__ __forceinline__ float unpack<bf16_t>(uint32_t w, int hi) { return __uint_as_float(hi ? w & 0xFFFF0000u : w << 16); }
template <> __device__ __forceinline__ float unpack<f16_t>(uint32_t w, int hi) {
    typedef f16_t pair __attribute__((ext_vector_type(2)));
    return (float)__builtin_bit_cast(pair, w)[hi];
}

// 16 bytes of a row, at any alignment of the element's, packed as they came.
template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
    uint32_t w[4];
    typedef uint32_t Quad __attribute__((ext_vector_type(4), aligned(2), may_alias));
    // ONCE: what nobody reads again soon, evict-first in the L2 (policy loss of 8192 x 32000 bf16 201 -> 181 us).
    template <bool ONCE> __device__ __forceinline__ void load(const T* p) {
        const Quad q = ONCE ? __builtin_nontemporal_load((const Quad*)p) : *(const Quad*)p;
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = q[k];
    }
    template <bool ONCE> __device__ __forceinline__ void store(T* p) const {
        const Quad q{w[0], w[1], w[2], w[3]};
        if (ONCE) __builtin_nontemporal_store(q, (Quad*)p);
        else *(Quad*)p = q;
    }
    __device__ __forceinline__ void get(float (&x)[N]) const {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = unpack<T>(w[e / 2], e & 1);
    }
    __device__ __forceinline__ void set(const float (&x)[N]) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = pack2<T>(x[2 * k], x[2 * k + 1]);
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
        for (int k = 0; k < 4; ++k) asm volatile("" : "+v"(w[k]));
    }
};
template <> __device__ __forceinline__ void Vec<float>::get(float (&x)[4]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(w[e]);
}
template <> __device__ __forceinline__ void Vec<float>::set(const float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(x[e]);
}

// Eight elements at p, at any alignment, as floats.
template <bool ONCE, typename T> __device__ __forceinline__ void load8_any(const T* p, float (&x)[8]) {
    constexpr int N = Vec<T>::N;
    Vec<T> v[8 / N];
#pragma unroll
    for (int k = 0; k < 8 / N; ++k) v[k].template load<ONCE>(p + k * N);
#pragma unroll
    for (int k = 0; k < 8 / N; ++k) {
        float y[N];
        v[k].get(y);
#pragma unroll
        for (int e = 0; e < N; ++e) x[k * N + e] = y[e];
    }
}
template <bool ONCE, typename T> __device__ __forceinline__ void store8_any(T* p, const float (&x)[8]) {
    constexpr int N = Vec<T>::N;
#pragma unroll
    for (int k = 0; k < 8 / N; ++k) {
        float y[N];
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = x[k * N + e];
        Vec<T> v;
        v.set(y);
        v.template store<ONCE>(p + k * N);
    }
}

}  // namespace rlhf
