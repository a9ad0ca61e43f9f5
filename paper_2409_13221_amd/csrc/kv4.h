// The cache of 4 bits (layout and rounding are stated in include/rlhf_ops.h): where things lie in a block, the 18 * HD bytes of one
// (page, layer, KV head).
#pragma once
#include <type_traits>

#include "common.h"

namespace rlhf {

template <int HD> struct Kv4 {
    static constexpr int PIECE = HD / 8;                 // bytes of codes of a lane of the matrix units: 16 or 8
    static constexpr int CODES = 8 * HD, PARAMS = HD, BLOCK = 18 * HD, GROUPS = HD / 64;
    static constexpr int V_CODES = CODES, K_PARAMS = 2 * CODES, V_PARAMS = K_PARAMS + PARAMS;
    // Byte and bit of dim d of token t.
    __host__ __device__ static constexpr int k_byte(int t, int d) { return ((d % 32 / 8) * 16 + t) * PIECE + d / 32 * 4 + d % 8 / 2; }
    __host__ __device__ static constexpr int k_bit(int d) { return 4 * (d % 2); }
    __host__ __device__ static constexpr int v_byte(int t, int d) { return V_CODES + (t / 4 * 16 + d % 16) * PIECE + d / 32 * 4 + t % 4; }
    __host__ __device__ static constexpr int v_bit(int d) { return 4 * (d % 32 / 16); }
    // Scale and center of 64 dims of token t, two halves from this byte on; of V: PARAMS further.
    __host__ __device__ static constexpr int param(int t, int d) { return K_PARAMS + (d / 64 * 16 + t) * 4; }
};

// A value on its way to T.  A step next to 65504, half's greatest, may lie beyond it, by up to 15 half steps of the scale and one of the center (76), and from 65520 on
// would round to infinity: it is held to 65504, as the values that went into the cache were.
template <typename T> __device__ __forceinline__ float within(float x) {
    if constexpr (std::is_same_v<T, f16_t>) return fabsf(x) > 65504.f && fabsf(x) < INFINITY ? copysignf(65504.f, x) : x;
    else return x;
}

}  // namespace rlhf
