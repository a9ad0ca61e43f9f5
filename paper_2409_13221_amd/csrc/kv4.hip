// Rows of K and V into the paged cache of 4 bits, and back (include/rlhf_ops.h states layout and rounding).
#include "kv4.h"

#include <algorithm>

#include "kernels.h"
#include "vec.h"

namespace rlhf {

// The whole number -8 .. 7 nearest to (x - c) / s, the even one half way, in double: in float the quotient would be rounded, and a value next to
// half way between two steps could go to the other one.
__device__ __forceinline__ int kv4_code(float x, float s, float c) {
    if (s == 0.f) return 0;
    const double d = (double)x - (double)c;
    double u = rint(d / (double)s);
    u = u < -8. ? -8. : u > 7. ? 7. : u;
    return (int)u;
}

// A wave takes one head's K or V of one row: lanes hold dims lane and lane + 64.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_kv4_append(Kv4Args a) {
    using L = Kv4<HD>;
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int r = (int)(w / (2 * a.n_kv_heads)), rest = (int)(w % (2 * a.n_kv_heads)), h = rest >> 1, is_v = rest & 1;
    if (r >= a.rows) return;
    const int slot = a.slot[r];
    if (slot < 0 || slot / 16 >= a.n_pages) return;
    const T* x = is_v ? (const T*)a.v + (size_t)r * a.ld_v + (size_t)h * HD : (const T*)a.k + (size_t)r * a.ld_k + (size_t)h * HD;
    uint8_t* block = (uint8_t*)a.pool + (((size_t)(slot / 16) * a.n_layers + a.layer) * a.n_kv_heads + h) * L::BLOCK;
    const int t = slot % 16;
#pragma unroll
    for (int g = 0; g < L::GROUPS; ++g) {
        const int d = g * 64 + lane;
        const float f = to_f32<T>(x[d]);
        const bool bad = __any(!(fabsf(f) <= 65504.f));
        const float lo = -wave_max(-f), hi = wave_max(f);
        const f16_t s = bad ? (f16_t)NAN : (f16_t)((hi - lo) * (1.f / 15.f));
        const f16_t c = bad ? (f16_t)NAN : (f16_t)(lo + 8.f * (float)s);
        const int u = bad ? 8 : 8 + kv4_code(f, (float)s, (float)c);
        const int other = __shfl_xor(u, is_v ? 16 : 1, kWave);
        if (is_v) {
            if (L::v_bit(d) == 0) block[L::v_byte(t, d)] = (uint8_t)(u | other << 4);
        } else {
            if (L::k_bit(d) == 0) block[L::k_byte(t, d)] = (uint8_t)(u | other << 4);
        }
        if (lane == 0) {
            f16_t* p = (f16_t*)(block + L::param(t, d) + is_v * L::PARAMS);
            p[0] = s;
            p[1] = c;
        }
    }
}

template <typename T, int HD>
__global__ __launch_bounds__(256) void k_kv4_read(Kv4Args a) {
    using L = Kv4<HD>;
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int r = (int)(w / (2 * a.n_kv_heads)), rest = (int)(w % (2 * a.n_kv_heads)), h = rest >> 1, is_v = rest & 1;
    if (r >= a.rows) return;
    T* x = is_v ? (T*)a.v + (size_t)r * a.ld_v + (size_t)h * HD : (T*)a.k + (size_t)r * a.ld_k + (size_t)h * HD;
    const int slot = a.slot[r];
    const bool inside = slot >= 0 && slot / 16 < a.n_pages;
    const uint8_t* block = (const uint8_t*)a.pool + (((size_t)(inside ? slot / 16 : 0) * a.n_layers + a.layer) * a.n_kv_heads + h) * L::BLOCK;
    const int t = slot & 15;
#pragma unroll
    for (int g = 0; g < L::GROUPS; ++g) {
        const int d = g * 64 + lane;
        float f = slot < 0 ? 0.f : NAN;
        if (inside) {
            const int u = (is_v ? block[L::v_byte(t, d)] >> L::v_bit(d) : block[L::k_byte(t, d)] >> L::k_bit(d)) & 15;
            const f16_t* p = (const f16_t*)(block + L::param(t, d) + is_v * L::PARAMS);
            f = (float)p[1] + (float)p[0] * (float)(u - 8);
        }
        x[d] = round_to<T>(f);
    }
}

size_t kv4_block_bytes(int head_dim) { return (size_t)18 * head_dim; }

template <typename T, bool APPEND>
static hipError_t kv4_typed(hipStream_t st, int head_dim, const Kv4Args& a) {
    const int most = (int)std::min<int64_t>(kLaunchThreads / 128 / a.n_kv_heads, 1 << 30);
    for (int first = 0; first < a.rows; first += most) {
        Kv4Args p = a;
        p.k = (T*)a.k + (size_t)first * a.ld_k;
        p.v = (T*)a.v + (size_t)first * a.ld_v;
        p.slot += first;
        p.rows = std::min(most, a.rows - first);
        const unsigned blocks = (unsigned)(((int64_t)p.rows * 2 * a.n_kv_heads + 3) / 4);
        if (APPEND) {
            if (head_dim == 128) k_kv4_append<T, 128><<<blocks, 256, 0, st>>>(p);
            else k_kv4_append<T, 64><<<blocks, 256, 0, st>>>(p);
        } else {
            if (head_dim == 128) k_kv4_read<T, 128><<<blocks, 256, 0, st>>>(p);
            else k_kv4_read<T, 64><<<blocks, 256, 0, st>>>(p);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_kv4_append(hipStream_t st, int dtype, int head_dim, const Kv4Args& a) {
    return dtype == kBF16 ? kv4_typed<bf16_t, true>(st, head_dim, a) : dtype == kF16 ? kv4_typed<f16_t, true>(st, head_dim, a) : kv4_typed<float, true>(st, head_dim, a);
}
hipError_t launch_kv4_read(hipStream_t st, int dtype, int head_dim, const Kv4Args& a) {
    return dtype == kBF16 ? kv4_typed<bf16_t, false>(st, head_dim, a) : dtype == kF16 ? kv4_typed<f16_t, false>(st, head_dim, a) : kv4_typed<float, false>(st, head_dim, a);
}

}  // namespace rlhf
