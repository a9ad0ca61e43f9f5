// Rows of K and V into the paged cache of 4 bits, and back (include/rlhf_ops.h states layout and rounding).
#include "kv4.h"

#include <algorithm>

#include "kernels.h"
#include "vec.h"

namespace rlhf {

// What a thread of both kernels has: dims 8 i .. 8 i + 7 (i = lane % (HD / 8)) of one head of one row; 8 threads share a group.  Its K codes are one word of a
// block.  Its V codes are nibbles of 8 bytes, which the thread with dims 16 further on or back fills up: each of the two moves four of the bytes.
template <int HD> struct Piece {
    using L = Kv4<HD>;
    static constexpr int LANES = HD / 8, ROWS = 64 / LANES;        // of a wave
    int i, t, d;
    __device__ __forceinline__ Piece(int lane, int slot) : i(lane % LANES), t(slot & 15), d(i * 8) {}
    __device__ __forceinline__ int k_word() const { return L::k_byte(t, d); }
    __device__ __forceinline__ bool upper() const { return i & 2; }          // holds the upper nibbles
    __device__ __forceinline__ int v_byte(int j) const { return L::v_byte(t, d + (upper() ? 4 : 0) + j); }      // j-th of its four
    __device__ __forceinline__ int param() const { return L::param(t, d); }
};
__device__ __forceinline__ uint32_t other_nibbles(uint32_t x) { return __shfl_xor(x, 2, kWave); }
// Nibbles 0 .. 3 of lo and hi as the lower and upper ones of four bytes.
__device__ __forceinline__ uint32_t spread_nibbles(uint32_t x) {
    x = (x | x << 8) & 0x00FF00FFu;
    return (x | x << 4) & 0x0F0F0F0Fu;
}
__device__ __forceinline__ uint32_t merge_nibbles(uint32_t lo, uint32_t hi) { return spread_nibbles(lo & 0xFFFFu) | spread_nibbles(hi & 0xFFFFu) << 4; }
// Least (greatest) of the 8 threads of a group.
template <int CTRL> __device__ __forceinline__ float from_lane(float x) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), CTRL, 15, 15, true));
}
template <typename F> __device__ __forceinline__ float over_group(float x, F f) {
    x = f(x, from_lane<0xB1>(x));                  // neighbours, pairs, halves of 8
    x = f(x, from_lane<0x4E>(x));
    return f(x, from_lane<0x141>(x));
}

// u, the nearest whole number to q, or the one on q's other side: whichever is nearest to (x - c) / s, which q is within half a step of; the even one half
// way.  x, c and s are floats and halves: differences and products of this size are exact in double.
__device__ __forceinline__ float settle(float q, float u, float x, float s, float c) {
    const float side = q < u ? -1.f : 1.f, rest = (float)fma(-(double)(u + 0.5f * side), (double)s, (double)x - (double)c) * side;
    const bool odd = (int)u & 1, on = (rest > 0.f) | ((rest == 0.f) & odd);
    return on ? u + side : u;
}

// A float, rounded as one, to half.  The compiler makes one instruction of a multiply-add and this conversion, which rounds once where the
// definition rounds twice (one group in some thousands had another scale).
__device__ __forceinline__ f16_t half_of_float(float x) {
    asm volatile("" : "+v"(x));
    return (f16_t)x;
}

// Codes of a thread's 8 values (4 bits each), scale and center of its group.  In float a quotient of up to 8.5 is off by 8.5 x 2^-22 by the difference, the
// reciprocal and the product; those within 2^-17 of half way between two steps are settled exactly.  Rounding to the nearest whole
// number is the addition of 1.5 x 2^23 (and 8, for the code), whose low bits are then the code.
__device__ __forceinline__ uint32_t kv4_pack(const float (&x)[8], uint32_t& params) {
    float lo = x[0], hi = x[0];                    // not a number if one of them is not
#pragma unroll
    for (int e = 1; e < 8; ++e) {
        lo = __builtin_elementwise_minimum(lo, x[e]);
        hi = __builtin_elementwise_maximum(hi, x[e]);
    }
    lo = over_group(lo, [](float a, float b) { return __builtin_elementwise_minimum(a, b); });
    hi = over_group(hi, [](float a, float b) { return __builtin_elementwise_maximum(a, b); });
    const bool bad = !(lo >= -65504.f) || !(hi <= 65504.f);
    const f16_t s = bad ? (f16_t)NAN : half_of_float((hi - lo) * (1.f / 15.f)), c = bad ? (f16_t)NAN : half_of_float(lo + 8.f * (float)s);
    params = (uint32_t)__builtin_bit_cast(uint16_t, s) | (uint32_t)__builtin_bit_cast(uint16_t, c) << 16;
    const float inv = (float)s == 0.f ? 0.f : __builtin_amdgcn_rcpf((float)s);
    constexpr float ZERO = 12582912.f;             // 1.5 x 2^23, code 0
    uint32_t code = 0, base = 0;
    float off = 0.f;
#pragma unroll
    for (int e = 7; e >= 0; --e) {
        const float q = (x[e] - (float)c) * inv, t = q + (ZERO + 8.f);
        off = fmaxf(off, fabsf(q - (t - (ZERO + 8.f))));
        code = (code << 4) + __float_as_uint(__builtin_amdgcn_fmed3f(t, ZERO, ZERO + 15.f));
        base = (base << 4) + 0x4B400000u;
    }
    code -= base;
    if (__any(off > 0.5f - 0x1p-17f)) {
        code = 0;
#pragma unroll
        for (int e = 7; e >= 0; --e) {
            const float q = (x[e] - (float)c) * inv;
            float u = q + (ZERO + 8.f) - (ZERO + 8.f);
            if (__any(fabsf(q - u) > 0.5f - 0x1p-17f)) u = settle(q, u, x[e], (float)s, (float)c);
            code = code << 4 | (uint32_t)(int)(__builtin_amdgcn_fmed3f(u, -8.f, 7.f) + 8.f);
        }
    }
    return bad || (float)s == 0.f ? 0x88888888u : code;
}

// A wave takes one head of 4 rows (of 64 dims: 8), K and V.  8192 rows of 32 heads of 128 bf16: 40 us, 4.3 TB/s of both directions, bound by vector
// instructions (with the quotients divided, and every one settled in double: 62).
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_kv4_append(Kv4Args a) {
    using L = Kv4<HD>;
    using P = Piece<HD>;
    const int lane = threadIdx.x & 63;
    const unsigned w = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = (int)(w % (unsigned)a.n_kv_heads), r = (int)(w / (unsigned)a.n_kv_heads) * P::ROWS + lane / P::LANES;
    const int slot = r < a.rows ? a.slot[r] : -1;
    const bool there = slot >= 0 && slot / 16 < a.n_pages;
    if (!__any(there)) return;
    const P p(lane, slot);
    constexpr int N = 16 / sizeof(T);
    Vec<T> rk[8 / N], rv[8 / N];
    const T *fk = (const T*)a.k + (size_t)(there ? r : 0) * a.ld_k + (size_t)h * HD + p.d, *fv = (const T*)a.v + (size_t)(there ? r : 0) * a.ld_v + (size_t)h * HD + p.d;
#pragma unroll
    for (int i = 0; i < 8 / N; ++i) {
        rk[i].template load<true>(fk + i * N);
        rv[i].template load<true>(fv + i * N);
    }
    float k[8], v[8];
#pragma unroll
    for (int i = 0; i < 8 / N; ++i) {
        float x[N], y[N];
        rk[i].get(x);
        rv[i].get(y);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            k[i * N + e] = x[e];
            v[i * N + e] = y[e];
        }
    }
    uint32_t pk, pv;
    const uint32_t ck = kv4_pack(k, pk), cv = kv4_pack(v, pv), other = other_nibbles(cv);
    if (!there) return;
    uint8_t* block = (uint8_t*)a.pool + (((size_t)(slot / 16) * a.n_layers + a.layer) * a.n_kv_heads + h) * L::BLOCK;
    *(uint32_t*)(block + p.k_word()) = ck;
    const uint32_t bytes = p.upper() ? merge_nibbles(other >> 16, cv >> 16) : merge_nibbles(cv, other);
#pragma unroll
    for (int j = 0; j < 4; ++j) block[p.v_byte(j)] = (uint8_t)(bytes >> 8 * j);
    if (p.i % 8 == 0) {
        *(uint32_t*)(block + p.param()) = pk;
        *(uint32_t*)(block + p.param() + L::PARAMS) = pv;
    }
}

__device__ __forceinline__ void kv4_unpack(uint32_t code, uint32_t params, float (&x)[8]) {
    const float s = unpack<f16_t>(params, 0), c = unpack<f16_t>(params, 1);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = fmaf(s, (float)((int)(code >> 4 * e & 15) - 8), c);
}

template <typename T> __device__ __forceinline__ void put8(T* to, const float (&x)[8]) {
    constexpr int N = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 8; i += N) {
        float y[N];
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = within<T>(x[i + e]);
        Vec<T> v;
        v.set(y);
        v.template store<false>(to + i);
    }
}

// The same back: 28 us, 6.1 TB/s; every V byte is read by one of two threads and handed to the other.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_kv4_read(Kv4Args a) {
    using L = Kv4<HD>;
    using P = Piece<HD>;
    const int lane = threadIdx.x & 63;
    const unsigned w = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = (int)(w % (unsigned)a.n_kv_heads), r = (int)(w / (unsigned)a.n_kv_heads) * P::ROWS + lane / P::LANES;
    const int slot = r < a.rows ? a.slot[r] : -1;
    const bool there = slot >= 0 && slot / 16 < a.n_pages;
    const P p(lane, slot);
    const uint8_t* block = (const uint8_t*)a.pool + (((size_t)(there ? slot / 16 : 0) * a.n_layers + a.layer) * a.n_kv_heads + h) * L::BLOCK;
    uint32_t ck = 0, bytes = 0, pk = 0, pv = 0;
    if (there) {
        ck = *(const uint32_t*)(block + p.k_word());
#pragma unroll
        for (int j = 0; j < 4; ++j) bytes |= (uint32_t)block[p.v_byte(j)] << 8 * j;
        pk = *(const uint32_t*)(block + p.param());
        pv = *(const uint32_t*)(block + p.param() + L::PARAMS);
    } else if (slot >= 0) {
        pk = pv = 0x7E007E00u;                     // not a number
    }
    const uint32_t other = other_nibbles(bytes), lo = p.upper() ? other : bytes, hi = p.upper() ? bytes : other;      // bytes 0 .. 3 and 4 .. 7
    uint32_t cv = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int at = 8 * j + (p.upper() ? 4 : 0);
        cv |= (lo >> at & 15) << 4 * j | (hi >> at & 15) << (4 * j + 16);
    }
    if (r >= a.rows) return;
    float x[8];
    kv4_unpack(ck, pk, x);
    put8<T>((T*)a.k + (size_t)r * a.ld_k + (size_t)h * HD + p.d, x);
    kv4_unpack(cv, pv, x);
    put8<T>((T*)a.v + (size_t)r * a.ld_v + (size_t)h * HD + p.d, x);
}

size_t kv4_block_bytes(int head_dim) { return (size_t)18 * head_dim; }

template <typename T, bool APPEND>
static hipError_t kv4_typed(hipStream_t st, int head_dim, const Kv4Args& a) {
    const int each = 512 / head_dim, most = (int)std::min<int64_t>((kLaunchThreads / 64 - 4) / a.n_kv_heads * each, 1 << 30);       // rows of a wave; of a launch
    for (int first = 0; first < a.rows; first += most) {
        Kv4Args p = a;
        p.k = (T*)a.k + (size_t)first * a.ld_k;
        p.v = (T*)a.v + (size_t)first * a.ld_v;
        p.slot += first;
        p.rows = std::min(most, a.rows - first);
        const unsigned blocks = (unsigned)(((int64_t)((p.rows + each - 1) / each) * a.n_kv_heads + 3) / 4);
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
