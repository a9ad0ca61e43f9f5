// Decode attention with a sliding window and sinks over the paged cache, of the activations' type or of 4 bits
// (include/rlhf_ops.h).
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "kv4.h"
#include "vec.h"

namespace rlhf {

// The visible tokens of a row: pages 0 .. n_sink - 1 and from `first` on, n_pages in all; of them the tokens below `sinks` and
// from lo on, below ctx.
struct Visible {
    int ctx, lo, sinks, n_sink, first, n_pages;
    __device__ __forceinline__ Visible(int ctx_, int window, int sinks_) : ctx(ctx_), lo(max(0, ctx_ - window)), sinks(sinks_) {
        first = lo / 16;
        n_sink = min(first, sinks / 16 + (sinks % 16 != 0));
        n_pages = n_sink + (ctx + 15) / 16 - first;
    }
    __device__ __forceinline__ int page(int i) const { return i < n_sink ? i : first + i - n_sink; }
    __device__ __forceinline__ bool sees(int token) const { return token < ctx && (token >= lo || token < sinks); }
};

// A row of the call: its context, 0 for a row of zeros, -1 where it lies outside page table or samples.
__device__ __forceinline__ int row_context(const WindowDecodeArgs& a, int r, const int*& table) {
    const int ctx = a.ctx_len[r], sample = a.row_sample[r];
    if (ctx <= 0) return 0;
    if (sample < 0 || sample >= a.n_samples || (ctx - 1) / 16 >= a.pt_stride) return -1;
    table = a.page_table + (size_t)sample * a.pt_stride;
    return ctx;
}

// One element of K (or V) of a token of a page.
template <typename T, int HD> struct PlainCache {
    const T* p;
    int heads;
    __device__ PlainCache(const WindowDecodeArgs& a, int page, int kh)
        : p((const T*)a.pool + (((size_t)page * a.n_layers + a.layer) * 2 * a.n_kv_heads + kh) * 16 * HD), heads(a.n_kv_heads) {}
    __device__ float k(int t, int d) const { return to_f32<T>(p[t * HD + d]); }
    __device__ float v(int t, int d) const { return to_f32<T>(p[(size_t)heads * 16 * HD + t * HD + d]); }
};
template <int HD> struct FourBitCache {
    using L = Kv4<HD>;
    const uint8_t* p;
    __device__ FourBitCache(const WindowDecodeArgs& a, int page, int kh)
        : p((const uint8_t*)a.pool + (((size_t)page * a.n_layers + a.layer) * a.n_kv_heads + kh) * L::BLOCK) {}
    __device__ float value(int at, int bit, int par) const {
        const f16_t* sc = (const f16_t*)(p + par);
        return (float)sc[1] + (float)sc[0] * (float)((p[at] >> bit & 15) - 8);
    }
    __device__ float k(int t, int d) const { return value(L::k_byte(t, d), L::k_bit(d), L::param(t, d)); }
    __device__ float v(int t, int d) const { return value(L::v_byte(t, d), L::v_bit(d), L::param(t, d) + L::PARAMS); }
};

// A wave takes a row, a query head and a part of the row's visible pages.
template <typename T, typename Cache, int HD>
__global__ __launch_bounds__(64) void k_window_decode(WindowDecodeArgs a) {
    const int lane = threadIdx.x;
    const int split = blockIdx.x % a.nsplit, h = blockIdx.x / a.nsplit % a.n_q_heads, r = blockIdx.x / a.nsplit / a.n_q_heads;
    const int kh = h / (a.n_q_heads / a.n_kv_heads);
    constexpr int D = HD / 64;
    const int* table = nullptr;
    const int ctx = row_context(a, r, table);
    const T* q = (const T*)a.q + (size_t)r * a.ld_q + (size_t)h * HD;
    float m = -INFINITY, l = 0.f, acc[D] = {};
    bool lost = ctx < 0;
    if (ctx > 0) {
        const Visible see(ctx, a.window, a.sinks);
        const int from = (int)((int64_t)see.n_pages * split / a.nsplit), to = (int)((int64_t)see.n_pages * (split + 1) / a.nsplit);
        for (int i = from; i < to; ++i) {
            const int pi = see.page(i), id = table[pi];
            if (id < 0 || id >= a.n_pages) { lost = true; break; }
            const Cache c(a, id, kh);
            float s = -INFINITY;
            if (lane < 16 && see.sees(pi * 16 + lane)) {
                s = 0.f;
                for (int d = 0; d < HD; ++d) s += to_f32<T>(q[d]) * c.k(lane, d);
                s *= rsqrtf((float)HD);
            }
            const float mn = fmaxf(m, wave_max(s)), ref = mn == -INFINITY ? 0.f : mn, keep = expf(m - ref);
            const float p = lane < 16 && see.sees(pi * 16 + lane) ? expf(s - ref) : 0.f;
            m = mn;
            l = l * keep + wave_sum(p);
#pragma unroll
            for (int e = 0; e < D; ++e) acc[e] *= keep;
            for (int t = 0; t < 16; ++t) {
                const float pt = __shfl(p, t, kWave);
                if (!see.sees(pi * 16 + t)) continue;
#pragma unroll
                for (int e = 0; e < D; ++e) acc[e] += pt * c.v(t, e * 64 + lane);
            }
        }
    }
    if (lost) l = NAN;
    if (a.nsplit == 1) {
        T* o = (T*)a.out + (size_t)r * a.ld_out + (size_t)h * HD;
#pragma unroll
        for (int e = 0; e < D; ++e) o[e * 64 + lane] = round_to<T>(ctx == 0 ? 0.f : acc[e] / l);
    } else {
        const size_t slot = blockIdx.x, slots = (size_t)a.rows * a.n_q_heads * a.nsplit;
        if (lane == 0) { a.part[2 * slot] = m; a.part[2 * slot + 1] = l; }
#pragma unroll
        for (int e = 0; e < D; ++e) a.part[2 * slots + slot * HD + e * 64 + lane] = acc[e];
    }
}

// The parts of a (row, query head) joined, a wave each.
template <typename T, int HD>
__global__ __launch_bounds__(64) void k_window_join(WindowDecodeArgs a) {
    const int lane = threadIdx.x, h = blockIdx.x % a.n_q_heads, r = blockIdx.x / a.n_q_heads;
    constexpr int D = HD / 64;
    const size_t slot = (size_t)blockIdx.x * a.nsplit, slots = (size_t)a.rows * a.n_q_heads * a.nsplit;
    const float2* ml = (const float2*)a.part + slot;
    float m = -INFINITY, l = 0.f, acc[D] = {};
    for (int s = 0; s < a.nsplit; ++s) m = fmaxf(m, ml[s].x);
    const float ref = m == -INFINITY ? 0.f : m;
    for (int s = 0; s < a.nsplit; ++s) {
        const float w = expf(ml[s].x - ref);
        l += w * ml[s].y;
#pragma unroll
        for (int e = 0; e < D; ++e) acc[e] += w * a.part[2 * slots + (slot + s) * HD + e * 64 + lane];
    }
    const bool empty = a.ctx_len[r] <= 0;
    T* o = (T*)a.out + (size_t)r * a.ld_out + (size_t)h * HD;
#pragma unroll
    for (int e = 0; e < D; ++e) o[e * 64 + lane] = round_to<T>(empty ? 0.f : acc[e] / l);
}

int window_decode_nsplit(int rows, int n_q_heads, int n_kv_heads, int max_ctx, int window, int sinks) {
    const int64_t pages = std::min<int64_t>((max_ctx + 15ll) / 16, (sinks + 15ll) / 16 + (window + 15ll) / 16 + 1);
    const int64_t blocks = (int64_t)rows * n_q_heads;
    return (int)std::max<int64_t>(1, std::min<int64_t>({64, pages / 4, 2048 / blocks}));
}

size_t window_decode_scratch_floats(int rows, int n_q_heads, int head_dim, int nsplit) {
    return (size_t)rows * n_q_heads * nsplit * (head_dim + 2);
}

template <typename T, bool FOUR, int HD>
static hipError_t decode_rows(hipStream_t st, const WindowDecodeArgs& a) {
    using Cache = std::conditional_t<FOUR, FourBitCache<HD>, PlainCache<T, HD>>;
    const int most = (int)std::min<int64_t>(std::max<int64_t>(1, kLaunchThreads / 64 / a.n_q_heads / a.nsplit), 1 << 24);
    for (int first = 0; first < a.rows; first += most) {
        WindowDecodeArgs p = a;
        p.q = (const T*)a.q + (size_t)first * a.ld_q;
        p.out = (T*)a.out + (size_t)first * a.ld_out;
        p.row_sample += first;
        p.ctx_len += first;
        p.rows = std::min(most, a.rows - first);
        const unsigned heads = (unsigned)p.rows * (unsigned)a.n_q_heads;
        k_window_decode<T, Cache, HD><<<heads * a.nsplit, 64, 0, st>>>(p);
        if (a.nsplit > 1) k_window_join<T, HD><<<heads, 64, 0, st>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
static hipError_t decode_typed(hipStream_t st, bool four, int hd, const WindowDecodeArgs& a) {
    if (four) return hd == 128 ? decode_rows<T, true, 128>(st, a) : decode_rows<T, true, 64>(st, a);
    return hd == 128 ? decode_rows<T, false, 128>(st, a) : decode_rows<T, false, 64>(st, a);
}

hipError_t launch_window_decode(hipStream_t st, int dtype, bool four_bits, int head_dim, const WindowDecodeArgs& a) {
    return dtype == kBF16 ? decode_typed<bf16_t>(st, four_bits, head_dim, a)
         : dtype == kF16  ? decode_typed<f16_t>(st, four_bits, head_dim, a)
                          : decode_typed<float>(st, four_bits, head_dim, a);
}

}  // namespace rlhf
