// Packed causal attention with a sliding window and sinks (the formulas are in include/rlhf_ops.h).
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "vec.h"

namespace rlhf {

// One query by one wave: lanes take 64 visible keys at a time for the scores, then HD / 64 dims each for the sum.  Only keys that the query
// sees are touched.
template <typename T, int HD>
__device__ void window_row(const WindowArgs& a, int s0, int i, int h, int lane) {
    const int kh = h / (a.n_q_heads / a.n_kv_heads);
    const T* q = (const T*)a.q + (size_t)(s0 + i) * a.ld_q + (size_t)h * HD;
    const T* k = (const T*)a.k + (size_t)s0 * a.ld_k + (size_t)kh * HD;
    const T* v = (const T*)a.v + (size_t)s0 * a.ld_v + (size_t)kh * HD;
    const float scale = rsqrtf((float)HD);
    const int lo = max(0, i - a.window + 1), n_sink = min(a.sinks, lo), n = n_sink + i - lo + 1;
    constexpr int D = HD / 64;
    float m = -INFINITY, l = 0.f, acc[D] = {};
    for (int c = 0; c < n; c += 64) {
        const int mine = c + lane, j = mine < n_sink ? mine : lo + mine - n_sink;
        float s = -INFINITY;
        if (mine < n) {
            s = 0.f;
            for (int d = 0; d < HD; d += 8) {
                float x[8], y[8];
                load8<T>(q + d, x);
                load8<T>(k + (size_t)j * a.ld_k + d, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) s += x[e] * y[e];
            }
            s *= scale;
        }
        const float mn = fmaxf(m, wave_max(s)), ref = mn == -INFINITY ? 0.f : mn, p = mine < n ? expf(s - ref) : 0.f, keep = expf(m - ref);
        m = mn;
        l = l * keep + wave_sum(p);
#pragma unroll
        for (int e = 0; e < D; ++e) acc[e] *= keep;
        for (int t = 0; t < min(64, n - c); ++t) {
            const int at = c + t, jj = at < n_sink ? at : lo + at - n_sink;
            const float pt = __shfl(p, t, kWave);
#pragma unroll
            for (int e = 0; e < D; ++e) acc[e] += pt * to_f32<T>(v[(size_t)jj * a.ld_v + e * 64 + lane]);
        }
    }
    T* o = (T*)a.out + (size_t)(s0 + i) * a.ld_out + (size_t)h * HD;
#pragma unroll
    for (int e = 0; e < D; ++e) o[e * 64 + lane] = round_to<T>(acc[e] / l);
}

// Whether a tile lies within the rows of the call; what it covers.
__device__ __forceinline__ bool tile_of(const WindowArgs& a, int tile, int& s0, int& q0, int& len) {
    s0 = a.tile_start[tile];
    q0 = a.tile_q0[tile];
    len = a.tile_len[tile];
    return s0 >= 0 && q0 >= 0 && len <= a.rows - s0 && q0 < len;
}

template <typename T, int HD>
__global__ __launch_bounds__(256) void k_window_rows(WindowArgs a) {
    int s0, q0, len;
    if (!tile_of(a, blockIdx.x / a.n_q_heads, s0, q0, len)) return;
    const int h = blockIdx.x % a.n_q_heads, lane = threadIdx.x & 63;
    for (int i = q0 + (threadIdx.x >> 6); i < min(len, q0 + kFlashTile); i += 4) window_row<T, HD>(a, s0, i, h, lane);
}

template <typename T>
static hipError_t window_typed(hipStream_t st, int head_dim, const WindowArgs& a) {
    const int most = (int)std::min<int64_t>(kLaunchThreads / 256 / a.n_q_heads, 1 << 30);
    for (int first = 0; first < a.n_tiles; first += most) {
        WindowArgs p = a;
        p.tile_start += first;
        p.tile_q0 += first;
        p.tile_len += first;
        p.n_tiles = std::min(most, a.n_tiles - first);
        const unsigned blocks = (unsigned)p.n_tiles * (unsigned)a.n_q_heads;
        if (head_dim == 128) k_window_rows<T, 128><<<blocks, 256, 0, st>>>(p);
        else k_window_rows<T, 64><<<blocks, 256, 0, st>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_window_attention(hipStream_t st, int dtype, int head_dim, const WindowArgs& a) {
    return dtype == kBF16 ? window_typed<bf16_t>(st, head_dim, a) : dtype == kF16 ? window_typed<f16_t>(st, head_dim, a) : window_typed<float>(st, head_dim, a);
}

}  // namespace rlhf
