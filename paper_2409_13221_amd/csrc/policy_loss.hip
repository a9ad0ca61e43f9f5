// Clipped policy loss with a KL term over logits, and its gradient (the formulas are in include/rlhf_ops.h).
// One workgroup per row: maximum, sum of exponentials, the row's scalars, then the gradient.
#include "common.h"
#include "kernels.h"

namespace rlhf {

// What a row needs after l = log_softmax(z)[y]: its three sums' terms and d loss / d l.
struct RowLoss { float policy, kl, cut, slope; };
__device__ __forceinline__ RowLoss row_loss(const PolicyArgs& a, int r, float w, float l) {
    const float adv = a.adv[r];
    const float rho = expf(l - a.lp_old[r]);
    const float held = rho < a.lo ? a.lo : rho > a.hi ? a.hi : rho;       // a NaN stays one, here and below
    const auto times = [adv](float x) { return adv == 0.f && x == x ? 0.f : x * adv; };    // 0, for a ratio that overflows too
    const float u = times(rho), c = times(held);
    const bool cut = u > c;
    RowLoss o{-(cut ? c : u) * w, 0.f, cut ? w : 0.f, cut ? 0.f : -u * w};
    if (a.lp_ref) {
        const float x = a.lp_ref[r] - l, em = expm1f(x);
        o.kl = (em - x) * w;
        if (a.kl_coef != 0.f) o.slope -= a.kl_coef * em * w;
    }
    return o;
}

__device__ __forceinline__ float block_max(float v, float* red) {
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float m = red[0];
    for (int i = 1; i < (int)blockDim.x >> 6; ++i) m = fmaxf(m, red[i]);
    return m;
}

template <typename T>
__global__ __launch_bounds__(256) void k_policy_row(PolicyArgs a) {
    __shared__ float red[16];
    __shared__ float s_row[2];
    const int r = blockIdx.x, t = threadIdx.x, V = a.vocab;
    const T* z = (const T*)a.logits + (size_t)r * a.ld;
    T* g = a.grad ? (T*)a.grad + (size_t)r * a.ld_grad : nullptr;
    const int y = a.tokens[r];
    const float w = a.weight ? a.weight[r] : 1.f;
    if (y < 0 || w == 0.f) {
        if (t == 0) { a.lp[r] = 0.f; for (int k = 0; k < 3; ++k) a.terms[(size_t)k * a.rows + r] = 0.f; }
        if (g) for (int i = t; i < V; i += 256) g[i] = from_f32<T>(0.f);
        return;
    }
    float m = -INFINITY;
    for (int i = t; i < V; i += 256) m = fmaxf(m, to_f32<T>(z[i]));
    m = block_max(m, red);
    float s = 0.f;
    for (int i = t; i < V; i += 256) s += expf(to_f32<T>(z[i]) - m);
    s = block_sum(s, red);
    if (t == 0) {
        const float l = y < V ? to_f32<T>(z[y]) - m - logf(s) : NAN;
        const RowLoss o = row_loss(a, r, w, l);
        a.lp[r] = l;
        a.terms[r] = o.policy;
        a.terms[(size_t)a.rows + r] = o.kl;
        a.terms[(size_t)2 * a.rows + r] = o.cut;
        s_row[0] = o.slope * a.grad_scale;
        s_row[1] = 1.f / s;
    }
    __syncthreads();
    if (!g) return;
    const float c = s_row[0], inv = s_row[1];
    for (int i = t; i < V; i += 256) {
        const float p = expf(to_f32<T>(z[i]) - m) * inv;
        g[i] = from_f32<T>(i == y ? c * (1.f - p) : -c * p);
    }
}

// The loss and its parts: every row's terms, summed in a fixed order.
__global__ __launch_bounds__(256) void k_policy_stats(const float* __restrict__ terms, int rows, float kl_coef, float* __restrict__ stats) {
    __shared__ double red[3][4];
    double s[3] = {0., 0., 0.};
    for (int i = threadIdx.x; i < rows; i += 256)
        for (int k = 0; k < 3; ++k) s[k] += terms[(size_t)k * rows + i];
    for (int k = 0; k < 3; ++k) {
        for (int o = 32; o > 0; o >>= 1) s[k] += __shfl_xor(s[k], o, kWave);
        if ((threadIdx.x & 63) == 0) red[k][threadIdx.x >> 6] = s[k];
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 0; k < 3; ++k) s[k] = (red[k][0] + red[k][1]) + (red[k][2] + red[k][3]);
        stats[0] = (float)(s[0] + (kl_coef != 0.f ? kl_coef * s[1] : 0.));
        stats[1] = (float)s[0];
        stats[2] = (float)s[1];
        stats[3] = (float)s[2];
    }
}

size_t policy_scratch_floats(int rows, int vocab) { return (size_t)3 * rows; }

hipError_t launch_policy_loss(hipStream_t st, int dtype, const PolicyArgs& a, float* stats) {
    if (a.rows > 0) {
        if (dtype == kBF16) k_policy_row<bf16_t><<<a.rows, 256, 0, st>>>(a);
        else if (dtype == kF16) k_policy_row<f16_t><<<a.rows, 256, 0, st>>>(a);
        else k_policy_row<float><<<a.rows, 256, 0, st>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    k_policy_stats<<<1, 256, 0, st>>>(a.terms, a.rows, a.kl_coef, stats);
    return hipGetLastError();
}

}  // namespace rlhf
