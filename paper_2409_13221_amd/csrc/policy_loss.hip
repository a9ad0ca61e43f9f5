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

// A row in registers: IT vectors of 16 bytes a thread, THREADS threads, read once, all loads in flight together.  Each wave takes
// its own maximum and sum of exponentials, one exchange joins them; the exponentials stay in the registers of the logits, so
// that the gradient is one product away.
template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
    // N elements at p, any alignment
    static __device__ __forceinline__ void load(const T* p, float* o) {
        T v[N];
        __builtin_memcpy(v, p, 16);
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = to_f32<T>(v[e]);
    }
    static __device__ __forceinline__ void store(T* p, const float* x) {
        T v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = from_f32<T>(x[e]);
        __builtin_memcpy(p, v, 16);
    }
};

// What joins the waves of a row (up to 16): maximum and sum of exp(z - maximum).  Every 16 lanes hold all waves' pairs.
template <int WAVES>
__device__ __forceinline__ void join_waves(float m, float s, float (*red)[2], float& M, float& S) {
    const int lane = threadIdx.x & 63;
    if (lane == 0) { red[threadIdx.x >> 6][0] = m; red[threadIdx.x >> 6][1] = s; }
    __syncthreads();
    m = red[lane % WAVES][0];
    s = red[lane % WAVES][1];
    M = m;
#pragma unroll
    for (int o = 1; o < WAVES; o <<= 1) M = fmaxf(M, __shfl_xor(M, o, kWave));
    S = s * __expf(m - M);                         // a row of -inf alone gives NaN
#pragma unroll
    for (int o = 1; o < WAVES; o <<= 1) S += __shfl_xor(S, o, kWave);
}

// Scalars of a row, by its first thread: outputs, and the gradient's factors (at the token, elsewhere) to `out`.
__device__ __forceinline__ void finish_row(const PolicyArgs& a, int r, int y, float w, float zy, float M, float S, float* out) {
    const float l = y < a.vocab ? zy - M - logf(S) : NAN;
    const RowLoss o = row_loss(a, r, w, l);
    a.lp[r] = l;
    a.terms[r] = o.policy;
    a.terms[(size_t)a.rows + r] = o.kl;
    a.terms[(size_t)2 * a.rows + r] = o.cut;
    out[0] = o.slope * a.grad_scale * (1.f - __expf(zy - M) / S);
    out[1] = -o.slope * a.grad_scale / S;
}

template <typename T>
__device__ __forceinline__ void left_out_row(const PolicyArgs& a, int r, T* g, int threads) {
    if (threadIdx.x < 3) a.terms[(size_t)threadIdx.x * a.rows + r] = 0.f;
    if (threadIdx.x == 0) a.lp[r] = 0.f;
    if (!g) return;
    constexpr int N = Vec<T>::N;
    const float zero[N] = {};
    for (int i = threadIdx.x * N; i < a.vocab; i += threads * N) {
        if (i + N <= a.vocab) Vec<T>::store(g + i, zero);
        else for (int e = i; e < a.vocab; ++e) g[e] = from_f32<T>(0.f);
    }
}

template <typename T, int IT, int THREADS, int WAVES_PER_SIMD>
__global__ __launch_bounds__(THREADS, WAVES_PER_SIMD) void k_policy_row(PolicyArgs a) {
    constexpr int N = Vec<T>::N;
    __shared__ float red[THREADS / 64][2];
    __shared__ float s_row[2];
    const int r = blockIdx.x, t = threadIdx.x, V = a.vocab;
    const T* z = (const T*)a.logits + (size_t)r * a.ld;
    T* g = a.grad ? (T*)a.grad + (size_t)r * a.ld_grad : nullptr;
    const int y = a.tokens[r];
    const float w = a.weight ? a.weight[r] : 1.f;
    if (y < 0 || w == 0.f) return left_out_row<T>(a, r, g, THREADS);
    const unsigned whole = V / N * N, last = whole + t;    // columns in vectors; the few behind them, one a thread
    float x[IT][N], xl = -INFINITY;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const unsigned i = (it * THREADS + t) * N;
        if (i < whole) Vec<T>::load(z + i, x[it]);
        else {
#pragma unroll
            for (int e = 0; e < N; ++e) x[it][e] = -INFINITY;
        }
    }
    if (last < (unsigned)V) xl = to_f32<T>(z[last]);
    const float zy = to_f32<T>(z[min(y, V - 1)]);
    float m = xl;
#pragma unroll
    for (int it = 0; it < IT; ++it)
#pragma unroll
        for (int e = 0; e < N; ++e) m = fmaxf(m, x[it][e]);
    m = wave_max(m);
    const float mm = m == -INFINITY ? 0.f : m;             // exp(-inf - 0) is 0, exp(-inf + inf) would be NaN
    float s = 0.f;
#pragma unroll
    for (int it = 0; it < IT; ++it)
#pragma unroll
        for (int e = 0; e < N; ++e) { x[it][e] = __expf(x[it][e] - mm); s += x[it][e]; }
    xl = __expf(xl - mm);
    s += xl;
    float M, S;
    join_waves<THREADS / 64>(m, wave_sum(s), red, M, S);
    if (t == 0) finish_row(a, r, y, w, zy, M, S, s_row);
    if (!g) return;
    __syncthreads();
    const float f = s_row[1] * __expf(mm - M);
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const unsigned i = (it * THREADS + t) * N;
#pragma unroll
        for (int e = 0; e < N; ++e) x[it][e] *= f;
        if (i < whole) Vec<T>::store(g + i, x[it]);
    }
    if (last < (unsigned)V) g[last] = from_f32<T>(xl * f);
    // the token's own column, by the thread that has just written it
    if (y < V && ((unsigned)y >= whole ? (unsigned)y == last : (y / N) % THREADS == t)) g[y] = from_f32<T>(s_row[0]);
}

// Rows that no workgroup's registers hold: read once for the statistics, and again, out of the caches, for the gradient.
template <typename T>
__global__ __launch_bounds__(1024) void k_policy_long_row(PolicyArgs a) {
    constexpr int N = Vec<T>::N;
    __shared__ float red[16][2];
    __shared__ float s_row[2];
    const int r = blockIdx.x, t = threadIdx.x, V = a.vocab;
    const T* z = (const T*)a.logits + (size_t)r * a.ld;
    T* g = a.grad ? (T*)a.grad + (size_t)r * a.ld_grad : nullptr;
    const int y = a.tokens[r];
    const float w = a.weight ? a.weight[r] : 1.f;
    if (y < 0 || w == 0.f) return left_out_row<T>(a, r, g, 1024);
    const float zy = to_f32<T>(z[min(y, V - 1)]);
    float m = -INFINITY, s = 0.f;
    for (int i = t * N; i < V; i += 1024 * N) {
        float x[N];
        if (i + N <= V) Vec<T>::load(z + i, x);
        else
            for (int e = 0; e < N; ++e) x[e] = i + e < V ? to_f32<T>(z[i + e]) : -INFINITY;
        float mx = m;
#pragma unroll
        for (int e = 0; e < N; ++e) mx = fmaxf(mx, x[e]);
        const float mm = mx == -INFINITY ? 0.f : mx;
        s *= m == -INFINITY ? 0.f : __expf(m - mm);
#pragma unroll
        for (int e = 0; e < N; ++e) s += __expf(x[e] - mm);
        m = mx;
    }
    const float mw = wave_max(m);
    s = wave_sum(m == -INFINITY ? s : s * __expf(m - mw));       // s holds NaN where a logit did
    float M, S;
    join_waves<16>(mw, s, red, M, S);
    if (t == 0) finish_row(a, r, y, w, zy, M, S, s_row);
    if (!g) return;
    __syncthreads();
    const float f = s_row[1];
    for (int i = t * N; i < V; i += 1024 * N) {
        float x[N];
        if (i + N <= V) {
            Vec<T>::load(z + i, x);
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = f * __expf(x[e] - M);
            Vec<T>::store(g + i, x);
        } else {
            for (int e = i; e < V; ++e) g[e] = from_f32<T>(f * __expf(to_f32<T>(z[e]) - M));
        }
        if (y >= i && y < min(i + N, V)) g[y] = from_f32<T>(s_row[0]);     // behind the thread's own store to the same place
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

template <typename T>
static void policy_rows(hipStream_t st, const PolicyArgs& a) {
    constexpr int N = Vec<T>::N;
#define RLHF_POLICY(PER_THREAD, THREADS, WAVES) \
    if (a.vocab <= PER_THREAD * THREADS) return k_policy_row<T, PER_THREAD / N, THREADS, WAVES><<<a.rows, THREADS, 0, st>>>(a)
    RLHF_POLICY(16, 256, 8);
    RLHF_POLICY(32, 256, 8);
    RLHF_POLICY(32, 1024, 8);
    RLHF_POLICY(64, 1024, 4);
    RLHF_POLICY(96, 1024, 4);
#undef RLHF_POLICY
    k_policy_long_row<T><<<a.rows, 1024, 0, st>>>(a);
}

hipError_t launch_policy_loss(hipStream_t st, int dtype, const PolicyArgs& a, float* stats) {
    if (a.rows > 0) {
        if (dtype == kBF16) policy_rows<bf16_t>(st, a);
        else if (dtype == kF16) policy_rows<f16_t>(st, a);
        else policy_rows<float>(st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    k_policy_stats<<<1, 256, 0, st>>>(a.terms, a.rows, a.kl_coef, stats);
    return hipGetLastError();
}

}  // namespace rlhf
