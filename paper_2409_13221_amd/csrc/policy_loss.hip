// Clipped policy loss with a KL term over logits, and its gradient (the formulas are in include/rlhf_ops.h).
// With p = softmax(z) and s = d loss / d l, the gradient of a row is s (onehot(y) - p): a row needs its maximum and its sum of
// exponentials before the first element of the gradient, and nothing else of itself.  Logits are read once and gradients
// written once, which is what bounds it: 8192 rows of 32000 bf16 (a tenth left out) 186 us = 5.3 TB/s, of float, all
// kept, 365 us = 5.7 TB/s; without gradient 4096 rows of 32000 float (a tenth left out) 74 us = 6.4 TB/s.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "vec.h"

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
    RowLoss o{-(cut ? c : u) * w, 0.f, cut ? w : u == u ? 0.f : u, cut ? 0.f : -u * w};
    if (a.lp_ref) {
        const float x = a.lp_ref[r] - l, em = expm1f(x);
        o.kl = (x == INFINITY ? x : em - x) * w;               // a token of probability 0
        if (a.kl_coef != 0.f) o.slope -= a.kl_coef * em * w;
    }
    return o;
}

// Running maximum m and sum s of exp(z - m) of a thread's logits; m = -inf, s = 0 to begin with.  __expf rounds x log2 e, which makes a term
// off by |x| 2^-24 of itself, either way: a sum, whose weight lies near the maximum, does not show it (float rows of 32000, 64 of them:
// with the gradient's exponential here too 12.6 us, so 11.2; log-probs 7.8e-8 off in both).
struct Running {
    float m = -INFINITY, s = 0.f;
    template <int N> __device__ __forceinline__ void add(const float (&x)[N]) {
        float mx = m;
#pragma unroll
        for (int e = 0; e < N; ++e) mx = fmaxf(mx, x[e]);
        const float ref = mx == -INFINITY ? 0.f : mx;          // exp(-inf - 0) is 0, exp(-inf + inf) would be NaN
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) t += __expf(x[e] - ref);
        s = s * __expf(m - ref) + t;
        m = mx;
    }
};

// What joins the waves of a row (up to 16): the maximum M, zy among it, and the sum R of exp(z - M) without zy's.  Every 16 lanes hold
// all waves' pairs.
template <int WAVES>
__device__ __forceinline__ void join_row(const Running& run, float zy, float (*red)[2], float& M, float& R) {
    const int lane = threadIdx.x & 63;
    float m = wave_max(run.m);
    float s = wave_sum(run.s * __expf(run.m - (m == -INFINITY ? 0.f : m)));
    if (WAVES > 1) {
        if (lane == 0) { red[threadIdx.x >> 6][0] = m; red[threadIdx.x >> 6][1] = s; }
        __syncthreads();
        m = red[lane % WAVES][0];
        s = red[lane % WAVES][1];
    }
    M = fmaxf(m, zy);
#pragma unroll
    for (int o = 1; o < WAVES; o <<= 1) M = fmaxf(M, __shfl_xor(M, o, kWave));
    R = s * __expf(m - M);                         // a row of -inf alone gives NaN
#pragma unroll
    for (int o = 1; o < WAVES; o <<= 1) R += __shfl_xor(R, o, kWave);
}

// Scalars of a row, by its first thread: outputs, and the gradient's factors (at the token, elsewhere) to `out`.
__device__ __forceinline__ void finish_row(const PolicyArgs& a, int r, int y, float w, float zy, float M, float R, float* out) {
    const float top = __expf(zy - M), S = R + top;
    // log of the sum and of what its rounding lost, all of R where that is far below a top of 1
    const float l = y < a.vocab ? zy - M - (logf(S) + (R - (S - top)) * __builtin_amdgcn_rcpf(S)) : NAN;
    const RowLoss o = row_loss(a, r, w, l);
    a.lp[r] = l;
    a.terms[r] = o.policy;
    a.terms[a.terms_ld + r] = o.kl;
    a.terms[2 * a.terms_ld + r] = o.cut;
    out[0] = o.slope * a.grad_scale * (R / S);
    out[1] = -o.slope * a.grad_scale / S;
}

// exp(x) of a distance x <= 0 from the maximum, as the gradient shows it column by column.  Gradients of 16 bits are rounded to 2^-8 and
// 2^-11 of themselves, beside which __expf is exact; of float ones it would be the largest error (2.7e-6 of themselves, so 1.2e-6).
template <typename T> __device__ __forceinline__ float exp_of(float x) {
    if (sizeof(T) == 2) return __expf(x);
    constexpr float hi = 1.44269504f, lo = 1.44269504088896340736 - (double)hi;        // log2 e
    const float t = x * hi, p = __builtin_amdgcn_exp2f(t);
    const float lost = fminf(fmaxf(fmaf(x, lo, fmaf(x, hi, -t)), -1.f), 1.f);          // of x log2 e by its rounding; a number where t is -inf
    return fmaf(p, lost * 0.693147181f, p);
}

// The vectors of a row start where what is written of it, or else what is read, reaches a 16-byte boundary; the few columns
// before and behind them go to a thread each.
template <typename T> __device__ __forceinline__ int columns_before(const T* row, int vocab) {
    return min((int)((0 - (uintptr_t)row) % 16 / sizeof(T)), vocab);
}

// The columns of a row outside the threads' streams of vectors, a thread each: those before and behind the vectors, and the vector that
// holds the token (`skip` of its vectors' columns; ~0u where the token is outside them).  The token's own is kept out of the sums:
// of a token that has nearly all of the probability, what matters is what it leaves, and that cannot be had from a sum that holds the
// token's 1 (a token 20 above 32000 others: gradient and log-prob off by 1e-3 of themselves, so 5e-7).  A branch or a select on it in
// each vector of the stream would spill it; a vector left out costs nothing.
struct Single {
    unsigned skip;
    int column;                  // of this thread; the row's length or more where it has none
    template <int N> static __device__ __forceinline__ Single of(int y, int head, unsigned whole, int vocab, int t) {
        const unsigned in = y - head, skip = in < whole ? in / N * N : ~0u;
        const int token = skip != ~0u && t < 3 * N ? head + (int)skip + t - 2 * N : vocab;
        return Single{skip, t >= 2 * N ? token : t < head ? t : t + (int)whole};
    }
};

template <typename T>
__device__ __forceinline__ void left_out_row(const PolicyArgs& a, int r, T* g, int t, int threads) {
    if (t < 3) a.terms[t * a.terms_ld + r] = 0.f;
    if (t == 0) a.lp[r] = 0.f;
    if (!g) return;
    constexpr int N = 16 / sizeof(T);
    Vec<T> zero;
    zero.fill(0.f);
    const int head = columns_before<T>(g, a.vocab), whole = (a.vocab - head) / N * N, odd = t < head ? t : t + whole;
    for (int i = t * N; i < whole; i += threads * N) zero.template store<true>(g + head + i);
    if (odd < a.vocab) g[odd] = round_to<T>(0.f);
}

// A row in registers: IT vectors of 16 bytes a thread, requested all at once.  Each is taken into the thread's running maximum and
// sum as it arrives, so that the exponentials hide behind the loads; the gradient takes them anew from the logits, which
// costs less than room for them in 32 bits would: a 16-bit row of 32000 is 16 registers of 1024 threads, and two such workgroups
// on a compute unit keep one's stores beside the other's loads (3000 rows of 50000 bf16: in 32 bits, one workgroup, 178 us;
// packed, two, 119).  From 13 vectors a thread on there is room for one: 1500 rows of 100003 half, all kept, 135 us = 4.4 TB/s.
// ROWS rows of THREADS threads each in a workgroup; more than one only where a row is one wave's.
template <typename T, int IT, int THREADS, int ROWS, int WAVES_PER_SIMD>
__global__ __launch_bounds__(THREADS * ROWS, WAVES_PER_SIMD) void k_policy_row(PolicyArgs a) {
    static_assert(ROWS == 1 || THREADS == kWave, "rows of more than a wave meet at barriers");
    constexpr int N = 16 / sizeof(T);
    __shared__ float red[THREADS / 64][2];
    __shared__ float s_row[2];
    const int r = blockIdx.x * ROWS + (ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS) : 0), t = threadIdx.x % THREADS, V = a.vocab;
    if (ROWS > 1 && r >= a.rows) return;
    const T* z = (const T*)a.logits + (size_t)r * a.ld;
    T* g = a.grad ? (T*)a.grad + (size_t)r * a.ld_grad : nullptr;
    const int y = a.tokens[r];
    const float w = a.weight ? a.weight[r] : 1.f;
    if (y < 0 || w == 0.f) return left_out_row<T>(a, r, g, t, THREADS);
    const int head = columns_before<T>(g ? g : z, V);
    const unsigned whole = (V - head) / N * N;
    const Single one = Single::of<N>(y, head, whole, V, t);
    z += head;
    if (g) g += head;
    Vec<T> x[IT];
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const unsigned i = (it * THREADS + t) * N;
        if (i < whole && i != one.skip) x[it].template load<true>(z + i);
        else x[it].fill(-INFINITY);
    }
    const float xl = one.column < V ? to_f32<T>(z[one.column - head]) : -INFINITY;
    const float zy = to_f32<T>(z[min(y, V - 1) - head]);
    Running run;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        float f[N];
        x[it].get(f);
        run.add(f);
        x[it].forget();
    }
    const float others[1] = {one.column == y ? -INFINITY : xl};
    run.add(others);
    float M, R, row[2];
    join_row<THREADS / 64>(run, zy, red, M, R);
    if (ROWS > 1) {
        finish_row(a, r, y, w, zy, M, R, row);
        if (!g) return;
    } else {
        if (t == 0) finish_row(a, r, y, w, zy, M, R, s_row);
        if (!g) return;
        __syncthreads();
        row[0] = s_row[0];
        row[1] = s_row[1];
    }
    if (one.column < V) g[one.column - head] = round_to<T>(one.column == y ? row[0] : row[1] * exp_of<T>(xl - M));
    int again = t;                                 // columns are numbered anew for the stores: kept, 22 of them would spill
    asm volatile("" : "+v"(again));
#pragma unroll
    for (int it = 0; it < IT; ++it) {
        const unsigned i = (it * THREADS + again) * N;
        float f[N];
        x[it].get(f);
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = row[1] * exp_of<T>(f[e] - M);
        x[it].set(f);
        if (i < whole && i != one.skip) x[it].template store<true>(g + i);
    }
}

// Rows that no workgroup's registers hold (beyond 90000 floats, 180000 of 16 bits): read once for the statistics, and again, out of
// the caches, for the gradient.  700 rows of 200000 bf16 133 us, of 300000 215 = 3.9 TB/s of what has to be read and written.
template <typename T>
__global__ __launch_bounds__(1024) void k_policy_long_row(PolicyArgs a) {
    constexpr int N = 16 / sizeof(T), IT = 4;
    __shared__ float red[16][2];
    __shared__ float s_row[2];
    const int r = blockIdx.x, t = threadIdx.x, V = a.vocab;
    const T* z = (const T*)a.logits + (size_t)r * a.ld;
    T* g = a.grad ? (T*)a.grad + (size_t)r * a.ld_grad : nullptr;
    const int y = a.tokens[r];
    const float w = a.weight ? a.weight[r] : 1.f;
    if (y < 0 || w == 0.f) return left_out_row<T>(a, r, g, t, 1024);
    const float zy = to_f32<T>(z[min(y, V - 1)]);
    const int head = columns_before<T>(g ? g : z, V), whole = (V - head) / N * N;
    const Single one = Single::of<N>(y, head, whole, V, t);
    const float xl = one.column < V ? to_f32<T>(z[one.column]) : -INFINITY, others[1] = {one.column == y ? -INFINITY : xl};
    z += head;
    if (g) g += head;
    Running run;
    for (int i0 = 0; i0 < whole; i0 += IT * 1024 * N) {
        Vec<T> x[IT];
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int i = i0 + (it * 1024 + t) * N;
            if (i < whole && (unsigned)i != one.skip) x[it].template load<false>(z + i);
            else x[it].fill(-INFINITY);
        }
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            float f[N];
            x[it].get(f);
            run.add(f);
        }
    }
    run.add(others);
    float M, R;
    join_row<16>(run, zy, red, M, R);
    if (t == 0) finish_row(a, r, y, w, zy, M, R, s_row);
    if (!g) return;
    __syncthreads();
    const float f = s_row[1];
    for (int i0 = 0; i0 < whole; i0 += IT * 1024 * N) {
        Vec<T> x[IT];
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int i = i0 + (it * 1024 + t) * N;
            if (i < whole && (unsigned)i != one.skip) x[it].template load<true>(z + i);
        }
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int i = i0 + (it * 1024 + t) * N;
            if (i >= whole) break;
            float d[N];
            x[it].get(d);
#pragma unroll
            for (int e = 0; e < N; ++e) d[e] = f * exp_of<T>(d[e] - M);
            x[it].set(d);
            if ((unsigned)i != one.skip) x[it].template store<true>(g + i);
        }
    }
    if (one.column < V) g[one.column - head] = round_to<T>(one.column == y ? s_row[0] : f * exp_of<T>(xl - M));
}

// Sums of the terms v [3][n] in a fixed order and in double: `each` of a kind a workgroup, to out[3][workgroups], or for one workgroup to
// stats.  The threads' sums meet in LDS, where a wave each takes one of the three: a third of the lane exchanges one after
// the other.
template <int THREADS, typename V>
__global__ __launch_bounds__(THREADS) void k_policy_stats(const V* __restrict__ v, int n, int each, float kl_coef, double* __restrict__ out,
                                                          float* __restrict__ stats) {
    __shared__ double part[3][THREADS], sum[3];
    const unsigned t = threadIdx.x, w = t >> 6, lane = t & 63, lo = blockIdx.x * (unsigned)each, hi = min((unsigned)n, lo + (unsigned)each);
    double s[3] = {0., 0., 0.};
    for (unsigned i = lo + t; i < hi; i += THREADS)
#pragma unroll
        for (int k = 0; k < 3; ++k) s[k] += v[(size_t)k * n + i];
#pragma unroll
    for (int k = 0; k < 3; ++k) part[k][t] = s[k];
    __syncthreads();
    if (w < 3) {
        double x = 0.;
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) x += part[w][i * 64 + lane];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
        if (lane == 0) sum[w] = x;
    }
    __syncthreads();
    if (t >= 3) return;
    if (!stats) { out[t * gridDim.x + blockIdx.x] = sum[t]; return; }
    stats[1 + t] = (float)sum[t];
    if (t == 0) stats[0] = (float)(sum[0] + (kl_coef != 0.f ? kl_coef * sum[1] : 0.));
}
template <typename V> static void last_stats(hipStream_t st, const V* v, int n, float kl_coef, float* stats) {
    if (n <= 1024) k_policy_stats<256, V><<<1, 256, 0, st>>>(v, n, n, kl_coef, nullptr, stats);
    else k_policy_stats<1024, V><<<1, 1024, 0, st>>>(v, n, n, kl_coef, nullptr, stats);
}

// More rows than this are summed in two steps.  Scratch: the rows' terms, and the first step's sums, doubles of two floats each from the next
// boundary of a double on.
constexpr int kStatsRows = 8192;
static int stats_blocks(int rows) { return rows > kStatsRows ? (rows + kStatsRows - 1) / kStatsRows : 0; }
size_t policy_scratch_floats(int rows, int vocab) {
    const size_t blocks = stats_blocks(rows);
    return 3 * ((size_t)rows + 2 * blocks) + (blocks > 0 ? 1 : 0);
}

// As few threads as hold a row with up to 8 vectors each: waves that wait for one another cost more than vectors.  us, with
// gradient, all rows kept: 8192 rows of 4096 bf16: a wave a row 28.0, 2 waves 30.8, 4 31.5, 8 40.1; of 8192: 4 waves 50.8, 8 54.6, a wave
// 57.8; of 16000: 8 waves 93, 16 122; of 32000: 8 waves 187, 4 with 16 vectors 190, 16 with 4 193.  Four rows of a wave share a workgroup
// where they are float (16384 rows of 2000 float 54.7, a workgroup each 57.1; of bf16 35.5 and 34.1, 65536 rows of 1000 bf16 65.4
// and 60.6).
// Beyond 8 vectors of 1024 threads, as many as needed (1200 rows of 104000 bf16: 13 106, 16 109; of 128256: 16 130, 22 136).  Rows that
// fit are kept in registers, which loses only next to where two workgroups a compute unit end, and there little (us, registers and read
// twice, 1200 rows: 65535 bf16 65 and 73, 70000 84 and 80, 85000 96 and 96, 104000 106 and 114, 128256 130 and 143, 160000 162 and
// 178, 180000 183 and 212; float 32771 72 and 74, 50257 105 and 113, 60000 114 and 133, 90000 173 and 208).
template <typename T>
static void policy_rows(hipStream_t st, const PolicyArgs& a) {
    constexpr int N = 16 / sizeof(T), SHARE = sizeof(T) == 4 ? 4 : 1;
#define RLHF_POLICY(IT, THREADS, ROWS, WAVES) \
    if (a.vocab < (IT * THREADS + 1) * N)     \
        return k_policy_row<T, IT, THREADS, ROWS, WAVES><<<(a.rows + ROWS - 1) / ROWS, THREADS * ROWS, 0, st>>>(a)
    RLHF_POLICY(2, 64, SHARE, 8);
    RLHF_POLICY(4, 64, SHARE, 8);
    RLHF_POLICY(8, 64, SHARE, 8);
    RLHF_POLICY(4, 256, 1, 8);
    RLHF_POLICY(4, 512, 1, 8);
    RLHF_POLICY(8, 512, 1, 8);
    RLHF_POLICY(8, 1024, 1, 8);
    RLHF_POLICY(13, 1024, 1, 4);
    RLHF_POLICY(16, 1024, 1, 4);
    RLHF_POLICY(22, 1024, 1, 4);
#undef RLHF_POLICY
    k_policy_long_row<T><<<a.rows, 1024, 0, st>>>(a);
}

// The rows in turns of what one launch holds at the threads a row that policy_rows takes: a wave's 64 (of up to four rows a workgroup), or up
// to 1024.
template <typename T>
static hipError_t policy_parts(hipStream_t st, const PolicyArgs& a) {
    const int64_t most = a.vocab < (8 * 64 + 1) * (16 / (int)sizeof(T)) ? kLaunchThreads / 256 * 4 : kLaunchThreads / 1024;
    for (int64_t first = 0; first < a.rows; first += most) {
        PolicyArgs p = a;
        p.logits = (const T*)a.logits + first * a.ld;
        p.grad = a.grad ? (T*)a.grad + first * a.ld_grad : nullptr;
        p.tokens += first;
        p.weight = a.weight ? a.weight + first : nullptr;
        p.lp_old += first;
        p.lp_ref = a.lp_ref ? a.lp_ref + first : nullptr;
        p.adv += first;
        p.lp += first;
        p.terms += first;
        p.rows = (int)std::min<int64_t>(most, a.rows - first);
        policy_rows<T>(st, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_policy_loss(hipStream_t st, int dtype, const PolicyArgs& a, float* stats) {
    if (a.vocab > 1 << 30 || a.rows > 1 << 30) return hipErrorInvalidValue;          // row and column numbers are ints
    const hipError_t e = dtype == kBF16 ? policy_parts<bf16_t>(st, a) : dtype == kF16 ? policy_parts<f16_t>(st, a) : policy_parts<float>(st, a);
    if (e != hipSuccess) return e;
    const int blocks = stats_blocks(a.rows);
    if (blocks > 0) {
        double* sums = (double*)(((uintptr_t)(a.terms + (size_t)3 * a.rows) + 7) / 8 * 8);
        k_policy_stats<1024, float><<<blocks, 1024, 0, st>>>(a.terms, a.rows, kStatsRows, a.kl_coef, sums, nullptr);
        last_stats(st, sums, blocks, a.kl_coef, stats);
    } else {
        last_stats(st, a.terms, a.rows, a.kl_coef, stats);
    }
    return hipGetLastError();
}

}  // namespace rlhf
