// Packed causal attention with a sliding window and sinks (the formulas are in include/rlhf_ops.h).
#include <algorithm>

#include "attn_tile.h"
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

// Whether a tile lies within the rows of the call and has queries from `part` on; what it covers.
__device__ __forceinline__ bool tile_of(const WindowArgs& a, int tile, int part, int& s0, int& q0, int& len) {
    s0 = a.tile_start[tile];
    q0 = a.tile_q0[tile];
    len = a.tile_len[tile];
    if (s0 < 0 || q0 < 0 || len > a.rows - s0 || q0 >= len) return false;
    q0 += part;
    return q0 < len;
}

// Workgroup -> (tile, first query in it, query head).  Units of a tile and KV head, whose query heads share K and V, go to the XCDs in turn, so that
// keys are read into one L2; the last tiles, with the most keys, come first (units side by side: 16384 tokens 1808 -> 1988 us, 2 x 8192 of
// 32 / 8 heads, window 1024 293 -> 318; tiles from the first: 8192 tokens of 32 heads 542 -> 642).
template <int QUERIES> __device__ __forceinline__ bool window_work(const WindowArgs& a, int& tile, int& part, int& h) {
    constexpr unsigned PARTS = kFlashTile / QUERIES;
    const unsigned G = a.n_q_heads / a.n_kv_heads, all = blockIdx.x / 8, i = all / PARTS, unit = i / G * 8 + blockIdx.x % 8;
    if (unit >= (unsigned)a.n_tiles * (unsigned)a.n_kv_heads) return false;
    tile = a.n_tiles - 1 - (int)(unit / a.n_kv_heads);
    part = (int)(PARTS - 1 - all % PARTS) * QUERIES;
    h = (int)(unit % a.n_kv_heads * G + i % G);
    return true;
}

// Key tiles of SIZE keys that queries first .. last see any of: 0 .. n_sink - 1 and from `from` on.
template <int SIZE> struct KeyTiles {
    int n_sink, from, n;
    __device__ __forceinline__ KeyTiles(int first, int last, int window, int sinks) {
        from = max(0, first - window + 1) / SIZE;
        n_sink = min(from, sinks / SIZE + (sinks % SIZE != 0));
        n = n_sink + last / SIZE - from + 1;
    }
    __device__ __forceinline__ int at(int j) const { return j < n_sink ? j : from + j - n_sink; }
};

__device__ __forceinline__ bool window_sees(const WindowArgs& a, int i, int j) { return j <= i && (j > i - a.window || j < a.sinks); }

typedef __attribute__((address_space(3))) void* lds_ptr_t;
__device__ __forceinline__ uint32_t lds_address(void* p) { return (uint32_t)(size_t)(lds_ptr_t)p; }
// 16 bytes a lane from base + lane + offset to LDS, `to` and on: 1024 bytes of a wave.  Written out, as the builtin makes the compiler wait for all loads in
// flight before it reads LDS; whoever reads waits for vmcnt and the workgroup first.  (It has no register to come back to; m0 has no other use in
// these kernels.)
__device__ __forceinline__ void load_to_lds(u32x4_t base, uint32_t lane, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(lane), "s"(base), "s"(offset) : "memory");
}
__device__ __forceinline__ u32x4_t buffer_base(const void* p) {
    return u32x4_t{(uint32_t)(uintptr_t)p, (uint32_t)((uintptr_t)p >> 32) & 0xFFFFu, 0xFFFFFFFFu, 0x00020000u};
}
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_t;

// References beyond this (log2) are off by more than a factor of 2 from the score that they were taken from, and weights then leave the range of
// their type: such queries are taken again, too.
constexpr float kFarthest = 0x1p24f;

// 16-bit types: 128 queries of a head a workgroup, 32 a wave, against 32 keys at a time.  K and V go from memory to LDS directly, one tile ahead;
// V is transposed as it is read from LDS, and the weights stay in the lanes that made them.  References of the weights follow the running maximum only
// where these would leave their range, so that most tiles do not rescale the sums.  A key that is hidden from a query has weight 0, and 0 times
// what is not a number is none: a wave whose result is not finite takes its queries again one by one, over visible keys alone.
// 32 keys leave registers for three workgroups a compute unit, 64 for two (64 instead: 16384 tokens 1808 -> 1871 us, 16 sequences of 200-800 85 -> 90; heads
// of 64 gain with long contexts, 4 x 4096 162 -> 150, and lose with short ones, 40 of 1-700 30.5 -> 31.6).
// 16384 tokens of 64 / 8 heads of 128, window 4096: 1.79 ms, 1.08 PFLOP/s of visible keys, the chip at its power limit (1.6 to 1.9 GHz).
// 16 sequences of 200-800, window 256: 80 us, 3.3 TB/s where a copy reaches 4.7.  Weights go to the matrix units rounded once to the type, of which an
// output is off by up to half a step of the values' spread (two terms would cost as many products again); what it is divided by is the sum of the rounded
// weights, by the matrix units too, so that equal values come out as they are.
template <typename T, int HD>
__global__ __launch_bounds__(256, 3) void k_window_flash(WindowArgs a) {
    using M = Matrix16<T>;
    constexpr int KT = 32, NF = KT / 16, NU = KT / 32, KS = HD / 32, DF = HD / 16, CH = HD / 8, ROWS = 64 / CH, LOADS = KT / (4 * ROWS), TILE = KT * HD;
    constexpr float START = M::TOP > 0.f ? 6.f : 0.f, MOST = M::TOP > 0.f ? M::TOP : 20.f;      // log2 of the greatest weight at a new reference, and ever
    __shared__ __attribute__((aligned(16))) T sK[2][TILE], sV[2][TILE];
    int tile, part, h, s0, q0, len;
    if (!window_work<kFlashTile>(a, tile, part, h) || !tile_of(a, tile, part, s0, q0, len)) return;
    const int kh = h / (a.n_q_heads / a.n_kv_heads);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, c = lane >> 4;
    constexpr float unit = kScoreUnit<HD>;
    const T* kb = (const T*)a.k + (size_t)s0 * a.ld_k + (size_t)kh * HD;
    const T* vb = (const T*)a.v + (size_t)s0 * a.ld_v + (size_t)kh * HD;
    const uint32_t ldk = (uint32_t)a.ld_k * 2, ldv = (uint32_t)a.ld_v * 2;

    // A load of a wave fills ROWS rows of a tile; place p of row t holds 16-byte piece p ^ (t % 16) of K and p ^ 4 (t % 4) of V (of 64 dims
    // ^ (t / 2 % 8) and ^ 4 (t / 2 % 2)), so that fragment reads spread over the banks.
    const int lrow = wave * ROWS + lane / CH, place = lane % CH;
    const int kpiece = CH == 16 ? place ^ (lrow & 15) : place ^ ((lrow >> 1) & 7), vpiece = CH == 16 ? place ^ ((lrow & 3) << 2) : place ^ (((lrow >> 1) & 1) << 2);
    const uint32_t kat = lrow * ldk + kpiece * 16, vat = lrow * ldv + vpiece * 16;
    const auto fetch = [&](int kt, int buf) {
        const u32x4_t rk = buffer_base(kb + (size_t)kt * KT * a.ld_k), rv = buffer_base(vb + (size_t)kt * KT * a.ld_v);
        const int last = len - 1 - kt * KT;
        if (last >= KT - 1) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load_to_lds(rk, kat, i * 4 * ROWS * ldk, lds_address(&sK[buf][(wave + i * 4) * ROWS * HD]));
#pragma unroll
            for (int i = 0; i < LOADS; ++i) load_to_lds(rv, vat, i * 4 * ROWS * ldv, lds_address(&sV[buf][(wave + i * 4) * ROWS * HD]));
        } else {                                   // rows behind the sequence: its last one
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const uint32_t row = min(lrow + i * 4 * ROWS, last);
                load_to_lds(rk, row * ldk + kpiece * 16, 0, lds_address(&sK[buf][(wave + i * 4) * ROWS * HD]));
                load_to_lds(rv, row * ldv + vpiece * 16, 0, lds_address(&sV[buf][(wave + i * 4) * ROWS * HD]));
            }
        }
    };

    const KeyTiles<KT> keys(q0, min(q0 + kFlashTile, len) - 1, a.window, a.sinks);
    fetch(keys.at(0), 0);
    const int w0 = q0 + wave * 32;                 // this wave's queries
    u32x4_t q[2][KS];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const T* p = (const T*)a.q + (size_t)(s0 + min(w0 + m * 16 + n, len - 1)) * a.ld_q + (size_t)h * HD + c * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[m][s] = *(const u32x4_t*)(p + s * 32);
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(q[0][s]), "+v"(q[1][s]));              // here, not in the loop, where a wait for them would be one for K and V
    f32x4_t o[DF][2];
#pragma unroll
    for (int d = 0; d < DF; ++d)
#pragma unroll
        for (int m = 0; m < 2; ++m) o[d][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    f32x4_t l[2] = {};                             // sums of the weights, in every row of the product
    float ref[2] = {-1e30f, -1e30f};
    bool far = false;
    // Token (modulo 16) of a lane's reads of V.  Sums d and d + 1 (even d) of a lane are dims 16 d + 8 c .. + 7, so that it stores 16 bytes at a time (16
    // sequences of 200-800, 32 heads of 128, window 1: 62.6 -> 58.4 us, 4.5 TB/s).
    const int vt = 4 * c + (n >> 2);
    const int vswap = (CH == 16 ? vt & 3 : (vt >> 1) & 1) << 2;

    if (keys.n > 1) fetch(keys.at(1), 1);
    for (int j = 0; j < keys.n; ++j) {
        const int kt = keys.at(j), buf = j & 1, first = kt * KT, last = first + KT - 1;
        if (j == 0 && keys.n > 1) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        __syncthreads();                           // tile j is there, and nobody reads tile j - 1 any more
        if (j > 0 && j + 1 < keys.n) fetch(keys.at(j + 1), buf ^ 1);
        if (w0 >= len || first > w0 + 31 || (last <= w0 - a.window && first >= a.sinks)) continue;       // nothing that this wave sees
        f32x4_t s[NF][2];
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int m = 0; m < 2; ++m) s[f][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                const int row = f * 16 + n, p = CH == 16 ? (k * 4 + c) ^ n : (k * 4 + c) ^ ((n >> 1) & 7);
                const u32x4_t x = *(const u32x4_t*)&sK[buf][row * HD + p * 8];
#pragma unroll
                for (int m = 0; m < 2; ++m) s[f][m] = M::qk(x, q[m][k], s[f][m]);
            }
        if (last > w0 || !(first > w0 + 31 - a.window || last < a.sinks)) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!window_sees(a, w0 + m * 16 + n, first + f * 16 + 4 * c + r)) s[f][m][r] = -INFINITY;
        }
        float top[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            float x = s[0][m][0];
#pragma unroll
            for (int e = 1; e < 4 * NF; ++e) x = __builtin_elementwise_maximum(x, s[e / 4][m][e % 4]);         // one instruction for two; a score that is no number shows in the result
            top[m] = x * unit;
        }
        if (__any(top[0] > ref[0] + MOST || top[1] > ref[1] + MOST)) {
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const float high = column_max(top[m]), now = high > ref[m] + MOST ? high - START : ref[m], keep = __builtin_amdgcn_exp2f(ref[m] - now);
                far |= __any(now != ref[m] && fabsf(now) > kFarthest);
                ref[m] = now;
                l[m] *= keep;
#pragma unroll
                for (int d = 0; d < DF; ++d) o[d][m] *= keep;
            }
        }
        u32x4_t p[2][NU];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                float w[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = __builtin_amdgcn_exp2f(fmaf(s[f][m][r], unit, -ref[m]));
                p[m][f >> 1][(f & 1) * 2] = pack2<T>(w[0], w[1]);
                p[m][f >> 1][(f & 1) * 2 + 1] = pack2<T>(w[2], w[3]);
            }
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int m = 0; m < 2; ++m) l[m] = M::qk(u32x4_t{M::ONES, M::ONES, M::ONES, M::ONES}, p[m][u], l[m]);
#pragma unroll
        for (int d = 0; d < DF; ++d)
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                T* at = &sV[buf][(u * 32 + vt) * HD + ((d / 2 * 4 + (n & 3)) ^ vswap) * 8 + (d & 1) * 4];
                const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(at + 16 * HD));
                const u32x2_t x = __builtin_bit_cast(u32x2_t, lo), y = __builtin_bit_cast(u32x2_t, hi);
#pragma unroll
                for (int m = 0; m < 2; ++m) o[d][m] = M::qk(u32x4_t{x[0], x[1], y[0], y[1]}, p[m][u], o[d][m]);
            }
    }

    float odd = 0.f;                               // not a number where a result is not finite
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const float inv = 1.f / l[m][0];
        const int i = w0 + m * 16 + n;
        if (i >= len) continue;
        T* out = (T*)a.out + (size_t)(s0 + i) * a.ld_out + (size_t)h * HD + 8 * c;
#pragma unroll
        for (int d = 0; d < DF; d += 2) {
            const f32x4_t x = o[d][m] * inv, y = o[d + 1][m] * inv;
            odd += 0.f * (((x[0] + x[1]) + (x[2] + x[3])) + ((y[0] + y[1]) + (y[2] + y[3])));
            *(u32x4_t*)(out + d * 16) = u32x4_t{pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3])};
        }
    }
    if (far || __any(odd != 0.f))
        for (int i = w0; i < min(w0 + 32, len); ++i) window_row<T, HD>(a, s0, i, h, lane);
}

// Float: 128 or 64 queries of a head a workgroup, 16 a wave, against 16 keys at a time, which go to LDS a tile ahead; bound by the float matrix rate (a tenth
// of the half one).  What is hidden is kept out as above.  8192 tokens of 64 / 8 heads of 128, window 1024: 2.11 ms, 123 TFLOP/s with the hidden part of
// the tiles (waves that read keys from memory for themselves: 3.29); 16 sequences of 200-800, 32 heads, window 256: 288 us (456).
// Four waves where tiles are mostly full: twice as many workgroups, nearer to each other in length (2 x 767, 8 heads of 128: 106 us with eight, 71 with
// four; 2000 tokens of 32 heads 363, 316; 4 x 4096, 12 of 64, window 1024 457, 409; two instead of four: 104, 404, 433); of short sequences the
// second half would be empty (256 of 20-60, 32 heads of 128 165, 228; 32 of 100, 40 of 64 42.6, 44.7).
template <int HD, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 4) void k_window_float(WindowArgs a) {
    constexpr int KT = 16, D = HD / 16, CH = HD / 4, ROWS = 64 / CH, EACH = KT / ROWS, LOADS = 2 * EACH / WAVES, TILE = KT * HD, QUERIES = 16 * WAVES;
    __shared__ __attribute__((aligned(16))) float sK[2][TILE], sV[2][TILE];
    int tile, part, h, s0, q0, len;
    if (!window_work<QUERIES>(a, tile, part, h) || !tile_of(a, tile, part, s0, q0, len)) return;
    const int kh = h / (a.n_q_heads / a.n_kv_heads);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, c = lane >> 4;
    const int w0 = q0 + wave * 16;
    const float* kb = (const float*)a.k + (size_t)s0 * a.ld_k + (size_t)kh * HD;
    const float* vb = (const float*)a.v + (size_t)s0 * a.ld_v + (size_t)kh * HD;
    constexpr float unit = kScoreUnit<HD>;
    // Place p of row t of K holds 16-byte piece p ^ t, so that a piece of 16 rows spreads over the banks; V lies as it is.  A load of a wave fills ROWS rows; of
    // the 2 EACH loads of a tile, K first, a wave takes every WAVES-th.
    const auto fetch = [&](int kt, int buf) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int load = wave + i * WAVES, first = load % EACH * ROWS, row = first + lane / CH, place = lane % CH;
            const uint32_t at = min(row, len - 1 - kt * KT);         // rows behind the sequence: its last one
            if (load < EACH) load_to_lds(buffer_base(kb + (size_t)kt * KT * a.ld_k), at * (uint32_t)a.ld_k * 4 + (place ^ row) * 16, 0, lds_address(&sK[buf][first * HD]));
            else load_to_lds(buffer_base(vb + (size_t)kt * KT * a.ld_v), at * (uint32_t)a.ld_v * 4 + place * 16, 0, lds_address(&sV[buf][first * HD]));
        }
    };
    const KeyTiles<KT> keys(q0, min(q0 + QUERIES, len) - 1, a.window, a.sinks);
    fetch(keys.at(0), 0);
    FloatQuery<HD> q;
    q.load((const float*)a.q + (size_t)(s0 + min(w0 + n, len - 1)) * a.ld_q + (size_t)h * HD, c);
#pragma unroll
    for (int s = 0; s < D; ++s) asm volatile("" : "+v"(q.q[s]));
    f32x4_t o[D];
#pragma unroll
    for (int d = 0; d < D; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    constexpr float MOST = 20.f;
    float ref = -1e30f, l = 0.f;
    bool far = false;
    for (int j = 0; j < keys.n; ++j) {
        const int buf = j & 1, first = keys.at(j) * KT, last = first + KT - 1;
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        __syncthreads();                           // tile j is there, and nobody reads tile j - 1 any more
        if (j + 1 < keys.n) fetch(keys.at(j + 1), buf ^ 1);
        if (w0 >= len || first > w0 + 15 || (last <= w0 - a.window && first >= a.sinks)) continue;      // nothing that this wave sees
        f32x4_t s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D; ++i) float_scores(*(const f32x4_t*)&sK[buf][n * HD + (((4 * i + c) ^ n) << 2)], q.q[i], s);
        if (last > w0 || !(first > w0 + 15 - a.window || last < a.sinks)) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (!window_sees(a, w0 + n, first + 4 * c + r)) s[r] = -INFINITY;
        }
        const float top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(s[0], s[1]), __builtin_elementwise_maximum(s[2], s[3])) * unit;
        if (__any(top > ref + MOST)) {
            const float high = column_max(top), now = high > ref + MOST ? high : ref, keep = __builtin_amdgcn_exp2f(ref - now);
            far |= __any(now != ref && fabsf(now) > kFarthest);
            ref = now;
            l *= keep;
#pragma unroll
            for (int d = 0; d < D; ++d) o[d] *= keep;
        }
        f32x4_t p;
#pragma unroll
        for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], unit, -ref));
        l += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < HD / 64; ++d) float_sums(*(const f32x4_t*)&sV[buf][(4 * c + i) * HD + 64 * d + 4 * n], p[i], o + 4 * d);
    }
    const float inv = 1.f / column_sum(l);
    float odd = 0.f;
    if (w0 + n < len) {
        float* out = (float*)a.out + (size_t)(s0 + w0 + n) * a.ld_out + (size_t)h * HD;
        each_dims<HD>(o, c, [&](int d, f32x4_t x) {
            x *= inv;
            odd += 0.f * ((x[0] + x[1]) + (x[2] + x[3]));
            *(f32x4_t*)(out + d) = x;
        });
    }
    if (far || __any(odd != 0.f))
        for (int i = w0; i < min(w0 + 16, len); ++i) window_row<float, HD>(a, s0, i, h, lane);
}

// A pass in launches of fewer than 2^32 threads, 128 / QUERIES workgroups of THREADS a tile and query head.
template <int QUERIES, int THREADS, typename F>
static hipError_t window_launches(const WindowArgs& a, F start) {
    constexpr int PARTS = kFlashTile / QUERIES;
    const int each = PARTS * a.n_q_heads, most = (int)std::min<int64_t>((kLaunchThreads / THREADS - 8 * each) / each, 1 << 30);
    for (int first = 0; first < a.n_tiles; first += most) {
        WindowArgs p = a;
        p.tile_start += first;
        p.tile_q0 += first;
        p.tile_len += first;
        p.n_tiles = std::min(most, a.n_tiles - first);
        start(((unsigned)p.n_tiles * (unsigned)a.n_kv_heads + 7) / 8 * 8 * (unsigned)(a.n_q_heads / a.n_kv_heads) * PARTS, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int HD> static hipError_t window_float(hipStream_t st, const WindowArgs& a) {
    if (a.rows > 96ll * a.n_tiles)
        return window_launches<64, 256>(a, [&](unsigned grid, const WindowArgs& p) { k_window_float<HD, 4><<<grid, 256, 0, st>>>(p); });
    return window_launches<128, 512>(a, [&](unsigned grid, const WindowArgs& p) { k_window_float<HD, 8><<<grid, 512, 0, st>>>(p); });
}

template <typename T, int HD> static hipError_t window_typed(hipStream_t st, const WindowArgs& a) {
    if constexpr (sizeof(T) == 4) return window_float<HD>(st, a);
    else return window_launches<128, 256>(a, [&](unsigned grid, const WindowArgs& p) { k_window_flash<T, HD><<<grid, 256, 0, st>>>(p); });
}

template <typename T> static hipError_t window_dims(hipStream_t st, int head_dim, const WindowArgs& a) {
    return head_dim == 128 ? window_typed<T, 128>(st, a) : window_typed<T, 64>(st, a);
}

hipError_t launch_window_attention(hipStream_t st, int dtype, int head_dim, const WindowArgs& a) {
    return dtype == kBF16 ? window_dims<bf16_t>(st, head_dim, a) : dtype == kF16 ? window_dims<f16_t>(st, head_dim, a) : window_dims<float>(st, head_dim, a);
}

}  // namespace rlhf
