// Packed causal attention with a sliding window and sinks (the formulas are in include/rlhf_ops.h).
#include <algorithm>
#include <type_traits>

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
// flight before it reads LDS; whoever reads waits for vmcnt and the workgroup first.  (It has no register to come back to.  m0 is
// reserved: the compiler keeps nothing in it, warns of it as a clobber, and makes no other use of it in these kernels.)
__device__ __forceinline__ void load_to_lds(u32x4_t base, uint32_t lane, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(lane), "s"(base), "s"(offset) : "memory");
}
__device__ __forceinline__ u32x4_t buffer_base(const void* p) {
    return u32x4_t{(uint32_t)(uintptr_t)p, (uint32_t)((uintptr_t)p >> 32) & 0xFFFFu, 0xFFFFFFFFu, 0x00020000u};
}
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_t;

// References beyond this (log2) are off by more than a factor of 2 from the score that they were taken from, and weights then leave the range of
// their type: such queries are taken again, each by itself.
constexpr float kFarthest = 0x1p24f;
// (An infinite one makes the result no number, which it is.)
__device__ __forceinline__ bool too_far(float ref) { return fabsf(ref) > kFarthest && ref < INFINITY; }
// A sum of weights that says nothing: scores of -infinity or below the first reference alone.  One that is no number comes from a score that is none.
__device__ __forceinline__ bool no_weight(float sum) { return sum == 0.f || sum == INFINITY; }
// Whether any of the four lanes that hold a column says so.
__device__ __forceinline__ bool column_any(bool x, int n) {
    uint64_t b = __ballot(x);
    b |= b >> 32;
    b |= b >> 16;
    return b >> n & 1;
}

// A key that is hidden from a query has weight 0, and 0 times what is not a number is none.  So a wave with a result that is not finite takes its tiles again,
// with values as they are needed: one pass each for the dims in which a query sees an infinity or what is no number, and one over the finite
// values, whose sums are, to the bit, what they would be if what a query does not see were not there.  (16384 tokens of 64 / 8 heads, window 4096: 1.86 ms, with
// one value of V that is no number 7.4, one that all see 21; query by query it was 78 and 239.)
enum class Take { FINITE, RISING, FALLING };         // values that are finite, else 0; 1 for +infinity or no number, else 0; for -infinity
template <Take W> __device__ __forceinline__ float take(float x) {
    if constexpr (W == Take::FINITE) return fabsf(x) < INFINITY ? x : 0.f;
    else return x != x || x == (W == Take::RISING ? INFINITY : -INFINITY) ? 1.f : 0.f;
}
// A value with bit `bit` of what was found: of infinities of both signs, or none, no number.
__device__ __forceinline__ float with_found(float x, uint32_t rising, uint32_t falling, int bit) {
    const bool up = rising >> bit & 1, down = falling >> bit & 1;
    return up ? (down ? NAN : INFINITY) : down ? -INFINITY : x;
}

// Queries of a head that a wave of the 16-bit kernel holds, columns n + 16 m, and what has been summed up for them.
template <typename T, int HD, int MQ> struct FlashQueries {
    using M = Matrix16<T>;
    static constexpr int KT = 32, NF = KT / 16, NU = KT / 32, KS = HD / 32, DF = HD / 16;
    static constexpr float START = M::TOP > 0.f ? 6.f : 0.f, MOST = M::TOP > 0.f ? M::TOP : 20.f;      // log2 of the greatest weight at a new reference, and ever
    static constexpr uint32_t ONE = M::ONES & 0xFFFFu;
    u32x4_t q[MQ][KS];
    f32x4_t o[DF][MQ], l[MQ];                      // l: sums of the weights, in every row of the product
    float ref[MQ];
    bool far[MQ];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int m = 0; m < MQ; ++m) {
#pragma unroll
            for (int d = 0; d < DF; ++d) o[d][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            l[m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            ref[m] = -1e30f;
            far[m] = false;
        }
    }
    // o += V^T p: value(d, u) gives 8 keys of a lane's row of sums d, 32 u + 4c .. + 3 and 16 further.
    template <typename F> __device__ __forceinline__ void sum(const u32x4_t (&p)[MQ][NU], F value) {
#pragma unroll
        for (int d = 0; d < DF; ++d)
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const u32x4_t x = value(d, u);
#pragma unroll
                for (int m = 0; m < MQ; ++m) o[d][m] = M::qk(x, p[m][u], o[d][m]);
            }
    }
    // The keys from `first` on: key(k, f) gives dims 32 k + 8 c .. + 7 of key 16 f + n.
    template <typename K, typename V> __device__ __forceinline__ void tile(const WindowArgs& a, int w0, int first, int n, int c, K key, V value) {
        constexpr float unit = kScoreUnit<HD>;
        const int last = first + KT - 1;
        f32x4_t s[NF][MQ];
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int m = 0; m < MQ; ++m) s[f][m] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                const u32x4_t x = key(k, f);
#pragma unroll
                for (int m = 0; m < MQ; ++m) s[f][m] = M::qk(x, q[m][k], s[f][m]);
            }
        if (last > w0 || !(first > w0 + 16 * MQ - 1 - a.window || last < a.sinks)) {
#pragma unroll
            for (int m = 0; m < MQ; ++m)
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!window_sees(a, w0 + m * 16 + n, first + f * 16 + 4 * c + r)) s[f][m][r] = -INFINITY;
        }
        float top[MQ];
        bool high = false;
#pragma unroll
        for (int m = 0; m < MQ; ++m) {
            float x = s[0][m][0];
#pragma unroll
            for (int e = 1; e < 4 * NF; ++e) x = __builtin_elementwise_maximum(x, s[e / 4][m][e % 4]);         // one instruction for two; a score that is no number shows in the result
            top[m] = x * unit;
            high |= top[m] > ref[m] + MOST;
        }
        if (__any(high)) {
#pragma unroll
            for (int m = 0; m < MQ; ++m) {
                const float most = column_max(top[m]), now = most > ref[m] + MOST ? most - START : ref[m], keep = __builtin_amdgcn_exp2f(ref[m] - now);
                far[m] |= now != ref[m] && too_far(now);
                ref[m] = now;
                l[m] *= keep;
#pragma unroll
                for (int d = 0; d < DF; ++d) o[d][m] *= keep;
            }
        }
        u32x4_t p[MQ][NU];
#pragma unroll
        for (int m = 0; m < MQ; ++m)
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
            for (int m = 0; m < MQ; ++m) l[m] = M::qk(u32x4_t{M::ONES, M::ONES, M::ONES, M::ONES}, p[m][u], l[m]);
        sum(p, value);
    }
    __device__ __forceinline__ static bool blind(const WindowArgs& a, int w0, int len, int first) {        // nothing that this wave sees
        return w0 >= len || first > w0 + 16 * MQ - 1 || (first + KT - 1 <= w0 - a.window && first >= a.sinks);
    }

    __device__ __forceinline__ void store(T* out, int m) const {
#pragma unroll
        for (int d = 0; d < DF; d += 2) {
            const f32x4_t x = o[d][m], y = o[d + 1][m];
            *(u32x4_t*)(out + d * 16) = u32x4_t{pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3])};
        }
    }
    // Sums over weights.  True where an output of the query is not finite.
    __device__ __forceinline__ bool divide(int m, int n) {
        const float inv = 1.f / l[m][0];
        float odd = 0.f;
#pragma unroll
        for (int d = 0; d < DF; ++d) {
            o[d][m] *= inv;
            odd += 0.f * ((o[d][m][0] + o[d][m][1]) + (o[d][m][2] + o[d][m][3]));
        }
        return column_any(odd != 0.f, n);
    }
};

// The lost ones of 16 queries of a wave over again, straight from memory; those that are not finite even so come back as alone.
template <typename T, int HD>
__device__ __forceinline__ void flash_again(const WindowArgs& a, const T* q, const KeyTiles<32>& keys, const T* kb, const T* vb, T* out, int w0, int len,
                                            bool lost, bool& alone, int n, int c) {
    using Q = FlashQueries<T, HD, 1>;
    const auto each_tile = [&](auto work) {
        for (int j = 0; j < keys.n; ++j)
            if (const int first = keys.at(j) * Q::KT; !Q::blind(a, w0, len, first)) work(first);
    };
    const auto row = [&](int key) { return (size_t)min(key, len - 1); };
    const auto values = [&](int first, auto what) {
        return [&a, &row, vb, first, n, c](int d, int u) {
            const T* v = vb + (d / 2 * 32 + (n >> 2) * 8 + (d & 1) * 4 + (n & 3));
            u32x4_t x;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int key = first + u * 32 + e / 2 * 16 + 4 * c + e % 2 * 2;
                x[e] = pack2<T>(take<decltype(what)::value>(to_f32<T>(v[row(key) * a.ld_v])), take<decltype(what)::value>(to_f32<T>(v[row(key + 1) * a.ld_v])));
            }
            asm volatile("" : "+v"(x) : : "memory");                   // loads of a step at a time, not of all: registers
            return x;
        };
    };
    const auto count = [&](auto what) {
        Q w;
        w.clear();
        each_tile([&](int first) {
            u32x4_t p[1][Q::NU];                   // 1 for what a query sees
#pragma unroll
            for (int e = 0; e < 4 * Q::NU; ++e) {
                const int key = first + e / 2 * 16 + 4 * c + e % 2 * 2;
                p[0][e / 4][e % 4] = (window_sees(a, w0 + n, key) ? Q::ONE : 0) | (window_sees(a, w0 + n, key + 1) ? Q::ONE << 16 : 0);
            }
            w.sum(p, values(first, what));
        });
        uint32_t bits = 0;
#pragma unroll
        for (int e = 0; e < 4 * Q::DF; ++e) bits |= w.o[e / 4][0][e % 4] > 0.f ? 1u << e : 0u;
        asm volatile("" : "+v"(bits));               // one register, not the sums that it was taken from
        return bits;
    };
    const uint32_t rising = count(std::integral_constant<Take, Take::RISING>()), falling = count(std::integral_constant<Take, Take::FALLING>());
    Q w;
#pragma unroll
    for (int s = 0; s < Q::KS; ++s) w.q[0][s] = *(const u32x4_t*)(q + s * 32);
    w.clear();
    each_tile([&](int first) {
        w.tile(a, w0, first, n, c, [&](int k, int f) { return *(const u32x4_t*)(kb + row(first + f * 16 + n) * a.ld_k + k * 32 + c * 8); },
               values(first, std::integral_constant<Take, Take::FINITE>()));
    });
    const bool odd = w.divide(0, n);
    alone |= lost && odd;
#pragma unroll
    for (int e = 0; e < 4 * Q::DF; ++e) w.o[e / 4][0][e % 4] = with_found(w.o[e / 4][0][e % 4], rising, falling, e);
    if (lost && !odd) w.store(out, 0);
}

// Queries first + b of the bits b that the 16 lanes c = 0 give.
template <typename T, int HD> __device__ __forceinline__ void take_alone(const WindowArgs& a, int s0, int first, int h, bool alone, int lane) {
    for (uint32_t left = (uint32_t)__ballot(alone) & 0xFFFFu; left; left &= left - 1) window_row<T, HD>(a, s0, first + __builtin_ctz(left), h, lane);
}

// 16-bit types: 128 queries of a head a workgroup, 32 a wave, against 32 keys at a time.  K and V go from memory to LDS directly, one tile ahead;
// V is transposed as it is read from LDS, and the weights stay in the lanes that made them.  References of the weights follow the running maximum only
// where these would leave their range, so that most tiles do not rescale the sums.  What a query's outputs are, to the bit, goes by what it sees alone.
// 32 keys leave registers for three workgroups a compute unit, 64 for two (64 instead: 16384 tokens 1808 -> 1871 us, 16 sequences of 200-800 85 -> 90; heads
// of 64 gain with long contexts, 4 x 4096 162 -> 150, and lose with short ones, 40 of 1-700 30.5 -> 31.6).
// 16384 tokens of 64 / 8 heads of 128, window 4096: 1.79 to 1.87 ms by card, 1.03 to 1.08 PFLOP/s of visible keys, the chip at its power limit (1.6 to 1.9 GHz).
// 16 sequences of 200-800, window 256: 72 to 82 us by what the caches hold, 3.2 TB/s and more where a copy reaches 4.7.
// Weights go to the matrix units rounded once to the type, of which an output is off by up to half a step of the values' spread (two terms would cost as
// many products again); what it is divided by is the sum of the rounded weights, by the matrix units too, so that equal values come out as they are
// (1 % slower than a sum of the weights as they were; heads of 64 3 to 5 %).
template <typename T, int HD>
__global__ __launch_bounds__(256, 3) void k_window_flash(WindowArgs a) {
    using Q = FlashQueries<T, HD, 2>;
    constexpr int KT = Q::KT, KS = Q::KS, CH = HD / 8, ROWS = 64 / CH, LOADS = KT / (4 * ROWS), TILE = KT * HD;
    __shared__ __attribute__((aligned(16))) T sK[2][TILE], sV[2][TILE];
    int tile, part, h, s0, q0, len;
    if (!window_work<kFlashTile>(a, tile, part, h) || !tile_of(a, tile, part, s0, q0, len)) return;
    const int kh = h / (a.n_q_heads / a.n_kv_heads);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, c = lane >> 4;
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
    const auto query = [&](int m) { return (const T*)a.q + (size_t)(s0 + min(w0 + m * 16 + n, len - 1)) * a.ld_q + (size_t)h * HD + c * 8; };
    const auto output = [&](int m) { return (T*)a.out + (size_t)(s0 + min(w0 + m * 16 + n, len - 1)) * a.ld_out + (size_t)h * HD + c * 8; };
    Q w;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const T* p = query(m);
#pragma unroll
        for (int s = 0; s < KS; ++s) w.q[m][s] = *(const u32x4_t*)(p + s * 32);
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(w.q[0][s]), "+v"(w.q[1][s]));          // here, not in the loop, where a wait for them would be one for K and V
    w.clear();
    // Token (modulo 16) of a lane's reads of V.  Sums d and d + 1 (even d) of a lane are dims 16 d + 8 c .. + 7, so that it stores 16 bytes at a time (16
    // sequences of 200-800, 32 heads of 128, window 1: 62.6 -> 58.4 us, 4.5 TB/s).
    const int vt = 4 * c + (n >> 2);
    const int vswap = (CH == 16 ? vt & 3 : (vt >> 1) & 1) << 2;

    if (keys.n > 1) fetch(keys.at(1), 1);
    for (int j = 0; j < keys.n; ++j) {
        const int buf = j & 1, first = keys.at(j) * KT;
        if (j == 0 && keys.n > 1) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        __syncthreads();                           // tile j is there, and nobody reads tile j - 1 any more
        if (j > 0 && j + 1 < keys.n) fetch(keys.at(j + 1), buf ^ 1);
        if (Q::blind(a, w0, len, first)) continue;
        w.tile(a, w0, first, n, c,
               [&](int k, int f) {
                   const int row = f * 16 + n, p = CH == 16 ? (k * 4 + c) ^ n : (k * 4 + c) ^ ((n >> 1) & 7);
                   return *(const u32x4_t*)&sK[buf][row * HD + p * 8];
               },
               [&](int d, int u) {
                   T* at = &sV[buf][(u * 32 + vt) * HD + ((d / 2 * 4 + (n & 3)) ^ vswap) * 8 + (d & 1) * 4];
                   const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(at + 16 * HD));
                   const u32x2_t x = __builtin_bit_cast(u32x2_t, lo), y = __builtin_bit_cast(u32x2_t, hi);
                   return u32x4_t{x[0], x[1], y[0], y[1]};
               });
    }

    bool lost[2], alone[2];                        // of a lane's queries
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const int i = w0 + m * 16 + n;
        const float sum = w.l[m][0];
        const bool odd = w.divide(m, n);
        alone[m] = i < len && (w.far[m] || no_weight(sum));
        lost[m] = i < len && !alone[m] && odd && sum == sum;
        if (i < len && !alone[m] && !lost[m]) w.store(output(m), m);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        if (__any(lost[m])) flash_again<T, HD>(a, query(m), keys, kb, vb, output(m), w0 + m * 16, len, lost[m], alone[m], n, c);
        take_alone<T, HD>(a, s0, w0 + m * 16, h, alone[m], lane);
    }
}

// What a wave of the float kernel holds: 16 queries of a head.
template <int HD> struct FloatQueries {
    static constexpr int KT = 16, D = HD / 16;
    static constexpr float MOST = 20.f;
    FloatQuery<HD> q;
    f32x4_t o[D];
    float l, ref;                                  // l: a lane's part of the sum of the weights
    bool far;

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int d = 0; d < D; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        l = 0.f;
        ref = -1e30f;
        far = false;
    }
    // value(i, d) gives dims 64 d + 4n .. + 3 of key 4c + i.
    template <typename F> __device__ __forceinline__ void sum(const f32x4_t& p, F value) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int d = 0; d < HD / 64; ++d) float_sums(value(i, d), p[i], o + 4 * d);
    }
    // key(i) gives dims 16 i + 4c .. + 3 of key n.
    template <typename K, typename V> __device__ __forceinline__ void tile(const WindowArgs& a, int w0, int first, int n, int c, K key, V value) {
        constexpr float unit = kScoreUnit<HD>;
        const int last = first + KT - 1;
        f32x4_t s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D; ++i) float_scores(key(i), q.q[i], s);
        if (last > w0 || !(first > w0 + 15 - a.window || last < a.sinks)) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (!window_sees(a, w0 + n, first + 4 * c + r)) s[r] = -INFINITY;
        }
        const float top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(s[0], s[1]), __builtin_elementwise_maximum(s[2], s[3])) * unit;
        if (__any(top > ref + MOST)) {
            const float high = column_max(top), now = high > ref + MOST ? high : ref, keep = __builtin_amdgcn_exp2f(ref - now);
            far |= now != ref && too_far(now);
            ref = now;
            l *= keep;
#pragma unroll
            for (int d = 0; d < D; ++d) o[d] *= keep;
        }
        f32x4_t p;
#pragma unroll
        for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], unit, -ref));
        l += (p[0] + p[1]) + (p[2] + p[3]);
        sum(p, value);
    }
    __device__ __forceinline__ static bool blind(const WindowArgs& a, int w0, int len, int first) {
        return w0 >= len || first > w0 + 15 || (first + KT - 1 <= w0 - a.window && first >= a.sinks);
    }
    __device__ __forceinline__ bool divide(float whole, int n) {
        const float inv = 1.f / whole;
        float odd = 0.f;
#pragma unroll
        for (int d = 0; d < D; ++d) {
            o[d] *= inv;
            odd += 0.f * ((o[d][0] + o[d][1]) + (o[d][2] + o[d][3]));
        }
        return column_any(odd != 0.f, n);
    }
    __device__ __forceinline__ void store(float* out, int c) const {
        each_dims<HD>(o, c, [&](int d, f32x4_t x) { *(f32x4_t*)(out + d) = x; });
    }
};

template <int HD>
__device__ __forceinline__ void float_again(const WindowArgs& a, const float* q, const KeyTiles<16>& keys, const float* kb, const float* vb, float* out, int w0, int len,
                            bool lost, bool& alone, int n, int c) {
    using Q = FloatQueries<HD>;
    const auto each_tile = [&](auto work) {
        for (int j = 0; j < keys.n; ++j)
            if (const int first = keys.at(j) * Q::KT; !Q::blind(a, w0, len, first)) work(first);
    };
    const auto row = [&](int key) { return (size_t)min(key, len - 1); };
    const auto values = [&](int first, auto what) {
        return [&a, &row, vb, first, n, c](int i, int d) {
            f32x4_t x = *(const f32x4_t*)(vb + row(first + 4 * c + i) * a.ld_v + 64 * d + 4 * n);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = take<decltype(what)::value>(x[e]);
            asm volatile("" : "+v"(x) : : "memory");                   // as above
            return x;
        };
    };
    const auto count = [&](auto what) {
        Q w;
        w.clear();
        each_tile([&](int first) {
            f32x4_t p;
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = window_sees(a, w0 + n, first + 4 * c + r) ? 1.f : 0.f;
            w.sum(p, values(first, what));
        });
        uint32_t bits = 0;
#pragma unroll
        for (int e = 0; e < 4 * Q::D; ++e) bits |= w.o[e / 4][e % 4] > 0.f ? 1u << e : 0u;
        asm volatile("" : "+v"(bits));               // one register, not the sums that it was taken from
        return bits;
    };
    const uint32_t rising = count(std::integral_constant<Take, Take::RISING>()), falling = count(std::integral_constant<Take, Take::FALLING>());
    Q w;
    w.q.load(q, c);
    w.clear();
    each_tile([&](int first) {
        w.tile(a, w0, first, n, c, [&](int i) {
                   f32x4_t x = *(const f32x4_t*)(kb + row(first + n) * a.ld_k + 16 * i + 4 * c);
                   asm volatile("" : "+v"(x) : : "memory");
                   return x;
               },
               values(first, std::integral_constant<Take, Take::FINITE>()));
    });
    const bool odd = w.divide(column_sum(w.l), n);
    alone |= lost && odd;
#pragma unroll
    for (int e = 0; e < 4 * Q::D; ++e) w.o[e / 4][e % 4] = with_found(w.o[e / 4][e % 4], rising, falling, e);
    if (lost && !odd) w.store(out, c);
}

// Float: 128 or 64 queries of a head a workgroup, 16 a wave, against 16 keys at a time, which go to LDS a tile ahead; bound by the float matrix rate (a tenth
// of the half one) where tiles are full.  8192 tokens of 64 / 8 heads of 128, window 1024: 2.11 ms, 123 TFLOP/s with the hidden part of
// the tiles (waves that read keys from memory for themselves: 3.29); 16 sequences of 200-800, 32 heads, window 256: 287 us, 88 TFLOP/s (456).
// Four waves where tiles are mostly full: twice as many workgroups, nearer to each other in length (2 x 767, 8 heads of 128: 106 us with eight, 71 with
// four; 2000 tokens of 32 heads 363, 316; 4 x 4096, 12 of 64, window 1024 457, 409; two instead of four: 104, 404, 433); of short sequences the
// second half would be empty (256 of 20-60, 32 heads of 128 165, 228; 32 of 100, 40 of 64 42.6, 44.7).
template <int HD, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 4) void k_window_float(WindowArgs a) {
    using Q = FloatQueries<HD>;
    constexpr int KT = Q::KT, CH = HD / 4, ROWS = 64 / CH, EACH = KT / ROWS, LOADS = 2 * EACH / WAVES, TILE = KT * HD, QUERIES = 16 * WAVES;
    __shared__ __attribute__((aligned(16))) float sK[2][TILE], sV[2][TILE];
    int tile, part, h, s0, q0, len;
    if (!window_work<QUERIES>(a, tile, part, h) || !tile_of(a, tile, part, s0, q0, len)) return;
    const int kh = h / (a.n_q_heads / a.n_kv_heads);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, c = lane >> 4;
    const int w0 = q0 + wave * 16;
    const float* kb = (const float*)a.k + (size_t)s0 * a.ld_k + (size_t)kh * HD;
    const float* vb = (const float*)a.v + (size_t)s0 * a.ld_v + (size_t)kh * HD;
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
    Q w;
    const auto query = [&]() { return (const float*)a.q + (size_t)(s0 + min(w0 + n, len - 1)) * a.ld_q + (size_t)h * HD; };
    w.q.load(query(), c);
#pragma unroll
    for (int s = 0; s < Q::D; ++s) asm volatile("" : "+v"(w.q.q[s]));
    w.clear();
    for (int j = 0; j < keys.n; ++j) {
        const int buf = j & 1, first = keys.at(j) * KT;
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        __syncthreads();                           // tile j is there, and nobody reads tile j - 1 any more
        if (j + 1 < keys.n) fetch(keys.at(j + 1), buf ^ 1);
        if (Q::blind(a, w0, len, first)) continue;
        w.tile(a, w0, first, n, c, [&](int i) { return *(const f32x4_t*)&sK[buf][n * HD + (((4 * i + c) ^ n) << 2)]; },
               [&](int i, int d) { return *(const f32x4_t*)&sV[buf][(4 * c + i) * HD + 64 * d + 4 * n]; });
    }
    const float sum = column_sum(w.l);
    const bool odd = w.divide(sum, n), mine = w0 + n < len;
    bool alone = mine && (w.far || no_weight(sum));
    const bool lost = mine && !alone && odd && sum == sum;
    float* out = (float*)a.out + (size_t)(s0 + min(w0 + n, len - 1)) * a.ld_out + (size_t)h * HD;
    if (mine && !alone && !lost) w.store(out, c);
    if (__any(lost)) float_again<HD>(a, query(), keys, kb, vb, out, w0, len, lost, alone, n, c);
    take_alone<float, HD>(a, s0, w0, h, alone, lane);
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
