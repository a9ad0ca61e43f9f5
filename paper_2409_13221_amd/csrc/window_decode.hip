// Decode attention with a sliding window and sinks over the paged cache, of the activations' type or of 4 bits
// (include/rlhf_ops.h).
#include <algorithm>

#include "attn_tile.h"
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

// ---- a page's K and V of one KV head as operands of the matrix units (attn_tile.h); a column is a query head, those beyond a KV head's own
// repeat the last one.

// A page's K and V of one KV head as a buffer that ends behind them, or, of a page that is not there, at once: such loads give zeros and touch no
// memory.  Every byte is read once a step: evict-first.
struct PageBuffer {
    __amdgpu_buffer_rsrc_t r;
    __device__ __forceinline__ PageBuffer(const void* base, uint32_t size) : r(__builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)size, 0x00020000)) {}
    template <typename V> __device__ __forceinline__ V get(uint32_t lane, uint32_t at, uint32_t plane = 0) const {
        if constexpr (sizeof(V) == 16) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(r, (int)(lane + at), (int)plane, 2));
        else return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b64(r, (int)(lane + at), (int)plane, 2));
    }
};
template <typename T, int HD> __device__ __forceinline__ PageBuffer plain_page(const WindowDecodeArgs& a, int page, int kh, bool there, uint32_t& plane) {
    const T* p = (const T*)a.pool + (((size_t)page * a.n_layers + a.layer) * 2 * a.n_kv_heads + kh) * 16 * HD;
    plane = (uint32_t)a.n_kv_heads * (16 * HD * sizeof(T));
    return PageBuffer(p, there ? plane + 16 * HD * sizeof(T) : 0);
}

constexpr float NONE = 1e9f;            // no offset yet

// A 16-bit cache.  K as it lies: a lane has 8 dims of token n.  V: dims D n .. D n + D - 1 (D = HD / 16) of its four tokens, so that a row of V
// is read by 16 lanes side by side; pairs of tokens are put together by byte permutations.  Weights go in as two terms of the type, which
// leaves 2^-16 of them and less (their products are exact): the output's own rounding is what is seen.  Matrix units are idle here anyway.
template <typename T_, int HD_> struct Cache16 {
    using T = T_;
    using M = Matrix16<T>;
    static constexpr int HD = HD_, D = HD / 16, KS = HD / 32;
    static constexpr float TOP = M::TOP;
    typedef uint32_t VRow __attribute__((ext_vector_type(D / 2)));
    struct Query {
        u32x4_t q[KS];
        float unit = 1.f;
        __device__ __forceinline__ void load(const T* p, int c) {
#pragma unroll
            for (int s = 0; s < KS; ++s) q[s] = *(const u32x4_t*)(p + s * 32 + c * 8);
        }
    };
    struct Sums {
        f32x4_t acc[D];
        __device__ __forceinline__ void clear() {
#pragma unroll
            for (int d = 0; d < D; ++d) acc[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        __device__ __forceinline__ void scale(float f) {
#pragma unroll
            for (int d = 0; d < D; ++d) acc[d] *= f;
        }
        // Four dims at a time: put(dim, values).
        template <typename F> __device__ __forceinline__ void each(int c, F put) const { FloatTile<HD>::each(acc, c, put); }
        __device__ __forceinline__ void finish() {}
    };
    struct Tile {
        u32x4_t k[KS];
        VRow v[4];
        __device__ __forceinline__ void load(const WindowDecodeArgs& a, int page, int kh, bool there, int n, int c) {
            uint32_t plane;
            const PageBuffer b = plain_page<T, HD>(a, page, kh, there, plane);
#pragma unroll
            for (int s = 0; s < KS; ++s) k[s] = b.get<u32x4_t>((n * HD + c * 8) * 2, s * 64);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = b.get<VRow>((4 * c * HD + n * D) * 2, i * HD * 2, plane);
        }
        __device__ __forceinline__ f32x4_t scores(const Query& q) const {
            f32x4_t s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KS; ++i) s = M::qk(k[i], q.q[i], s);
            return s;
        }
        __device__ __forceinline__ void hide(int i) {
#pragma unroll
            for (int w = 0; w < D / 2; ++w) v[i][w] = 0;
        }
        __device__ __forceinline__ float spare() const { return -TOP; }
        __device__ __forceinline__ bool too_large(const f32x4_t&) const { return false; }
        __device__ __forceinline__ void add(const f32x4_t& p, const Query&, Sums& o) const {
            const u32x2_t hi{pack2<T>(p[0], p[1]), pack2<T>(p[2], p[3])};
            const u32x2_t lo{pack2<T>(p[0] - unpack<T>(hi[0], 0), p[1] - unpack<T>(hi[0], 1)), pack2<T>(p[2] - unpack<T>(hi[1], 0), p[3] - unpack<T>(hi[1], 1))};
#pragma unroll
            for (int w = 0; w < D / 2; ++w)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t sel = half ? 0x07060302u : 0x05040100u;
                    const u32x2_t x{__builtin_amdgcn_perm(v[1][w], v[0][w], sel), __builtin_amdgcn_perm(v[3][w], v[2][w], sel)};
                    o.acc[2 * w + half] = M::pv(x, lo, M::pv(x, hi, o.acc[2 * w + half]));
                }
        }
    };
};

template <int HD_> struct CacheFloat {
    using T = float;
    static constexpr int HD = HD_;
    using Query = FloatQuery<HD>;
    using Sums = typename Cache16<f16_t, HD>::Sums;
    struct Tile : FloatTile<HD> {
        __device__ __forceinline__ void load(const WindowDecodeArgs& a, int page, int kh, bool there, int n, int c) {
            uint32_t plane;
            const PageBuffer b = plain_page<float, HD>(a, page, kh, there, plane);
            constexpr int D = HD / 16;
#pragma unroll
            for (int s = 0; s < D; ++s) this->k[s] = b.get<f32x4_t>((n * HD + c * 4) * 4, s * 64);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int d = 0; d < D / 4; ++d) this->v[i][d] = b.get<f32x4_t>((4 * c * HD + n * D) * 4, (i * HD + d * 4) * 4, plane);
        }
        __device__ __forceinline__ void hide(int i) {
#pragma unroll
            for (int d = 0; d < HD / 64; ++d) this->v[i][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        __device__ __forceinline__ float spare() const { return 0.f; }
        __device__ __forceinline__ bool too_large(const f32x4_t&) const { return false; }
        __device__ __forceinline__ void add(const f32x4_t& p, const Query&, Sums& o) const { FloatTile<HD>::add(p, o.acc); }
    };
};

// A cache of 4 bits.  Codes become halves u = -8 .. 7 by putting their bits into the mantissa of 1024: 9 instructions for 8 of them.  With scale s and
// center c of each token and 64 dims (group g),
//   q.k = sum over g of s_g (sum q u) + c_g (sum of q in g),   o = sum over tokens of (p s_g) u + p c_g:
// the matrix units take q and p s_g, the rest is a few multiply-adds a token.  A query is scaled to have its greatest magnitude in [2^14, 2^15)
// and taken as halves, exact from half and bfloat16 down to 2^-39 of that; from float in three terms.  Weights p are scaled such that p s_g fits
// half (spare), in one term, of float calls two.
template <typename T_, int HD_> struct Cache4 {
    using T = T_;
    using L = Kv4<HD_>;
    static constexpr int HD = HD_, KS = HD / 32, GROUPS = L::GROUPS, TERMS = sizeof(T) == 4 ? 3 : 1;
    typedef uint32_t Codes __attribute__((ext_vector_type(KS)));
    // Eight codes of a word as halves, in the order 0 4 1 5 2 6 3 7.  `magic`, 1024 twice, comes in a vector register: with the mask in a scalar one,
    // and-or is one instruction.
    static __device__ __forceinline__ void halves(uint32_t x, uint32_t magic, uint32_t (&h)[4]) {
        typedef f16_t pair __attribute__((ext_vector_type(2)));
        const auto low = [magic](uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(pair, (w & 0x000F000Fu) | magic) - pair{1032, 1032}); };
        const auto high = [magic](uint32_t w) {
            const pair v = __builtin_bit_cast(pair, (w & 0x00F000F0u) | magic), f{0.0625, 0.0625}, o{-72, -72};
            return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(v, f, o));
        };
        h[0] = low(x);
        h[1] = high(x);
        h[2] = low(x >> 8);
        h[3] = high(x >> 8);
    }
    static __device__ __forceinline__ uint32_t magic() {
        uint32_t m = 0x64006400u;
        asm("" : "+v"(m));
        return m;
    }
    struct Query {
        u32x4_t q[KS][TERMS];
        float sum[GROUPS], unit;
        uint32_t magic;
        __device__ __forceinline__ void load(const T* p, int c) {
            magic = Cache4::magic();
            float f[KS][8], m = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                load8<T>(p + s * 32 + c * 8, f[s]);
#pragma unroll
                for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(f[s][e]));
            }
            m = column_max(m);
            const int up = m > 0.f && m < INFINITY ? min(100, 14 - ilogbf(m)) : 0;
            unit = ldexpf(1.f, -up);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                sum[g] = 0.f;
#pragma unroll
                for (int s = 2 * g; s < 2 * g + 2; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[g] += f[s][e] = ldexpf(f[s][e], up);
                sum[g] = column_sum(sum[g]);
            }
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int t = 0; t < TERMS; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t h = pack2<f16_t>(f[s][e], f[s][e + 4]);
                        q[s][t][e] = h;
                        f[s][e] -= unpack<f16_t>(h, 0);
                        f[s][e + 4] -= unpack<f16_t>(h, 1);
                    }
        }
    };
    struct Sums {
        f32x4_t acc[HD / 16];
        float center[GROUPS];
        __device__ __forceinline__ void clear() {
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) acc[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) center[g] = 0.f;
        }
        __device__ __forceinline__ void scale(float f) {
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) acc[d] *= f;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) center[g] *= f;
        }
        __device__ __forceinline__ void finish() {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) center[g] = column_sum(center[g]);
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) acc[d] += center[d / 4];
        }
        template <typename F> __device__ __forceinline__ void each(int c, F put) const {
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) put(16 * d + 4 * c, acc[d]);
        }
    };
    struct Tile {
        Codes k, v;
        u32x4_t kp[GROUPS], vp[GROUPS];            // (scale, center) of the lane's four tokens
        static __device__ __forceinline__ float scale_of(uint32_t w) { return unpack<f16_t>(w, 0); }
        static __device__ __forceinline__ float center_of(uint32_t w) { return unpack<f16_t>(w, 1); }
        __device__ __forceinline__ void load(const WindowDecodeArgs& a, int page, int kh, bool there, int n, int c) {
            const PageBuffer b((const uint8_t*)a.pool + (((size_t)page * a.n_layers + a.layer) * a.n_kv_heads + kh) * L::BLOCK, there ? L::BLOCK : 0);
            k = b.get<Codes>((16 * c + n) * L::PIECE, 0);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) kp[g] = b.get<u32x4_t>(16 * c, L::param(0, 64 * g));
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) vp[g] = b.get<u32x4_t>(16 * c, L::PARAMS + L::param(0, 64 * g));
            v = b.get<Codes>((16 * c + n) * L::PIECE, L::V_CODES);
        }
        __device__ __forceinline__ f32x4_t scores(const Query& q) const {
            const uint32_t m = q.magic;
            f32x4_t s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                f32x4_t raw{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 2 * g; i < 2 * g + 2; ++i) {
                    uint32_t h[4];
                    halves(k[i], m, h);
                    const u32x4_t x{h[0], h[1], h[2], h[3]};
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) raw = Matrix16<f16_t>::qk(x, q.q[i][t], raw);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) s[r] = fmaf(scale_of(kp[g][r]), raw[r], fmaf(center_of(kp[g][r]), q.sum[g], s[r]));
            }
            return s;
        }
        __device__ __forceinline__ void hide(int i) {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) vp[g][i] = 0;
        }
        // What to add to the reference (log2) for p s of at most 2^10 here.
        __device__ __forceinline__ float spare() const {
            float s = 0.f;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int r = 0; r < 4; ++r) s = fmaxf(s, fabsf(scale_of(vp[g][r])));
            s = wave_max(s);
            return s > 0.f ? (float)ilogbf(s) - 9.f : -14.f;
        }
        __device__ __forceinline__ float weight(const f32x4_t& p, int g, int r) const { return fmaf(p[r], scale_of(vp[g][r]), 0.f); }
        // Whether a p s leaves half: no more than one page in many has scales 2^5 times those that the reference was chosen for.
        __device__ __forceinline__ bool too_large(const f32x4_t& p) const {
            float s = 0.f;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int r = 0; r < 4; ++r) s = fmaxf(s, fabsf(weight(p, g, r)));
            return __any(s > 32768.f);
        }
        __device__ __forceinline__ void add(const f32x4_t& p, const Query& q, Sums& o) const {
            const uint32_t m = q.magic;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                float w[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    w[r] = weight(p, g, r);
                    o.center[g] = fmaf(p[r], center_of(vp[g][r]), o.center[g]);
                }
                const u32x2_t hi{pack2<f16_t>(w[0], w[2]), pack2<f16_t>(w[1], w[3])};
                u32x2_t lo{0, 0};
                if (TERMS > 1)
                    lo = u32x2_t{pack2<f16_t>(w[0] - unpack<f16_t>(hi[0], 0), w[2] - unpack<f16_t>(hi[0], 1)),
                                 pack2<f16_t>(w[1] - unpack<f16_t>(hi[1], 0), w[3] - unpack<f16_t>(hi[1], 1))};
#pragma unroll
                for (int i = 2 * g; i < 2 * g + 2; ++i) {
                    uint32_t h[4];
                    halves(v[i], m, h);                     // tokens (0, 2) of dims 32 i + n, of dims 32 i + 16 + n, then (1, 3) alike
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const u32x2_t x{h[e], h[2 + e]};
                        f32x4_t& acc = o.acc[2 * i + e];
                        acc = Matrix16<f16_t>::pv(x, hi, acc);
                        if (TERMS > 1) acc = Matrix16<f16_t>::pv(x, lo, acc);
                    }
                }
            }
        }
    };
};

// A workgroup takes a row, a KV head (up to 16 of its query heads) and a part of the row's visible pages; its waves take these in turn, a page in
// flight while one is worked on, and meet in LDS.  m: greatest score; weights are exp2(z - ref), ref = m + spare in log2.
template <typename C, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_window_decode(WindowDecodeArgs a) {
    using T = typename C::T;
    constexpr int HD = C::HD;
    extern __shared__ float lds[];                 // [WAVES][heads][HD] sums, then [WAVES][heads] references, [WAVES][heads] weights
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, c = lane >> 4;
    const int G = a.n_q_heads / a.n_kv_heads, blocks = (G + 15) / 16;
    unsigned b = blockIdx.x;
    const int split = b % a.nsplit;
    b /= a.nsplit;
    const int hb = b % blocks;
    b /= blocks;
    const int kh = b % a.n_kv_heads, r = b / a.n_kv_heads, h0 = kh * G + hb * 16, heads = min(16, G - hb * 16), room = min(16, G);
    const int* table = nullptr;
    const int ctx = row_context(a, r, table);
    float m = -INFINITY, l = 0.f, ref = -INFINITY, off = NONE;
    typename C::Sums o;
    o.clear();
    bool lost = ctx < 0;
    if (ctx > 0) {
        typename C::Query q;
        q.load((const T*)a.q + (size_t)r * a.ld_q + (size_t)(h0 + min(n, heads - 1)) * HD, c);
        const float unit = q.unit * (1.44269504088896f * rsqrtf((float)HD));
        const Visible see(ctx, a.window, a.sinks);
        const int from = (int)((int64_t)see.n_pages * split / a.nsplit), to = (int)((int64_t)see.n_pages * (split + 1) / a.nsplit);
        const int mine = to - from > wave ? (to - from - wave + WAVES - 1) / WAVES : 0;
        const auto index = [&](int j) { return see.page(from + wave + j * WAVES); };
        const auto page = [&](int j) { return table[index(min(j, mine - 1))]; };
        const auto fetch = [&](typename C::Tile& t, int id, bool more) {
            const bool inside = (unsigned)id < (unsigned)a.n_pages;
            lost |= !inside;
            t.load(a, inside ? id : 0, kh, inside && more, n, c);
        };
        const auto step = [&](typename C::Tile& t, int j) {
            f32x4_t s = t.scores(q);
            const int first = index(j) * 16;
            if (first + 15 >= ctx || !(first >= see.lo || first + 15 < see.sinks)) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!see.sees(first + 4 * c + i)) {
                        s[i] = -INFINITY;
                        t.hide(i);
                    }
            }
            const float mn = fmaxf(m, column_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))));
            if (off == NONE) off = t.spare();
            f32x4_t p;
#pragma unroll 1
            for (int again = 0; again < 2; ++again) {              // twice where the offset is chosen anew
                const float rn = mn == -INFINITY ? 0.f : fmaf(mn, unit, off);
                if (__any(!(rn == ref))) {
                    const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref - rn);
                    l *= keep;
                    o.scale(keep);
                    ref = rn;
                }
                m = mn;
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[i], unit, -rn));
                if (!t.too_large(p)) break;
                off = t.spare();
            }
            l += (p[0] + p[1]) + (p[2] + p[3]);
            t.add(p, q, o);
        };
        // Two pages in flight, their numbers one step ahead.  Loads behind the last page are issued too, of nothing: so every wait in the loop is for a known
        // number of loads.
        if (mine > 0) {
            typename C::Tile t0, t1;
            int id0 = page(0), id1 = page(1);
            fetch(t0, id0, true);
            for (int j = 0; j < mine; j += 2) {
                fetch(t1, id1, j + 1 < mine);
                id0 = page(j + 2);
                id1 = page(j + 3);
                step(t0, j);
                fetch(t0, id0, j + 2 < mine);
                if (j + 1 < mine) step(t1, j + 1);
            }
        }
    }
    if (lost) l = NAN;
    l = column_sum(l);
    o.finish();
    if (m == -INFINITY) ref = -INFINITY;           // nothing seen, or scores of -inf alone
    float* s_ref = lds + WAVES * room * HD;
    float* s_l = s_ref + WAVES * room;
    if (n < heads) {
        o.each(c, [&](int d, f32x4_t x) { *(f32x4_t*)(lds + (wave * room + n) * HD + d) = x; });
        if (c == 0) {
            s_ref[wave * room + n] = ref;
            s_l[wave * room + n] = l;
        }
    }
    __syncthreads();
    const size_t slots = (size_t)a.rows * a.n_q_heads * a.nsplit;
    for (int i = threadIdx.x; i < heads * (HD / 4); i += WAVES * 64) {
        const int h = i / (HD / 4), d = i % (HD / 4) * 4;
        float top = -INFINITY, sum = 0.f;
        f32x4_t x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, s_ref[w * room + h]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(s_ref[w * room + h] - top);
            sum += f * s_l[w * room + h];
            x += f * *(const f32x4_t*)(lds + (w * room + h) * HD + d);
        }
        if (a.nsplit == 1) {
            T* out = (T*)a.out + (size_t)r * a.ld_out + (size_t)(h0 + h) * HD + d;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = round_to<T>(ctx == 0 ? 0.f : x[e] / sum);
        } else {
            const size_t slot = ((size_t)r * a.n_q_heads + h0 + h) * a.nsplit + split;
            if (d == 0) { a.part[2 * slot] = top; a.part[2 * slot + 1] = sum; }
            *(f32x4_t*)(a.part + 2 * slots + slot * HD + d) = x;
        }
    }
}

// The parts of a (row, query head) joined: a wave each, or of many parts four, whose sums meet in LDS.
template <typename T, int HD, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_window_join(WindowDecodeArgs a) {
    constexpr int LANES = HD / 4, GROUPS = WAVES * 64 / LANES;         // a group of lanes takes every GROUPS-th part, four dims a lane
    __shared__ f32x4_t s_x[GROUPS][LANES];
    __shared__ float s_w[64], s_l;
    const int t = threadIdx.x, g = t / LANES, d = t % LANES * 4, h = blockIdx.x % a.n_q_heads, r = blockIdx.x / a.n_q_heads;
    const size_t slot = (size_t)blockIdx.x * a.nsplit, slots = (size_t)a.rows * a.n_q_heads * a.nsplit;
    if (t < 64) {                                                      // nsplit <= 64
        const float2 ml = t < a.nsplit ? ((const float2*)a.part)[slot + t] : make_float2(-INFINITY, 0.f);
        const float m = wave_max(ml.x), w = __builtin_amdgcn_exp2f(ml.x - (m == -INFINITY ? 0.f : m)), l = wave_sum(w * ml.y);
        s_w[t] = w;
        if (t == 0) s_l = l;
    }
    __syncthreads();
    f32x4_t x{0.f, 0.f, 0.f, 0.f};
    for (int s = g; s < a.nsplit; s += GROUPS) x += s_w[s] * *(const f32x4_t*)(a.part + 2 * slots + (slot + s) * HD + d);
    s_x[g][d / 4] = x;
    __syncthreads();
    if (t >= LANES) return;
    for (int i = 1; i < GROUPS; ++i) x += s_x[i][t];
    const bool empty = a.ctx_len[r] <= 0;
    T* o = (T*)a.out + (size_t)r * a.ld_out + (size_t)h * HD + d;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = round_to<T>(empty ? 0.f : x[e] / s_l);
}

// Waves of a workgroup; four where 16 heads' sums of eight would take more than 64 KB of LDS.
static int decode_waves(int group) { return group > 8 ? 4 : 8; }

int window_decode_nsplit(int rows, int n_q_heads, int n_kv_heads, int max_ctx, int window, int sinks) {
    const int64_t pages = std::min<int64_t>((max_ctx + 15ll) / 16, (sinks + 15ll) / 16 + (window + 15ll) / 16 + 1);
    const int group = n_q_heads / n_kv_heads, waves = decode_waves(group);
    const int64_t blocks = (int64_t)rows * n_kv_heads * ((group + 15) / 16);
    return (int)std::max<int64_t>(1, std::min<int64_t>({64, pages / (2 * waves), 4096 / waves / blocks}));
}

size_t window_decode_scratch_floats(int rows, int n_q_heads, int head_dim, int nsplit) {
    return (size_t)rows * n_q_heads * nsplit * (head_dim + 2);
}

template <typename C>
static hipError_t decode_rows(hipStream_t st, const WindowDecodeArgs& a) {
    using T = typename C::T;
    const int group = a.n_q_heads / a.n_kv_heads, waves = decode_waves(group);
    const int64_t blocks = (int64_t)a.n_kv_heads * ((group + 15) / 16) * a.nsplit;
    const int most = (int)std::min<int64_t>(kLaunchThreads / (64 * waves) / std::max<int64_t>(blocks, a.n_q_heads), 1 << 24);
    const size_t lds = (size_t)waves * std::min(16, group) * (C::HD + 2) * sizeof(float);
    for (int first = 0; first < a.rows; first += most) {
        WindowDecodeArgs p = a;
        p.q = (const T*)a.q + (size_t)first * a.ld_q;
        p.out = (T*)a.out + (size_t)first * a.ld_out;
        p.row_sample += first;
        p.ctx_len += first;
        p.rows = std::min(most, a.rows - first);
        const unsigned grid = (unsigned)(p.rows * blocks);
        if (waves == 8) k_window_decode<C, 8><<<grid, 512, lds, st>>>(p);
        else k_window_decode<C, 4><<<grid, 256, lds, st>>>(p);
        const unsigned heads = (unsigned)p.rows * (unsigned)a.n_q_heads;
        if (a.nsplit > 8) k_window_join<T, C::HD, 4><<<heads, 256, 0, st>>>(p);
        else if (a.nsplit > 1) k_window_join<T, C::HD, 1><<<heads, 64, 0, st>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_window_decode(hipStream_t st, int dtype, bool four_bits, int head_dim, const WindowDecodeArgs& a) {
#define RLHF_DECODE(HD)                                                                                           \
    if (head_dim == HD) {                                                                                         \
        if (dtype == kBF16) return four_bits ? decode_rows<Cache4<bf16_t, HD>>(st, a) : decode_rows<Cache16<bf16_t, HD>>(st, a); \
        if (dtype == kF16) return four_bits ? decode_rows<Cache4<f16_t, HD>>(st, a) : decode_rows<Cache16<f16_t, HD>>(st, a);    \
        return four_bits ? decode_rows<Cache4<float, HD>>(st, a) : decode_rows<CacheFloat<HD>>(st, a);            \
    }
    RLHF_DECODE(64)
    RLHF_DECODE(128)
#undef RLHF_DECODE
    return hipErrorInvalidValue;
}

}  // namespace rlhf
