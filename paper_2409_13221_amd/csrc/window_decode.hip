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

// A workgroup's row, KV head, up to 16 of its query heads from h0 on (of `room` in LDS), and part of the row's visible pages.
struct DecodeWork {
    int split, r, kh, h0, heads, room;
    __device__ __forceinline__ explicit DecodeWork(const WindowDecodeArgs& a) {
        const int G = a.n_q_heads / a.n_kv_heads, blocks = (G + 15) / 16;
        unsigned b = blockIdx.x;
        split = b % a.nsplit;
        b /= a.nsplit;
        const int hb = b % blocks;
        b /= blocks;
        kh = b % a.n_kv_heads;
        r = b / a.n_kv_heads;
        h0 = kh * G + hb * 16;
        heads = min(16, G - hb * 16);
        room = min(16, G);
    }
};

// The waves' sums, references and weights in LDS joined: to the output, or as one of nsplit parts.
template <typename T, int HD, int WAVES>
__device__ __forceinline__ void join_waves(const WindowDecodeArgs& a, const DecodeWork& w, int ctx, const float* lds) {
    const float *s_ref = lds + WAVES * w.room * HD, *s_l = s_ref + WAVES * w.room;
    const size_t slots = (size_t)a.rows * a.n_q_heads * a.nsplit;
    for (int i = threadIdx.x; i < w.heads * (HD / 4); i += WAVES * 64) {
        const int h = i / (HD / 4), d = i % (HD / 4) * 4;
        float top = -INFINITY, sum = 0.f;
        f32x4_t x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < WAVES; ++k) top = fmaxf(top, s_ref[k * w.room + h]);
#pragma unroll
        for (int k = 0; k < WAVES; ++k) {
            const float f = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((s_ref[k * w.room + h] - top) * kScoreUnit<HD>);
            sum += f * s_l[k * w.room + h];
            x += f * *(const f32x4_t*)(lds + (k * w.room + h) * HD + d);
        }
        if (a.nsplit == 1) {
            T* out = (T*)a.out + (size_t)w.r * a.ld_out + (size_t)(w.h0 + h) * HD + d;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = round_to<T>(ctx == 0 ? 0.f : within<T>(x[e] / sum));
        } else {
            const size_t slot = ((size_t)w.r * a.n_q_heads + w.h0 + h) * a.nsplit + w.split;
            if (d == 0) ((float2*)(a.part + slots * HD))[slot] = make_float2(top, sum);
            *(f32x4_t*)(a.part + slot * HD + d) = x;
        }
    }
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
// A lane's byte offsets in a page, of K and of V.  opaque(): what is added to them stays an immediate of the loads, not a register each.
struct LaneOffsets {
    uint32_t k, v;
    __device__ __forceinline__ LaneOffsets opaque() const {
        LaneOffsets o = *this;
        asm volatile("" : "+v"(o.k), "+v"(o.v));
        return o;
    }
};
template <typename T, int HD> __device__ __forceinline__ LaneOffsets plain_offsets(int n, int c) {
    return LaneOffsets{(n * HD + c * (16 / (uint32_t)sizeof(T))) * (uint32_t)sizeof(T), (4 * c * HD + n * (sizeof(T) == 4 ? 4 : HD / 16)) * (uint32_t)sizeof(T)};
}
// Where the pages of a layer and KV head lie: page i at first + i * stride, V `plane` bytes behind K, `size` bytes in all.
struct Pages {
    const uint8_t* first;
    size_t stride;
    uint32_t plane, size;
    __device__ __forceinline__ PageBuffer at(int page, bool there) const { return PageBuffer(first + (size_t)page * stride, there ? size : 0); }
};
template <typename T, int HD> __device__ __forceinline__ Pages plain_pages(const WindowDecodeArgs& a, int kh) {
    const size_t tile = 16 * HD * sizeof(T), layer = 2 * tile * a.n_kv_heads;
    return Pages{(const uint8_t*)a.pool + a.layer * layer + kh * tile, layer * a.n_layers, (uint32_t)(tile * a.n_kv_heads), (uint32_t)(tile * a.n_kv_heads + tile)};
}

// A 16-bit cache.  K as it lies: a lane has 8 dims of token n.  V: dims D n .. D n + D - 1 (D = HD / 16) of its four tokens, so that a row of V
// is read by 16 lanes side by side; pairs of tokens are put together by byte permutations.  Weights go in as two terms of the type, which
// leaves 2^-16 of them and less (their products are exact): the output's own rounding is what is seen.  Matrix units are idle here anyway.
template <typename T_, int HD_> struct Cache16 {
    using T = T_;
    using M = Matrix16<T>;
    static constexpr int HD = HD_, D = HD / 16, KS = HD / 32;
    static constexpr float START = M::TOP > 0.f ? 6.f : 0.f, MOST = M::TOP > 0.f ? M::TOP : 20.f;
    typedef uint32_t VRow __attribute__((ext_vector_type(D / 2)));
    static __device__ __forceinline__ LaneOffsets offsets(int n, int c) { return plain_offsets<T, HD>(n, c); }
    static __device__ __forceinline__ Pages pages(const WindowDecodeArgs& a, int kh) { return plain_pages<T, HD>(a, kh); }
    struct Query {
        u32x4_t q[KS];
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
        template <typename F> __device__ __forceinline__ void each(int c, F put) const {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int d = 0; d < D; d += 4) put((4 * c + r) * D + d, f32x4_t{acc[d][r], acc[d + 1][r], acc[d + 2][r], acc[d + 3][r]});
        }
    };
    struct Tile {
        u32x4_t k[KS];
        VRow v[4];
        __device__ __forceinline__ void load(const Pages& pages, int page, bool there, const LaneOffsets& lane) {
            const PageBuffer b = pages.at(page, there);
#pragma unroll
            for (int s = 0; s < KS; ++s) k[s] = b.get<u32x4_t>(lane.k, s * 64);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = b.get<VRow>(lane.v, i * HD * 2, pages.plane);
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
        __device__ __forceinline__ void add(const f32x4_t& p, Sums& o) const {
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
    static constexpr int HD = HD_, D = HD / 16;
    static constexpr float START = 0.f, MOST = 20.f;
    using Query = FloatQuery<HD>;
    static __device__ __forceinline__ LaneOffsets offsets(int n, int c) { return plain_offsets<float, HD>(n, c); }
    static __device__ __forceinline__ Pages pages(const WindowDecodeArgs& a, int kh) { return plain_pages<float, HD>(a, kh); }
    struct Sums : Cache16<f16_t, HD>::Sums {
        template <typename F> __device__ __forceinline__ void each(int c, F put) const { each_dims<HD>(this->acc, c, put); }
    };
    struct Tile {
        f32x4_t k[D], v[4][HD / 64];
        __device__ __forceinline__ void load(const Pages& pages, int page, bool there, const LaneOffsets& lane) {
            const PageBuffer b = pages.at(page, there);
#pragma unroll
            for (int s = 0; s < D; ++s) k[s] = b.get<f32x4_t>(lane.k, s * 64);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int d = 0; d < HD / 64; ++d) v[i][d] = b.get<f32x4_t>(lane.v, (i * HD + d * 64) * 4, pages.plane);
        }
        __device__ __forceinline__ f32x4_t scores(const Query& q) const {
            f32x4_t s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < D; ++i) float_scores(k[i], q.q[i], s);
            return s;
        }
        __device__ __forceinline__ void hide(int i) {
#pragma unroll
            for (int d = 0; d < HD / 64; ++d) v[i][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        __device__ __forceinline__ void add(const f32x4_t& p, Sums& o) const {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int d = 0; d < HD / 64; ++d) float_sums(v[i][d], p[i], o.acc + 4 * d);
        }
    };
};

// A workgroup takes a row, a KV head (up to 16 of its query heads) and a part of the row's visible pages; its waves take these in turn, a page in
// flight while one is worked on, and meet in LDS.  Weights are 2^START exp((s - ref) / sqrt(HD)); ref follows the greatest score of its column only
// where a weight would leave its range (2^MOST): most pages take no exchange between lanes.  ref is a score itself, and subtracted before scaling: where
// scores are large, a scaled one's rounding would be a factor of any size.
// Bound by the cache's bytes: 64 rows of 300-2560 tokens, 32 heads of 128, window 1024, half: 157 us, 6.1 TB/s; in float, 16 heads: 164 us.  Registers for
// two waves a SIMD at least (16 bits take 125: four fit; asked for three, float spills: 297 us).
template <typename C, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void k_window_decode(WindowDecodeArgs a) {
    using T = typename C::T;
    constexpr int HD = C::HD;
    extern __shared__ float lds[];                 // [WAVES][heads][HD] sums, then [WAVES][heads] references, [WAVES][heads] weights
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, c = lane >> 4;
    const DecodeWork w(a);
    const int* table = nullptr;
    const int ctx = row_context(a, w.r, table);
    float l = 0.f, ref = -INFINITY;                // ref: -inf as long as nothing but scores of -inf was seen
    typename C::Sums o;
    o.clear();
    bool lost = ctx < 0;
    if (ctx > 0) {
        typename C::Query q;
        q.load((const T*)a.q + (size_t)w.r * a.ld_q + (size_t)(w.h0 + min(n, w.heads - 1)) * HD, c);
        constexpr float UNIT = kScoreUnit<HD>, HIGHEST = (C::MOST - C::START) / UNIT;         // HIGHEST: of s - ref
        const Visible see(ctx, a.window, a.sinks);
        const int from = (int)((int64_t)see.n_pages * w.split / a.nsplit), to = (int)((int64_t)see.n_pages * (w.split + 1) / a.nsplit);
        const int mine = to - from > wave ? (to - from - wave + WAVES - 1) / WAVES : 0;
        const Pages pages = C::pages(a, w.kh);
        const auto index = [&](int j) { return see.page(from + wave + j * WAVES); };
        const LaneOffsets offsets = C::offsets(n, c);
        const auto page = [&](int j) { return table[index(min(j, mine - 1))]; };
        const auto fetch = [&](typename C::Tile& t, int id, bool more) {
            const bool inside = (unsigned)id < (unsigned)a.n_pages;
            lost |= !inside;
            t.load(pages, inside ? id : 0, inside && more, offsets.opaque());
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
            f32x4_t d = s - ref, p;
            if (__any(!(fmaxf(fmaxf(d[0], d[1]), fmaxf(d[2], d[3])) <= HIGHEST))) {
                const float top = column_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])));
                const float now = ref == -INFINITY || top - ref > HIGHEST ? top : ref, keep = now == ref ? 1.f : __builtin_amdgcn_exp2f((ref - now) * UNIT);
                l *= keep;
                o.scale(keep);
                ref = now;
                d = s - (ref == -INFINITY ? 0.f : ref);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(d[i], UNIT, C::START));
            l += (p[0] + p[1]) + (p[2] + p[3]);
            t.add(p, o);
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
    if (n < w.heads) {
        o.each(c, [&](int d, f32x4_t x) { *(f32x4_t*)(lds + (wave * w.room + n) * HD + d) = x; });
        if (c == 0) {
            lds[WAVES * w.room * HD + wave * w.room + n] = ref;
            lds[WAVES * w.room * (HD + 1) + wave * w.room + n] = l;
        }
    }
    __syncthreads();
    join_waves<T, HD, WAVES>(a, w, ctx, lds);
}

// Two codes as masked, v 2^-24 or v 2^-20: as they are, or (SHIFT 10) 2^14 times as large.
template <int SHIFT> __device__ __forceinline__ uint32_t code_pair(uint32_t x) {
    if constexpr (SHIFT == 24) return x;
    typedef f16_t f16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, x) * f16x2_t{16384.f, 16384.f});
}

// The 8 codes of a word of K as the halves v 2^-18, in pairs (0, 4), (1, 5), (2, 6), (3, 7).
__device__ __forceinline__ u32x4_t key_codes(uint32_t k) {
    constexpr uint32_t MASK = 0x03C003C0u;
    return u32x4_t{k << 6 & MASK, k << 2 & MASK, k >> 2 & MASK, k >> 6 & MASK};
}

// One query head over the pages that a wave has had, value by value in float: weights exp((s - ref) / sqrt(HD)), their sum to *l and what they sum up to
// o[HD].  For heads of which the weights times scales were too small for half (below).
template <typename T, int HD, int PAGES, int WAVES>
__device__ __forceinline__ void kv4_head(const WindowDecodeArgs& a, const DecodeWork& w, const Visible& see, const int* table, int first, int to, int h, float ref,
                                         float* out, float* l, int lane) {
    using L = Kv4<HD>;
    constexpr int KS = HD / 32;
    typedef uint32_t Codes __attribute__((ext_vector_type(KS)));
    const int n = lane & 15, c = lane >> 4;
    const size_t layer = (size_t)a.n_kv_heads * L::BLOCK;
    float q[KS][8], o[HD / 16] = {}, sum = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) load8<T>((const T*)a.q + (size_t)w.r * a.ld_q + (size_t)(w.h0 + h) * HD + s * 32 + c * 8, q[s]);
    for (int j = first; j < to; j += WAVES * PAGES)
        for (int i = j; i < min(j + PAGES, to); ++i) {
            const int page = see.page(i), id = table[page];
            if ((unsigned)id >= (unsigned)a.n_pages) continue;         // the row is lost anyway
            const uint8_t* block = (const uint8_t*)a.pool + ((size_t)id * a.n_layers + a.layer) * layer + (size_t)w.kh * L::BLOCK;
            const Codes k = *(const Codes*)(block + lane * L::PIECE), v = *(const Codes*)(block + L::V_CODES + lane * L::PIECE);
            const bool seen = see.sees(page * 16 + n);
            float z = 0.f, scale[L::GROUPS], center[L::GROUPS];        // of V of token n
#pragma unroll
            for (int g = 0; g < L::GROUPS; ++g) {
                const uint32_t kp = *(const uint32_t*)(block + n * 4 + L::param(0, 64 * g)), vp = *(const uint32_t*)(block + n * 4 + L::param(0, 64 * g) + L::PARAMS);
                scale[g] = seen ? unpack<f16_t>(vp, 0) : 0.f;
                center[g] = seen ? unpack<f16_t>(vp, 1) : 0.f;
#pragma unroll
                for (int s = 2 * g; s < 2 * g + 2; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) z = fmaf(q[s][e], fmaf(unpack<f16_t>(kp, 0), (float)((int)(k[s] >> 4 * e & 15) - 8), unpack<f16_t>(kp, 1)), z);
            }
            z = column_sum(z);
            const float p = seen ? __builtin_amdgcn_exp2f((z - ref) * kScoreUnit<HD>) : 0.f;
            sum += p;
#pragma unroll
            for (int e = 0; e < 4; ++e) {                              // token 4c + e, dims 16 d + n
                const float pt = __shfl(p, 4 * c + e, kWave);
#pragma unroll
                for (int g = 0; g < L::GROUPS; ++g) {
                    const float st = __shfl(scale[g], 4 * c + e, kWave), ct = __shfl(center[g], 4 * c + e, kWave);
#pragma unroll
                    for (int d = 4 * g; d < 4 * g + 4; ++d) o[d] = fmaf(pt, fmaf(st, (float)((int)(v[d / 2] >> (8 * e + 4 * (d & 1)) & 15) - 8), ct), o[d]);
                }
            }
        }
#pragma unroll
    for (int s = 1; s < 16; s <<= 1) sum += __shfl_xor(sum, s, kWave);
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) {
        o[d] = column_sum(o[d]);
        if (c == 0) out[16 * d + n] = o[d];
    }
    if (lane == 0) *l = sum;
}

// The groups (a bit each) in which any of the V scales of what a wave has seen is not 0.
template <int HD, int PAGES, int WAVES>
__device__ __forceinline__ uint32_t kv4_scaled(const WindowDecodeArgs& a, const DecodeWork& w, const Visible& see, const int* table, int first, int to, int lane) {
    using L = Kv4<HD>;
    uint32_t any = 0;
    const int n = lane & 15;
    for (int p = lane >> 4;; p += 4) {             // 16 lanes a page
        const int i = first + p / PAGES * (WAVES * PAGES) + p % PAGES;
        if (first + p / PAGES * (WAVES * PAGES) >= to) break;
        if (i >= to) continue;
        const int page = see.page(i), id = table[page];
        if ((unsigned)id >= (unsigned)a.n_pages || !see.sees(page * 16 + n)) continue;
        const uint8_t* block = (const uint8_t*)a.pool + (((size_t)id * a.n_layers + a.layer) * a.n_kv_heads + w.kh) * L::BLOCK;
#pragma unroll
        for (int g = 0; g < L::GROUPS; ++g) any |= unpack<f16_t>(*(const uint32_t*)(block + n * 4 + L::param(0, 64 * g) + L::PARAMS), 0) != 0.f ? 1u << g : 0u;
    }
    uint32_t all = 0;
#pragma unroll
    for (int g = 0; g < L::GROUPS; ++g) all |= __any(any >> g & 1) ? 1u << g : 0u;
    return all;
}

// A cache of 4 bits.  The bits of a code v = u + 8, masked where they lie, are the half v 2^-24 or (the upper of a byte) v 2^-20, below half's normal range
// and exact to the matrix units: 5 instructions for 8 codes of V; those of K, which decide exponents, are shifted to the top of the mantissa, 8
// instructions (below).  With scale s and center c of each token and 64 dims (group g),
//   q.k = sum over g of s_g (sum q v - 8 sum q) + c_g (sum of q in g),   o = sum over tokens of (p s_g) v - 8 (p s_g) + p c_g:
// the matrix units take q and p s_g, the rest is a few multiply-adds a token.  What a token costs beside its codes would outweigh them if 16 lanes
// worked on each for the 16 rows of a matrix product, so it is dealt out: scores are Q K^T with the query heads, up to HEADS = 16 / PAGES of them, repeated in
// all rows, and of PAGES pages' scores a quad of rows (lanes c) keeps the page that is its own: a lane has one token of PAGES x 16 for R heads.
// Weights p s_g go to the lanes of the second product through LDS.
// 64 rows of 512-4096 tokens, 32 heads of 128: 115 us, 6.0 TB/s (68 with all pages in L2; lanes of four tokens for all 16 rows: 142).  PAGES goes by the query
// heads of a KV head, 1, up to 4, up to 8, more: with PAGES = 2 for one head 137, 1 for it 182; for two heads 78 with 4, 81 with 2; for
// eight (174 MB instead of 690) 47 with 2, 65 with 1 (49.5 now, with what is said below): bound by the steps of a wave there, two waves a SIMD.  Waves that ask for registers for three a
// SIMD: one head 115, eight 217.
// A query is scaled to have its greatest magnitude in [2^14, 2^15) and taken as halves, exact from half and bfloat16 down to 2^-35 of that.  Of float calls it
// comes in two terms, as p s_g does, which leave 2^-24.  The matrix units do not normalize what is below half's normal range before they align a sum:
// codes v 2^-24 would leave 2^-17 of a score's greatest term (one of 3500: half outputs off by 0.4 %, 13 times what the formula in float32 is), those
// shifted up leave 2^-23 and less (one head 114 -> 115.5 us, two 78.5 -> 80, eight 47 -> 48.7).  Sums of V lose as much of their greatest term, which is far
// below the half step that p s_g is rounded by; float calls take codes of V 2^14 times as large (one head 127 us).
// Weights are such that p s_g fits half: 2^10 for the largest scales that come first, less where larger ones follow.  Half a step of the least that half
// holds is 2^-25, so that heads with less of p s_g than LEAST in a group, 2^-15 of that or (float) 2^-9, are taken again by kv4_head (64 rows of 512-4096
// tokens: 115.5 us, all heads again 276; where all scales of V are 0, which is looked up first, 151; without this two heads 80 us, with it 82).
template <typename T, int HD, int PAGES, int R, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void k_kv4_decode(WindowDecodeArgs a) {
    using L = Kv4<HD>;
    constexpr int KS = HD / 32, GROUPS = L::GROUPS, TERMS = sizeof(T) == 4 ? 2 : 1, HEADS = 16 / PAGES, QUADS = HEADS / 4;
    constexpr int K_SHIFT = 18, V_SHIFT = TERMS > 1 ? 10 : 24;
    constexpr float K_CODE = 1.f / (1 << K_SHIFT), V_CODE = 1.f / (1 << V_SHIFT), MOST = 4.f;         // MOST: log2 of the greatest weight, above the offset
    constexpr float LEAST = TERMS > 1 ? 1.f : 0x1p-6f;                // of a head's sum of p s_g in half (below)
    typedef uint32_t Codes __attribute__((ext_vector_type(KS)));
    extern __shared__ float lds[];                 // as above; while pages are worked on, weights [WAVES][TERMS][GROUPS][PAGES][HEADS][16 tokens] of half
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, c = lane >> 4;
    const DecodeWork w(a);
    const int* table = nullptr;
    const int ctx = row_context(a, w.r, table);
    const int own = c / QUADS, quad = c % QUADS;   // the lane's page of PAGES, and its heads 4 quad + r
    float l[R] = {}, ref[R], wsum[GROUPS][R] = {}, csum[GROUPS][R] = {};
    float off = INFINITY;                          // weights are 2^-off exp((s - ref) / sqrt(HD)); infinite: none yet
    f32x4_t o[HD / 16];                            // heads 4 quad + r, dim 16 d + n; in units of V_CODE, odd d of 16 V_CODE
#pragma unroll
    for (int r = 0; r < R; ++r) ref[r] = -INFINITY;
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    bool lost = ctx < 0;
    if (ctx > 0) {
        const int mine_head = min(n % HEADS, w.heads - 1);         // of row n of Q and of the weights
        u32x4_t q[KS][TERMS];
        f32x4_t first[GROUPS];                                     // -8 times the sum of q in the group, in units of K_CODE
        int back[R];                                               // score = 2^back s
        {
            const T* p = (const T*)a.q + (size_t)w.r * a.ld_q + (size_t)(w.h0 + mine_head) * HD + c * 8;
            float f[KS][8], m = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                load8<T>(p + s * 32, f[s]);
#pragma unroll
                for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(f[s][e]));
            }
            m = column_max(m);
            const int up = m > 0.f && m < INFINITY ? min(100, 14 - ilogbf(m)) : 0;
#pragma unroll
            for (int r = 0; r < R; ++r) back[r] = __shfl(K_SHIFT - up, 4 * quad + r, kWave);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                float sum = 0.f;
#pragma unroll
                for (int s = 2 * g; s < 2 * g + 2; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum += f[s][e] = ldexpf(f[s][e], up);
                sum = column_sum(sum) * (-8.f * K_CODE);
#pragma unroll
                for (int r = 0; r < 4; ++r) first[g][r] = __shfl(sum, 4 * quad + r, kWave);
            }
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int t = 0; t < TERMS; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {                  // codes of a word come in the order 0 4 1 5 2 6 3 7
                        const uint32_t h = pack2<f16_t>(f[s][e], f[s][e + 4]);
                        q[s][t][e] = h;
                        f[s][e] -= unpack<f16_t>(h, 0);
                        f[s][e + 4] -= unpack<f16_t>(h, 1);
                    }
        }
        const Visible see(ctx, a.window, a.sinks);
        const int from = (int)((int64_t)see.n_pages * w.split / a.nsplit), to = (int)((int64_t)see.n_pages * (w.split + 1) / a.nsplit);
        const size_t layer = (size_t)a.n_kv_heads * L::BLOCK, stride = layer * a.n_layers;
        const uint8_t* base = (const uint8_t*)a.pool + a.layer * layer + (size_t)w.kh * L::BLOCK;
        const uint32_t piece = lane * L::PIECE;
        uint16_t* weights = (uint16_t*)lds + wave * (TERMS * GROUPS * 256);
        // token n lies at place (0 2 1 3)[n % 4] of its four, the order of the codes of V
        uint16_t* put = weights + (own * HEADS + 4 * quad) * 16 + (n & 12) + (n & 1) * 2 + (n >> 1 & 1);
        const uint16_t* get = weights + mine_head * 16 + 4 * c;
        constexpr float UNIT = kScoreUnit<HD>, HIGHEST = MOST / UNIT;

        struct Tile {
            Codes k[PAGES], v[PAGES];
            uint32_t kp[GROUPS], vp[GROUPS];       // (scale, center) of the lane's token
        };
        const auto number = [&](int j) {           // of the lane's page in block j; of a block behind the last, the last page
            return table[see.page(min(from + (wave + j * WAVES) * PAGES + own, to - 1))];
        };
        const auto fetch = [&](Tile& t, int id, int j) {
            const bool inside = (unsigned)id < (unsigned)a.n_pages;
            lost |= !inside;
            id = inside ? id : 0;
#pragma unroll
            for (int p = 0; p < PAGES; ++p) {
                const int page = __builtin_amdgcn_readlane(id, p * (64 / PAGES));
                const PageBuffer b(base + (size_t)page * stride, from + (wave + j * WAVES) * PAGES + p < to ? L::BLOCK : 0);
                uint32_t at = piece;
                asm volatile("" : "+v"(at));       // offsets stay immediates of the loads, not a register each
                t.k[p] = b.get<Codes>(at, 0);
                t.v[p] = b.get<Codes>(at, L::V_CODES);
            }
            const uint8_t* par = base + (size_t)id * stride + n * 4;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                t.kp[g] = __builtin_nontemporal_load((const uint32_t*)(par + L::param(0, 64 * g)));
                t.vp[g] = __builtin_nontemporal_load((const uint32_t*)(par + L::PARAMS + L::param(0, 64 * g)));
            }
        };
        const auto rescale = [&](const float (&keep)[4]) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                l[r] *= keep[r];
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    wsum[g][r] *= keep[r];
                    csum[g][r] *= keep[r];
                }
            }
#pragma unroll
            for (int d = 0; d < HD / 16; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[d][r] *= keep[r];
        };
        const auto over_tokens = [&](float x) {    // greatest over all tokens of the head
#pragma unroll
            for (int s = 1; s < 16; s <<= 1) x = fmaxf(x, __shfl_xor(x, s, kWave));
#pragma unroll
            for (int s = 16 * QUADS; s < 64; s <<= 1) x = fmaxf(x, __shfl_xor(x, s, kWave));
            return x;
        };
        const auto step = [&](Tile& t, int j) {
            float s[R];
            {
                f32x4_t raw[GROUPS];
#pragma unroll
                for (int p = 0; p < PAGES; ++p)
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) {
                        f32x4_t x = first[g];
#pragma unroll
                        for (int i = 2 * g; i < 2 * g + 2; ++i) {
                            const u32x4_t h = key_codes(t.k[p][i]);
#pragma unroll
                            for (int e = 0; e < TERMS; ++e) x = Matrix16<f16_t>::qk(q[i][e], h, x);
                        }
#pragma unroll
                        for (int r = 0; r < R; ++r) raw[g][r] = p == 0 || own == p ? x[r] : raw[g][r];
                    }
#pragma unroll
                for (int r = 0; r < R; ++r) s[r] = 0.f;
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    const float center = unpack<f16_t>(t.kp[g], 1) * -0.125f;
#pragma unroll
                    for (int r = 0; r < R; ++r) s[r] = fmaf(unpack<f16_t>(t.kp[g], 0), raw[g][r], fmaf(center, first[g][r], s[r]));
                }
            }
            const int i = from + (wave + j * WAVES) * PAGES + own;
            const bool seen = i < to && see.sees(see.page(i) * 16 + n);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) t.vp[g] = seen ? t.vp[g] : 0;
            float d[R], p[R], top = -INFINITY;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                s[r] = seen ? ldexpf(s[r], back[r]) : -INFINITY;
                d[r] = s[r] - ref[r];
                top = r == 0 ? d[r] : fmaxf(top, d[r]);
            }
            const auto scale = [&](int g) { return unpack<f16_t>(t.vp[g], 0); };
            if (__any(!(top <= HIGHEST))) {
                if (off == INFINITY) {             // p s is at most 2^10 for the scales here; later ones may be 2^5 times as large
                    float m = 0.f;
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) m = fmaxf(m, fabsf(scale(g)));
                    m = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(wave_max(m))));
                    off = m > 0.f && m < INFINITY ? (float)ilogbf(m) - 9.f : -14.f;
                }
                float keep[4] = {1.f, 1.f, 1.f, 1.f};
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float high = over_tokens(s[r]), now = ref[r] == -INFINITY || high - ref[r] > HIGHEST ? high : ref[r];
                    keep[r] = now == ref[r] ? 1.f : __builtin_amdgcn_exp2f((ref[r] - now) * UNIT);
                    ref[r] = now;
                    d[r] = s[r] - (now == -INFINITY ? 0.f : now);
                }
                rescale(keep);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(d[r], UNIT, -off));
            float ps[GROUPS][R], high = 0.f;
            const auto multiply = [&]() {
                high = 0.f;
#pragma unroll
                for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        ps[g][r] = fmaf(p[r], scale(g), 0.f);
                        high = fmaxf(high, fabsf(ps[g][r]));
                    }
            };
            multiply();
            if (__any(high > 32768.f)) {           // much larger scales than before: all weights 2^by times smaller from here on
                high = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(wave_max(high))));
                const float by = high < INFINITY ? (float)ilogbf(high) - 9.f : 60.f, f = __builtin_amdgcn_exp2f(-by);
                const float keep[4] = {f, f, f, f};
#pragma unroll
                for (int r = 0; r < R; ++r) p[r] *= f;
                rescale(keep);
                off += by;
                multiply();
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                l[r] += p[r];
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    csum[g][r] = fmaf(p[r], unpack<f16_t>(t.vp[g], 1), csum[g][r]);
                    float rest = ps[g][r];
#pragma unroll
                    for (int x = 0; x < TERMS; ++x) {
                        const f16_t h = (f16_t)rest;
                        put[(x * GROUPS + g) * 256 + r * 16] = __builtin_bit_cast(uint16_t, h);
                        wsum[g][r] += (float)h;    // as the matrix units see them
                        rest -= (float)h;
                    }
                }
            }
            __builtin_amdgcn_wave_barrier();       // a wave's LDS accesses keep their order; this states it to the compiler
            asm volatile("" : : : "memory");
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int x = 0; x < TERMS; ++x)
#pragma unroll
                    for (int pp = 0; pp < PAGES; pp += 2) {
                        const u32x2_t wa = *(const u32x2_t*)(get + (x * GROUPS + g) * 256 + pp * HEADS * 16);
                        const u32x2_t wb = PAGES > 1 ? *(const u32x2_t*)(get + (x * GROUPS + g) * 256 + (PAGES > 1 ? pp + 1 : 0) * HEADS * 16) : u32x2_t{0, 0};
#pragma unroll
                        for (int i = 2 * g; i < 2 * g + 2; ++i) {
                            const uint32_t va = t.v[pp][i], vb = PAGES > 1 ? t.v[PAGES > 1 ? pp + 1 : 0][i] : 0;
#pragma unroll
                            for (int d = 0; d < 2; ++d) {          // tokens (0, 2), (1, 3) of dims 32 i + n, then of dims 32 i + 16 + n
                                const uint32_t mask = d ? 0x00F000F0u : 0x000F000Fu;
                                const u32x2_t a2{code_pair<V_SHIFT>(va & mask), code_pair<V_SHIFT>(va >> 8 & mask)};
                                if (PAGES > 1) {
                                    const u32x4_t h{a2[0], a2[1], code_pair<V_SHIFT>(vb & mask), code_pair<V_SHIFT>(vb >> 8 & mask)};
                                    o[2 * i + d] = Matrix16<f16_t>::qk(u32x4_t{wa[0], wa[1], wb[0], wb[1]}, h, o[2 * i + d]);
                                } else {
                                    o[2 * i + d] = Matrix16<f16_t>::pv(wa, a2, o[2 * i + d]);
                                }
                            }
                        }
                    }
            asm volatile("" : : : "memory");
            __builtin_amdgcn_wave_barrier();
        };
        const int blocks = (to - from + PAGES - 1) / PAGES, mine = blocks > wave ? (blocks - wave + WAVES - 1) / WAVES : 0;
        // Two blocks in flight, page numbers a step further ahead.  Loads of pages behind the last are issued too, of nothing: so every wait in the loop is
        // for a known number of loads.
        if (mine > 0) {
            Tile t0, t1;
            int id0 = number(0), id1 = number(1);
            fetch(t0, id0, 0);
            for (int j = 0; j < mine; j += 2) {
                id0 = number(j + 2);
                fetch(t1, id1, j + 1);
                step(t0, j);
                id1 = number(j + 3);
                fetch(t0, id0, j + 2);
                if (j + 1 < mine) step(t1, j + 1);
            }
        }
    }
    lost = __any(lost);
    const float whole = off == INFINITY ? 1.f : ldexpf(1.f, (int)off);
    const auto total = [&](float x) {              // over all tokens of the head
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) x += __shfl_xor(x, s, kWave);
#pragma unroll
        for (int s = 16 * QUADS; s < 64; s <<= 1) x += __shfl_xor(x, s, kWave);
        return x;
    };
    __syncthreads();                               // nobody reads weights any more
    uint32_t few = 0;                              // bit 4 g + r: the lane's head has too little of p s_g; 16 further: it has, and nothing
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int h = 4 * quad + r;
        const float all = total(l[r]) * whole;
        float more[GROUPS];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const float weight = total(wsum[g][r]);
            if (all > 0.f && fabsf(weight) < LEAST) few |= (weight == 0.f ? 0x10001u : 1u) << (4 * g + r);
            more[g] = total(csum[g][r]) - 8.f * weight;
        }
        if (own == 0 && h < w.heads) {
            float* to = lds + (wave * w.room + h) * HD + n;
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) to[16 * d] = fmaf(o[d][r], (d & 1 ? 0.0625f : 1.f) / V_CODE, more[d / 4]) * whole;
            if (n == 0) {
                lds[WAVES * w.room * HD + wave * w.room + h] = ref[r];
                lds[WAVES * w.room * (HD + 1) + wave * w.room + h] = lost ? NAN : all;
            }
        }
    }
    if (__builtin_expect(__any(few != 0) && !lost, 0)) {
        const Visible see(ctx, a.window, a.sinks);
        const int first = (int)((int64_t)see.n_pages * w.split / a.nsplit) + wave * PAGES, to = (int)((int64_t)see.n_pages * (w.split + 1) / a.nsplit);
        uint32_t scaled = (1u << GROUPS) - 1;      // nothing is right where all scales are 0
        if (__any(few >> 16 != 0)) scaled = kv4_scaled<HD, PAGES, WAVES>(a, w, see, table, first, to, lane);
        uint32_t again = 0;                        // a bit a head
        for (int g = 0; g < GROUPS; ++g)
            for (int r = 0; r < R; ++r) {
                const uint64_t low = __ballot(few >> (4 * g + r) & 1 && (scaled >> g & 1 || !(few >> (16 + 4 * g + r) & 1)));
                for (int x = 0; x < QUADS; ++x) again |= (uint32_t)(low >> 16 * x & 1) << (4 * x + r);
            }
        again &= (1u << w.heads) - 1;
        asm volatile("" : : : "memory");
        __builtin_amdgcn_wave_barrier();
        for (; again; again &= again - 1) {
            const int h = __builtin_ctz(again), slot = wave * w.room + h;
            kv4_head<T, HD, PAGES, WAVES>(a, w, see, table, first, to, h, lds[WAVES * w.room * HD + slot], lds + slot * HD, lds + WAVES * w.room * (HD + 1) + slot, lane);
        }
    }
    __syncthreads();
    join_waves<T, HD, WAVES>(a, w, ctx, lds);
}

// The parts of a (row, query head) joined, by four waves whose sums meet in LDS: of 64 parts (64 heads of 128) 4.3 us, with one wave 10.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_window_join(WindowDecodeArgs a) {
    constexpr int LANES = HD / 4, GROUPS = 256 / LANES;         // a group of lanes takes every GROUPS-th part, four dims a lane
    __shared__ f32x4_t s_x[GROUPS][LANES];
    __shared__ float s_w[64], s_l;
    const int t = threadIdx.x, g = t / LANES, d = t % LANES * 4, h = blockIdx.x % a.n_q_heads, r = blockIdx.x / a.n_q_heads;
    const size_t slot = (size_t)blockIdx.x * a.nsplit, slots = (size_t)a.rows * a.n_q_heads * a.nsplit;
    if (t < 64) {                                                      // nsplit <= 64
        const float2 ml = t < a.nsplit ? ((const float2*)(a.part + slots * HD))[slot + t] : make_float2(-INFINITY, 0.f);
        const float m = wave_max(ml.x), w = __builtin_amdgcn_exp2f((ml.x - (m == -INFINITY ? 0.f : m)) * kScoreUnit<HD>), l = wave_sum(w * ml.y);
        s_w[t] = w;
        if (t == 0) s_l = l;
    }
    __syncthreads();
    f32x4_t x{0.f, 0.f, 0.f, 0.f};
    for (int s = g; s < a.nsplit; s += GROUPS) x += s_w[s] * *(const f32x4_t*)(a.part + (slot + s) * HD + d);
    s_x[g][d / 4] = x;
    __syncthreads();
    if (t >= LANES) return;
    for (int i = 1; i < GROUPS; ++i) x += s_x[i][t];
    const bool empty = a.ctx_len[r] <= 0;
    T* o = (T*)a.out + (size_t)r * a.ld_out + (size_t)h * HD + d;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = round_to<T>(empty ? 0.f : within<T>(x[e] / s_l));
}

// Pages that a row may see.
static int64_t visible_pages(int64_t max_pages, int window, int sinks) {
    return std::min<int64_t>(max_pages, (sinks + 15ll) / 16 + (window + 15ll) / 16 + 1);
}
// Workgroups of a call in one part.
static int64_t decode_blocks(int rows, int n_q_heads, int n_kv_heads) { return (int64_t)rows * n_kv_heads * ((n_q_heads / n_kv_heads + 15) / 16); }

// Waves of a workgroup over a plain cache: most where contexts are long, four where 16 heads' sums of eight would take more than 64 KB of LDS.
static int most_waves(int group) { return group > 8 ? 4 : 8; }
// Eight with 64 pages and more to a row or in parts, four below, and one where eight pages or fewer meet workgroups enough to fill the chip: starting idle
// waves then costs more than the pages (95 rows of 15-50 tokens, 32 heads of 128: 8 waves 29.4 us, 4 19.8, 1 14.3; 64 rows of 128 tokens 36, 26.4,
// 25.2; 16 rows of 500 28.3, 26.3, 31.3; 16 rows of 2000, 12 heads of 64 26.1, 26.7, 62).  The pages that a row can have are the table's width: on one wider
// than the contexts need, short rows take the time of eight waves.
static int decode_waves(const WindowDecodeArgs& a) {
    const int group = a.n_q_heads / a.n_kv_heads;
    const int64_t pages = visible_pages(a.pt_stride, a.window, a.sinks), blocks = decode_blocks(a.rows, a.n_q_heads, a.n_kv_heads);
    if (a.nsplit > 1 || pages >= 64) return most_waves(group);
    return pages <= 8 && blocks >= 1024 ? 1 : 4;
}
// Four over 4 bits; where workgroups fill the chip one for short rows, and two for longer ones, or where there are so many that long and short ones even out
// (64 rows of 256 tokens, 32 heads of 128: 4 waves 29.4 us, 2 21.6, 1 18.2; 136 rows of 40-4072, 64 / 8 heads, window 587, float 48.5, 46.5,
// 51.6; 256 rows of 16-2048, 32 heads 238, 202, 208; but 64 rows of 512-4096 138, 147, 147, and 16 rows of 500 12.3, 12.4, 13.4).  Eight:
// 64 rows of 512-4096 121 us where four take 115, 131072 tokens 47, 38.
static int kv4_waves(const WindowDecodeArgs& a) {
    const int64_t pages = visible_pages(a.pt_stride, a.window, a.sinks), blocks = decode_blocks(a.rows, a.n_q_heads, a.n_kv_heads);
    if (a.nsplit > 1 || blocks < 1024) return 4;
    return pages <= 32 ? 1 : pages <= 96 || blocks >= 4096 ? 2 : 4;
}

// Into how many parts the visible pages of a row are cut, by the waves of the plain cache's kernel for both: none below 6 pages a wave, where joining costs more than it gives (two rows of 12 heads of
// 64, 700 tokens 7.5 us in one part, 7.8 in four; 1000 tokens 9.2 and 8.2); else a power of two, which leaves the parts of a row's heads on as few XCDs as
// there are (32 heads of 128, 4000 tokens: 8 parts 16.0 us, 12 18.6, 16 16.2), of a page a wave at least and of 2048 waves in all (8 rows of
// 8 KV heads, 2000 tokens: 4 parts 15.8 us, 2 21.7, 8 17.2), or 4096 with 32 pages a wave and more (one row of 131072 tokens in 4 bits, 8 KV
// heads: 64 parts 39 us, 32 44).
int window_decode_nsplit(int rows, int n_q_heads, int n_kv_heads, int max_ctx, int window, int sinks) {
    const int64_t pages = visible_pages((max_ctx + 15ll) / 16, window, sinks);
    const int waves = most_waves(n_q_heads / n_kv_heads);
    const int64_t all = decode_blocks(rows, n_q_heads, n_kv_heads) * waves;
    if (pages < 6 * waves) return 1;
    int n = 1;
    while (n < 64 && 2 * n * waves <= pages && 2 * n * all <= (pages >= 32 * n * waves ? 4096 : 2048)) n *= 2;
    return n;
}

size_t window_decode_scratch_floats(int rows, int n_q_heads, int head_dim, int nsplit) {
    return (size_t)rows * n_q_heads * nsplit * (head_dim + 2);
}

// The rows in turns of what one launch holds: `start` launches `blocks` workgroups of `waves` waves a row.
template <typename T, int HD, typename F>
static hipError_t in_turns(hipStream_t st, const WindowDecodeArgs& a, int waves, F start) {
    const int64_t blocks = decode_blocks(1, a.n_q_heads, a.n_kv_heads) * a.nsplit;
    const int most = (int)std::min<int64_t>(kLaunchThreads / (64 * waves) / std::max<int64_t>(blocks, a.n_q_heads), 1 << 24);
    for (int first = 0; first < a.rows; first += most) {
        WindowDecodeArgs p = a;
        p.q = (const T*)a.q + (size_t)first * a.ld_q;
        p.out = (T*)a.out + (size_t)first * a.ld_out;
        p.row_sample += first;
        p.ctx_len += first;
        p.rows = std::min(most, a.rows - first);
        start((unsigned)(p.rows * blocks), p);
        const unsigned heads = (unsigned)p.rows * (unsigned)a.n_q_heads;
        if (a.nsplit > 1) k_window_join<T, HD><<<heads, 256, 0, st>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename C>
static hipError_t decode_rows(hipStream_t st, const WindowDecodeArgs& a) {
    const int waves = decode_waves(a);
    const size_t lds = (size_t)waves * std::min(16, a.n_q_heads / a.n_kv_heads) * (C::HD + 2) * sizeof(float);
    return in_turns<typename C::T, C::HD>(st, a, waves, [&](unsigned grid, const WindowDecodeArgs& p) {
        if (waves == 8) k_window_decode<C, 8><<<grid, 512, lds, st>>>(p);
        else if (waves == 4) k_window_decode<C, 4><<<grid, 256, lds, st>>>(p);
        else k_window_decode<C, 1><<<grid, 64, lds, st>>>(p);
    });
}

template <typename T, int HD, int WAVES>
static hipError_t kv4_typed(hipStream_t st, const WindowDecodeArgs& a) {
    const int group = a.n_q_heads / a.n_kv_heads;
    const size_t sums = (size_t)WAVES * std::min(16, group) * (HD + 2) * sizeof(float), weights = (size_t)WAVES * (sizeof(T) == 4 ? 2 : 1) * (HD / 64) * 512;
    const size_t lds = std::max(sums, weights);
    return in_turns<T, HD>(st, a, WAVES, [&](unsigned grid, const WindowDecodeArgs& p) {
        if (group == 1) k_kv4_decode<T, HD, 4, 1, WAVES><<<grid, WAVES * 64, lds, st>>>(p);
        else if (group <= 4) k_kv4_decode<T, HD, 4, 4, WAVES><<<grid, WAVES * 64, lds, st>>>(p);
        else if (group <= 8) k_kv4_decode<T, HD, 2, 4, WAVES><<<grid, WAVES * 64, lds, st>>>(p);
        else k_kv4_decode<T, HD, 1, 4, WAVES><<<grid, WAVES * 64, lds, st>>>(p);
    });
}

template <typename T, int HD>
static hipError_t kv4_rows(hipStream_t st, const WindowDecodeArgs& a) {
    const int waves = kv4_waves(a);
    return waves == 1 ? kv4_typed<T, HD, 1>(st, a) : waves == 2 ? kv4_typed<T, HD, 2>(st, a) : kv4_typed<T, HD, 4>(st, a);
}

hipError_t launch_window_decode(hipStream_t st, int dtype, bool four_bits, int head_dim, const WindowDecodeArgs& a) {
#define RLHF_DECODE(HD)                                                                                                        \
    if (head_dim == HD) {                                                                                                      \
        if (dtype == kBF16) return four_bits ? kv4_rows<bf16_t, HD>(st, a) : decode_rows<Cache16<bf16_t, HD>>(st, a);          \
        if (dtype == kF16) return four_bits ? kv4_rows<f16_t, HD>(st, a) : decode_rows<Cache16<f16_t, HD>>(st, a);             \
        return four_bits ? kv4_rows<float, HD>(st, a) : decode_rows<CacheFloat<HD>>(st, a);                                    \
    }
    RLHF_DECODE(64)
    RLHF_DECODE(128)
#undef RLHF_DECODE
    return hipErrorInvalidValue;
}

}  // namespace rlhf
