// Embedding lookup with scaling, and the gradient of its table.  Rows go through registers once.  The lookup is bound by memory: 8192
// rows of 4096 bf16 17 us = 5.6 TB/s.  The gradient is bound by memory where the table is large (8192 rows of 4096 bf16 into
// 32000 x 4096 float 123 us = 4.8 TB/s, into bf16 76 us; added to it, 172 MB, 57 us), and by the round trips that depend on each other where it is small
// (tokens, places, rows, chunks: 32768 rows of 768 half, half of them one token, 55 us where memory alone would take 18).
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "vec.h"

namespace rlhf {

// How threads lie over rows of d columns.  A thread has H pieces of C columns of a row, 16 bytes of the wider type each; `wide` threads (a
// power of two, 8 to 256) lie side by side, their first pieces next to each other, then their second ones, so that the lanes of a
// wave write whole lines; 256 / wide rows share a workgroup, and grid.y covers what is wider than one.
template <typename A, typename B> struct Shape {
    static constexpr int C = sizeof(A) == 2 && sizeof(B) == 2 ? 8 : 4, H = 8 / C;
};
struct Grid { int wide_log2, slices; };
// p, ld: what the pieces go by (my_columns); rows that start off a boundary may have a piece more.  At most 2^most threads side by
// side.
template <typename T> static Grid grid_of(const T* p, size_t ld, int d, int C, int H, int most = 8) {
    const bool on_boundary = (uintptr_t)p % (C * sizeof(T)) == 0 && ld % C == 0;
    const int pieces = (d + (on_boundary ? C - 1 : 2 * C - 2)) / C;
    int lg = 3;
    while (lg < most && (H << lg) < pieces) ++lg;
    return Grid{lg, (pieces + (H << lg) - 1) / (H << lg)};
}
// Row and column numbers are ints.
static bool sizes_fit(int rows, int d, int vocab) { return rows <= 1 << 30 && vocab <= 1 << 30 && d <= 1 << 22; }

// A piece is the columns [lo, hi) of a row, C or, at the row's ends, fewer.  It is read as the C columns from `at` on, which are
// inside the row wherever that has C columns: a short piece reads some of its neighbour's, since loads one by one would
// have to be waited for before the next row's are sent (32768 rows of 768 half, half of them one token: 66 us, so 55).
struct Cols { int at, lo, hi; };
template <int C> __device__ __forceinline__ Cols cols_of(int lo, int hi, int d) { return Cols{min(lo, max(0, d - C)), lo, hi}; }

// This thread's pieces of a row at p: pieces meet where the row reaches a boundary of C elements.
template <int C, int H, typename T> __device__ __forceinline__ void my_columns(const T* p, int slice, int wide_log2, int d, Cols (&cols)[H]) {
    const int shift = (int)((uintptr_t)p % (C * sizeof(T)) / sizeof(T));
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const int piece = ((slice * H + h) << wide_log2) + (threadIdx.x & ((1 << wide_log2) - 1));
        cols[h] = cols_of<C>(max(0, piece * C - shift), min(d, piece * C - shift + C), d);
    }
}

// A piece as it lies in memory, of a row of d columns.
template <typename T, int C> struct Piece {
    Vec<T, C> v;
    template <bool ONCE> __device__ __forceinline__ void load(const T* row, const Cols& c, int d) {
        if (c.lo >= c.hi) return;
        if (c.at + C <= d) return v.template load<ONCE>(row + c.at);
        float x[C];                     // rows of fewer than C columns
#pragma unroll
        for (int e = 0; e < C; ++e) x[e] = c.at + e < d ? to_f32<T>(row[c.at + e]) : 0.f;
        v.set(x);
    }
    template <bool ONCE> __device__ __forceinline__ void store(T* row, const Cols& c) const {
        if (c.hi - c.lo == C) return v.template store<ONCE>(row + c.lo);
        float x[C];
        v.get(x);
#pragma unroll
        for (int e = 0; e < C; ++e)
            if (c.at + e >= c.lo && c.at + e < c.hi) row[c.at + e] = round_to<T>(x[e]);
    }
};

template <typename T, typename O>
__global__ __launch_bounds__(256) void k_embed_rows(const T* __restrict__ table, size_t ld_table, const int* __restrict__ tokens,
                                                    O* __restrict__ out, size_t ld_out, float scale, int rows, int d, int vocab, int wide_log2) {
    constexpr int C = Shape<T, O>::C, H = Shape<T, O>::H;
    const int r = blockIdx.x * (256 >> wide_log2) + (threadIdx.x >> wide_log2);
    if (r >= rows) return;
    const int v = tokens[r];
    const bool known = (unsigned)v < (unsigned)vocab;
    O* o = out + (size_t)r * ld_out;
    Cols cols[H];
    my_columns<C, H>(o, blockIdx.y, wide_log2, d, cols);
    Piece<T, C> in[H];
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (known) in[h].template load<false>(table + (size_t)v * ld_table, cols[h], d);
#pragma unroll
    for (int h = 0; h < H; ++h) {
        float x[C];
        in[h].v.get(x);
#pragma unroll
        for (int e = 0; e < C; ++e) x[e] = known ? x[e] * scale : v < 0 ? 0.f : NAN;
        Piece<O, C> res;
        res.v.set(x);
        // the next reader is on any of the 8 XCDs, so little is lost: 8192 rows of 4096 bf16 into float 37 us, evict-first 26
        res.template store<true>(o, cols[h]);
    }
}

// ---- gradient: rows grouped by token, then every token's rows summed, in float and in an order that follows from the tokens and sizes: a run
// up to a chunk long in ascending order; a longer one chunk by chunk, the chunks' sums joined by workers that take every WORKERS-th; few
// rows (k_few_rows_grad) dealt to a workgroup's groups in turn, the groups' sums joined.
// The vocabulary is dealt to 2^log2 buckets by its low bits (frequent tokens have neighbouring ids), `subs` tokens each, and the
// rows to `parts` parts, 256 workgroups together unless the vocabulary is large.  A workgroup for each bucket and part reads
// all tokens out of the L2, counts its bucket's and how many lie in earlier buckets, and puts the rows of its part into their
// places: a row's place follows from the counts alone, so there are no sort passes over memory and no atomics whose order
// could show.  Alone it takes 8.8 us for 8192 tokens and 17 to 18 for 32768.
struct Buckets { int log2, subs, parts; };
constexpr int kMaxSubs = 512;
static Buckets buckets_of(int vocab) {
    int lg = 6;
    while (((int64_t)vocab + (1ll << lg) - 1) >> lg > kMaxSubs) ++lg;
    return Buckets{lg, (int)(((int64_t)vocab + (1ll << lg) - 1) >> lg), lg < 8 ? 256 >> lg : 1};
}
// A place of the grouped order: which row it holds, and the run of its token, the places [start, start + count).
struct Place { int row, token, start, count; };
struct Run { int start, count; };

// use(token, whether it is this lane's, the lanes that have it) for each token among those of the lanes with `has`.
template <typename Use> __device__ __forceinline__ void each_token(bool has, int token, Use use) {
    for (uint64_t m = __ballot(has); m; m = __ballot(has)) {
        const int t = __builtin_amdgcn_readlane(token, __ffsll((unsigned long long)m) - 1);
        const bool same = has && token == t;
        use(t, same, __ballot(same));
        has = has && !same;
    }
}

constexpr int kAhead = 16, kPlace = 8;  // tokens a lane has in flight while they are counted, and while their rows are placed
template <int AHEAD> __device__ __forceinline__ void load_tokens(const int* tokens, int i, int end, int (&v)[AHEAD]) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) v[j] = i + j * 64 < end ? tokens[i + j * 64] : -1;
}

// LDS, in ints: next [16][subs], the count and later the next place of a wave's rows of a token; run [subs], start and count;
// early [subs], rows of earlier parts.
static size_t group_lds_bytes(const Buckets& b) { return (size_t)b.subs * 19 * sizeof(int); }

__device__ __forceinline__ void group_tokens(const int* __restrict__ tokens, int n, int vocab, const Buckets& b, int mine, int part,
                                             Place* __restrict__ places, Run* __restrict__ runs, int* __restrict__ total) {
    extern __shared__ int next[];
    __shared__ int s_part[16], s_before[16];
    Run* s_run = (Run*)(next + 16 * b.subs);
    int* early = next + 18 * b.subs;
    const int t = threadIdx.x, w = t >> 6, lane = t & 63, mask = (1 << b.log2) - 1;
    for (int i = t; i < 19 * b.subs; i += 1024) next[i] = 0;
    __syncthreads();
    // rows of a part, a sixteenth of it for each wave to place; and of a wave to count
    const int piece = (n + b.parts * 1024 - 1) / (b.parts * 1024) * 64, from = min(n, part * 16 * piece), to = min(n, from + 16 * piece);
    const int share = ((n + 1023) >> 10) << 6, first = min(n, w * share), end = min(n, first + share);
    int before = 0;
    for (int i0 = first; i0 < end; i0 += 64 * kAhead) {
        int v[kAhead];
        load_tokens(tokens, i0 + lane, end, v);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int key = (unsigned)v[j] < (unsigned)vocab ? v[j] & mask : INT32_MAX;
            before += key < mine;
            const uint64_t hits = __ballot(key == mine);
            if (hits == 0) continue;
            // 64 rows lie in one wave's piece.  One token's are counted at once (equal addresses are served one by one, and padding
            // fills waves), the others' lane by lane.
            const int i = i0 + j * 64, lead = __ffsll((unsigned long long)hits) - 1;
            int* const also = i < from ? early : i < to ? next + (i - from) / piece * b.subs : nullptr;
            const bool same = key == mine && v[j] == __builtin_amdgcn_readlane(v[j], lead);
            const int many = __popcll(__ballot(same)), sub = v[j] >> b.log2;
            if (key != mine || (same && lane != lead)) continue;
            atomicAdd(&s_run[sub].count, same ? many : 1);
            if (also) atomicAdd(&also[sub], same ? many : 1);
        }
    }
    for (int o = 32; o > 0; o >>= 1) before += __shfl_xor(before, o, kWave);
    if (lane == 0) s_before[w] = before;
    __syncthreads();
    int base = 0;
    for (int i = 0; i < 16; ++i) base += s_before[i];
    const int count = t < b.subs ? s_run[t].count : 0;
    int sum = count;                                               // inclusive over the tokens of the bucket
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(sum, o, kWave);
        if (lane >= o) sum += x;
    }
    if (lane == 63) s_part[w] = sum;
    __syncthreads();
    for (int i = 0; i < w; ++i) sum += s_part[i];
    if (t < b.subs) {
        int at = base + sum - count;
        s_run[t].start = at;
        if (part == 0) runs[(size_t)mine * b.subs + t] = Run{at, count};
        at += early[t];
        for (int i = 0; i < 16; ++i) {
            const int c = next[i * b.subs + t];
            next[i * b.subs + t] = at;
            at += c;
        }
    }
    if (mine == mask && part == 0 && t == 1023) *total = base + sum;
    __syncthreads();
    const int mine0 = min(to, from + w * piece), mine1 = min(to, mine0 + piece);
    int last = -1, at = 0;                                         // a token in a row of rows: its place is at hand
    for (int i0 = mine0; i0 < mine1; i0 += 64 * kPlace) {
        int v[kPlace];
        load_tokens(tokens, i0 + lane, mine1, v);
#pragma unroll
        for (int j = 0; j < kPlace; ++j)
            each_token((unsigned)v[j] < (unsigned)vocab && (v[j] & mask) == mine, v[j], [&](int token, bool same, uint64_t rows) {
                const int sub = token >> b.log2;
                if (token != last) {
                    if (last >= 0 && lane == 0) next[w * b.subs + (last >> b.log2)] = at;
                    // lane 0's store before the wave's load; the hardware keeps the order, the compiler need not (no instructions)
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                    at = next[w * b.subs + sub];
                    last = token;
                }
                if (same) places[at + __popcll(rows & ((1ull << lane) - 1))] = Place{i0 + j * 64 + lane, token, s_run[sub].start, s_run[sub].count};
                at += __popcll(rows);
            });
    }
}

__device__ __forceinline__ Run run_of(const Run* runs, const Buckets& b, int v) {
    return runs[(size_t)(v & ((1 << b.log2) - 1)) * b.subs + (v >> b.log2)];
}

// Zeros for the rows [from, to) of the table that have no token (runs == NULL: for all), by workgroups of THREADS threads,
// kZeroRows rows a thread.  `wide` threads lie over a row, a slice of it if it is wider.  ld, d: the table's, or those of the
// same memory as rows of another length, the last of which ends where all `elements` do.
struct Clear { int from, to, wide_log2, slices, d; size_t ld, elements; };
constexpr int kZeroRows = 8;
template <int THREADS, typename T>
__device__ __forceinline__ void clear_rows(T* __restrict__ dtable, const Clear& c, unsigned block, const Run* runs, const Buckets& b) {
    constexpr int C = 16 / sizeof(T);
    const int per = THREADS >> c.wide_log2, slice = block % c.slices;
    const int r0 = c.from + (int)(block / c.slices) * (per * kZeroRows) + (threadIdx.x >> c.wide_log2);
    const int piece = (slice << c.wide_log2) + (threadIdx.x & ((1 << c.wide_log2) - 1));
    bool empty[kZeroRows];
#pragma unroll
    for (int k = 0; k < kZeroRows; ++k) {
        const int r = r0 + k * per;
        empty[k] = r < c.to && (!runs || run_of(runs, b, r).count == 0);
    }
    Piece<T, C> zero;
    zero.v.fill(0.f);
#pragma unroll
    for (int k = 0; k < kZeroRows; ++k) {
        if (!empty[k]) continue;
        const size_t at = (size_t)(r0 + k * per) * c.ld;
        T* o = dtable + at;
        const int shift = (int)((uintptr_t)o % 16 / sizeof(T)), d = c.elements ? (int)min((size_t)c.d, c.elements - at) : c.d;
        zero.template store<true>(o, cols_of<C>(max(0, piece * C - shift), min(d, piece * C - shift + C), d));
    }
}
template <int THREADS> static int64_t clear_blocks(const Clear& c) {
    const int64_t per = (int64_t)(THREADS >> c.wide_log2) * kZeroRows;
    return (c.to - c.from + per - 1) / per * c.slices;
}

// The grouping, and beside it (workgroups behind the buckets) zeros for as many rows of the table as go out in its time.
template <typename T>
__global__ __launch_bounds__(1024) void k_group_and_clear(const int* __restrict__ tokens, int n, int vocab, Buckets b, Place* __restrict__ places,
                                                          Run* __restrict__ runs, int* __restrict__ total, T* __restrict__ dtable, Clear clear) {
    const int groups = n > 0 ? b.parts << b.log2 : 0;
    if ((int)blockIdx.x < groups) group_tokens(tokens, n, vocab, b, blockIdx.x / b.parts, blockIdx.x % b.parts, places, runs, total);
    else clear_rows<1024>(dtable, clear, blockIdx.x - groups, nullptr, b);
}

// x += rows index(0) .. index(count - 1) of m in that order, FLIGHT rows in flight, as they lie in memory.  The indices come a group
// of lanes at a time, so that no row waits for its own: `width` lanes (a power of two) of a wave share the rows, and all of
// them have to be here, those without columns too.  d: columns of a row of m.
template <int FLIGHT, int C, int H, typename G, typename Index>
__device__ __forceinline__ void sum_rows(const G* __restrict__ m, size_t ld, int d, int count, int width, Index index, const Cols (&cols)[H],
                                         float (&x)[H][C]) {
    const int lane = threadIdx.x & 63, mine = lane & (width - 1), base = lane - mine;
    for (int p0 = 0; p0 < count; p0 += width) {
        const int many = min(width, count - p0), r = index(p0 + min(mine, many - 1));
        for (int p = 0; p < many; p += FLIGHT) {
            Piece<G, C> y[FLIGHT][H];
#pragma unroll
            for (int k = 0; k < FLIGHT; ++k) {
                const int row = __shfl(r, base + min(p + k, many - 1), kWave);
                if (p + k < many)
#pragma unroll
                    for (int h = 0; h < H; ++h) y[k][h].template load<true>(m + (size_t)row * ld, cols[h], d);
            }
#pragma unroll
            for (int k = 0; k < FLIGHT; ++k)
                if (p + k < many)
#pragma unroll
                    for (int h = 0; h < H; ++h) {
                        float f[C];
                        y[k][h].v.get(f);
#pragma unroll
                        for (int e = 0; e < C; ++e) x[h][e] += f[e];
                    }
        }
    }
}

// The order is cut into chunks, of 32 places or more (what is grouped has over 512 rows).  A run of more places than a chunk has is long: workgroups of their own sum what each chunk holds of
// it (of at most two long runs: one that began before the chunk, one that begins in it), and k_long_runs joins the sums.
constexpr int kFlight = 8;
struct Chunks {
    float* part;            // [chunks][2][ld]
    size_t ld;
    int size, count;
};

struct GradArgs {
    const Place* places;    // [*total]
    const int* total;
    const Run* runs;
    Buckets b;
    Chunks c;
    size_t ld_dout, ld_table;
    float scale;
    int rows, d, wide_log2, slices;
    Clear clear;
    unsigned table_blocks, clear_blocks;
    int window;             // places of the order that share threads
};

template <int C, int H, typename G>
__device__ __forceinline__ void sum_chunk(const G* __restrict__ dout, const GradArgs& a, int k, int slice) {
    // The chunk's ends are read together with the number of places, which only the last chunk waits for.
    const int from = k * a.c.size, guess = min(a.rows, from + a.c.size);
    const Place head = a.places[from], tail = a.places[guess - 1];
    const int total = *a.total, to = min(total, guess);
    if (from >= to) return;
    Cols cols[H];
    my_columns<C, H>((const G*)nullptr, slice, a.wide_log2, a.d, cols);
    const Place ends[2] = {head, to == guess ? tail : a.places[to - 1]};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const Place& run = ends[s];
        if (run.count <= a.c.size || s != (run.start > from)) continue;       // slot 1: it begins behind the chunk's first place
        const int p = max(from, run.start), end = min(to, run.start + run.count);
        float x[H][C] = {};
        sum_rows<kFlight, C, H>(dout, a.ld_dout, a.d, end - p, min(64, 1 << a.wide_log2), [&](int i) { return a.places[p + i].row; }, cols, x);
        float* part = a.c.part + ((size_t)k * 2 + s) * a.c.ld;
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int e = 0; e < C; e += 4) {
                const Cols& c = cols[h];
                Piece<float, 4> o;
                o.v.set({x[h][e], x[h][e + 1], x[h][e + 2], x[h][e + 3]});
                o.template store<false>(part, Cols{c.at + e, max(c.lo, c.at + e), min(c.hi, c.at + e + 4)});
            }
    }
}

// Everything but the joining of long runs.  Workgroups in front: chunks of long runs.  Behind them: a window of places of the order
// each, and the short runs that begin there.  In between, evenly: zeros for rows without a token, which keep the
// memory busy while the sums wait for their rows (8192 rows of 4096 into 32000 x 4096 float: one after the other
// 90 + 36 us).
template <typename G, typename T, bool ACCUMULATE>
__global__ __launch_bounds__(256) void k_table_grad(const G* __restrict__ dout, T* __restrict__ dtable, GradArgs a) {
    constexpr int C = Shape<G, T>::C, H = Shape<G, T>::H;
    unsigned block = blockIdx.x;
    if (!ACCUMULATE && a.clear_blocks > 0) {
        const uint64_t all = a.table_blocks + a.clear_blocks;
        const unsigned before = (unsigned)((uint64_t)block * a.clear_blocks / all);
        if ((uint64_t)(block + 1ull) * a.clear_blocks / all > before) return clear_rows<256>(dtable, a.clear, before, a.runs, a.b);
        block -= before;
    }
    const int per = 256 >> a.wide_log2, chunk_groups = (a.c.count + per - 1) / per, slice = block % a.slices;
    int place = block / a.slices;
    if (place < chunk_groups) {
        const int k = place * per + (threadIdx.x >> a.wide_log2);
        if (k < a.c.count) sum_chunk<C, H>(dout, a, k, slice);
        return;
    }
    place -= chunk_groups;
    // workgroups go to the 8 XCDs in turn: the eight of a turn are exchanged by the other digits of their number, else runs of
    // 64 places would all begin on one XCD
    unsigned digits = place >> 3;
    digits ^= digits >> 3;
    digits ^= digits >> 6;
    digits ^= digits >> 12;
    const int p0 = ((place ^ (digits & 7)) * per + (threadIdx.x >> a.wide_log2)) * a.window;
    if (p0 >= a.rows) return;
    // the window's places and the next ones, one a lane of the group, read together with the number of places
    const int lane = threadIdx.x & 63, width = min(64, 1 << a.wide_log2), mine = lane & (width - 1), base = lane - mine, seen = min(width, 16);
    const Place w = a.places[min(p0 + min(mine, seen - 1), a.rows - 1)];
    const int total = *a.total;
    // from the first place of the window where a run begins to the end of the last short run that does
    const uint64_t begins = __ballot(mine < a.window && p0 + mine < total && w.start == p0 + mine) >> base & (~0ull >> (64 - width));
    if (begins == 0) return;
    int at = p0 + __ffsll((unsigned long long)begins) - 1;
    const int last = 63 - __clzll((long long)begins), many = __shfl(w.count, base + last, kWave);
    const int end = p0 + last + (many > a.c.size ? 0 : many);
    Cols cols[H];
    my_columns<C, H>((const T*)nullptr, slice, a.wide_log2, a.d, cols);
    // rows in the order of their places, kBatch in flight; a run is stored where the next begins
    constexpr int kBatch = ACCUMULATE ? 4 : 8;
    float x[H][C];
    Piece<T, C> old[H];
    T* o = nullptr;
    const auto flush = [&]() {
        if (!o) return;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            float f[C];
            if (ACCUMULATE) old[h].v.get(f);
#pragma unroll
            for (int e = 0; e < C; ++e) f[e] = ACCUMULATE ? f[e] + a.scale * x[h][e] : a.scale * x[h][e];
            Piece<T, C> res;
            res.v.set(f);
            res.template store<false>(o, cols[h]);
        }
    };
    // the places of the first batch are there already; those of the others come while the rows of the one before do
    const auto batch = [&](int p) { return a.places[min(p + min(mine, kBatch - 1), max(end, 1) - 1)]; };
    Place q;
    if (at - p0 + kBatch <= seen) {
        const int from = base + at - p0 + min(mine, kBatch - 1);
        q = Place{__shfl(w.row, from, kWave), __shfl(w.token, from, kWave), __shfl(w.start, from, kWave), 0};
    } else {
        q = batch(at);
    }
    for (; at < end; at += kBatch) {
        Piece<G, C> row[kBatch][H];
        Piece<T, C> had[kBatch][H];
        int token[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int r = __shfl(q.row, base + k, kWave), start = __shfl(q.start, base + k, kWave);
            token[k] = __shfl(q.token, base + k, kWave);
            if (start != at + k) token[k] = -1;             // the run goes on
            if (at + k < end)
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    row[k][h].template load<true>(dout + (size_t)r * a.ld_dout, cols[h], a.d);
                    if (ACCUMULATE && token[k] >= 0) had[k][h].template load<false>(dtable + (size_t)token[k] * a.ld_table, cols[h], a.d);
                }
        }
        if (at + kBatch < end) q = batch(at + kBatch);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (at + k >= end) break;
            if (token[k] >= 0) {
                flush();
                o = dtable + (size_t)token[k] * a.ld_table;
            }
#pragma unroll
            for (int h = 0; h < H; ++h) {
                float f[C];
                row[k][h].v.get(f);
                if (ACCUMULATE && token[k] >= 0) old[h] = had[k][h];
#pragma unroll
                for (int e = 0; e < C; ++e) x[h][e] = token[k] >= 0 ? f[e] : x[h][e] + f[e];
            }
        }
    }
    flush();
}

// Joins the chunks of long runs.  A workgroup looks through the runs of a bucket and has 4 * LANES columns of the long ones; LANES lanes
// take every (kJoinThreads / LANES)-th chunk, and all meet in LDS.  What bounds it is how fast one compute unit reads (about 30 GB/s
// from memory): narrow columns where there are few.
constexpr int kJoinThreads = 1024;
template <typename T, bool ACCUMULATE, int LANES>
__global__ __launch_bounds__(kJoinThreads) void k_long_runs(T* __restrict__ dtable, GradArgs a) {
    static_assert(kJoinThreads >= kMaxSubs, "a thread a token of the bucket");
    constexpr int WORKERS = kJoinThreads / LANES;
    __shared__ float part[4][kJoinThreads];
    __shared__ int s_token[kMaxSubs], s_n;
    __shared__ Run s_run[kMaxSubs];
    const int t = threadIdx.x, w = t / LANES, lo = (blockIdx.y * LANES + t % LANES) * 4;
    const Cols cols[1] = {{lo, lo, min(a.d, lo + 4)}};        // the sums' rows are padded to fours
    if (t == 0) s_n = 0;
    __syncthreads();
    if (t < a.b.subs) {
        const Run run = a.runs[(size_t)blockIdx.x * a.b.subs + t];
        if (run.count > a.c.size) {
            const int at = atomicAdd(&s_n, 1);
            s_token[at] = t << a.b.log2 | blockIdx.x;
            s_run[at] = run;
        }
    }
    __syncthreads();
    for (int j = 0; j < s_n; ++j) {                  // in any order: each is a row of its own
        const Run run = s_run[j];
        const int first = run.start / a.c.size, chunks = (run.start + run.count - 1) / a.c.size - first + 1, slot = run.start > first * a.c.size;
        float x[1][4] = {};
        sum_rows<kFlight, 4, 1>(a.c.part, a.c.ld, (int)a.c.ld, max(0, (chunks - w + WORKERS - 1) / WORKERS), LANES,
                                [&](int i) { const int c = w + WORKERS * i; return (first + c) * 2 + (c == 0 ? slot : 0); }, cols, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) part[e][t] = x[0][e];
        __syncthreads();
        if (t < LANES) {
            for (int i = 1; i < min(chunks, WORKERS); ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[0][e] += part[e][i * LANES + t];
            T* o = dtable + (size_t)s_token[j] * a.ld_table;
            Piece<T, 4> res;
            float f[4] = {};
            if (ACCUMULATE) {
                res.template load<false>(o, cols[0], a.d);
                res.v.get(f);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] += a.scale * x[0][e];
            res.v.set(f);
            res.template store<false>(o, cols[0]);
        }
        __syncthreads();
    }
}

// Few rows: no grouping ahead.  A workgroup a row; that of a token's first row finds the others, deals them to its groups of `wide`
// threads, and joins their sums.  The longest run possible is what limits it: up to 16 round trips of kFlight rows for a
// group (512 rows of 4096, added to a table: 15 us, 27 if half of them are one token, 40 if all; grouped first, 25 to 31 us
// whatever the tokens are).
constexpr int kFewRows = 2048;
static bool few_rows(int rows, int d) { return rows <= kFewRows && rows <= 16 * kFlight * (256 >> grid_of((const float*)nullptr, 0, d, 4, 2, 6).wide_log2); }

template <typename G, typename T, bool ACCUMULATE>
__global__ __launch_bounds__(256) void k_few_rows_grad(const G* __restrict__ dout, size_t ld_dout, const int* __restrict__ tokens, T* __restrict__ dtable,
                                                       size_t ld_table, float scale, int n, int d, int vocab, int wide_log2) {
    constexpr int C = Shape<G, T>::C, H = Shape<G, T>::H, EACH = kFewRows / 256;
    __shared__ uint16_t s_rows[kFewRows];
    __shared__ int s_wave[4];
    __shared__ float part[8][256];
    const int t = threadIdx.x, w = t >> 6, lane = t & 63, v = tokens[blockIdx.x];
    if ((unsigned)v >= (unsigned)vocab) return;
    T* o = dtable + (size_t)v * ld_table;
    Cols cols[H];
    my_columns<C, H>((const T*)nullptr, blockIdx.y, wide_log2, d, cols);
    const int group = t >> wide_log2, groups = 256 >> wide_log2;
    Piece<T, C> old[H];
    if (ACCUMULATE && group == 0)
#pragma unroll
        for (int h = 0; h < H; ++h) old[h].template load<false>(o, cols[h], d);
    // the rows of the token, in ascending order: a thread looks at EACH neighbours
    bool same[EACH];
    int many = 0;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int j = t * EACH + k;
        same[k] = j < n && tokens[j] == v;
        many += same[k];
    }
    int sum = many;
#pragma unroll
    for (int e = 1; e < 64; e <<= 1) {
        const int x = __shfl_up(sum, e, kWave);
        if (lane >= e) sum += x;
    }
    if (lane == 63) s_wave[w] = sum;
    __syncthreads();
    int at = sum - many, count = 0;
    for (int k = 0; k < 4; ++k) {
        if (k < w) at += s_wave[k];
        count += s_wave[k];
    }
#pragma unroll
    for (int k = 0; k < EACH; ++k)
        if (same[k]) s_rows[at++] = (uint16_t)(t * EACH + k);
    __syncthreads();
    if (s_rows[0] != blockIdx.x) return;                 // an earlier row's
    float x[H][C] = {};
    sum_rows<kFlight, C, H>(dout, ld_dout, d, max(0, (count - group + groups - 1) / groups), 1 << wide_log2,
                            [&](int j) { return (int)s_rows[group + groups * j]; }, cols, x);
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int e = 0; e < C; ++e) part[h * C + e][t] = x[h][e];
    __syncthreads();
    if (group > 0) return;
    for (int g = 1; g < min(count, groups); ++g)
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int e = 0; e < C; ++e) x[h][e] += part[h * C + e][(g << wide_log2) + t];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        float f[C];
        if (ACCUMULATE) old[h].v.get(f);
#pragma unroll
        for (int e = 0; e < C; ++e) f[e] = ACCUMULATE ? f[e] + scale * x[h][e] : scale * x[h][e];
        old[h].v.set(f);
        old[h].template store<false>(o, cols[h]);
    }
}

#define RLHF_TYPES2(A, B, CALL)                                                        \
    do {                                                                               \
        if (A == kBF16) { using X = bf16_t; RLHF_TYPES1(B, CALL) }                     \
        else if (A == kF16) { using X = f16_t; RLHF_TYPES1(B, CALL) }                  \
        else { using X = float; RLHF_TYPES1(B, CALL) }                                 \
    } while (0)
#define RLHF_TYPES1(B, CALL)                                                           \
    if (B == kBF16) { using Y = bf16_t; CALL; }                                        \
    else if (B == kF16) { using Y = f16_t; CALL; }                                     \
    else { using Y = float; CALL; }

template <typename T, typename O>
static void embed_rows(hipStream_t st, const T* table, size_t ld_table, const int* tokens, float scale, O* out, size_t ld_out, int rows, int d,
                       int vocab) {
    const Grid g = grid_of(out, ld_out, d, Shape<T, O>::C, Shape<T, O>::H);
    const int per = 256 >> g.wide_log2;
    const int64_t most = kLaunchThreads / 256 * per;
    for (int64_t first = 0; first < rows; first += most) {
        const int part = (int)std::min<int64_t>(most, rows - first);
        k_embed_rows<T, O><<<dim3((part + per - 1) / per, g.slices), 256, 0, st>>>(table, ld_table, tokens + first, out + first * ld_out, ld_out, scale,
                                                                                  part, d, vocab, g.wide_log2);
    }
}

hipError_t launch_embed_rows(hipStream_t st, int tdt, int odt, const void* table, size_t ld_table, const int* tokens, float scale,
                             void* out, size_t ld_out, int rows, int d, int vocab) {
    if (rows <= 0) return hipSuccess;
    if (!sizes_fit(rows, d, vocab)) return hipErrorInvalidValue;
    RLHF_TYPES2(tdt, odt, (embed_rows(st, (const X*)table, ld_table, tokens, scale, (Y*)out, ld_out, rows, d, vocab)));
    return hipGetLastError();
}

// Places of the order a chunk has: summing a chunk and joining the chunks of the longest run then take about as long.
static int chunk_size(int n) {
    int c = 32;
    while ((int64_t)c * c * 64 < n) c *= 2;
    return c;
}
struct GradScratch { size_t runs, places, total, part, bytes; };
static GradScratch grad_scratch(int rows, int d, int vocab) {
    const auto up = [](size_t x) { return (x + 15) / 16 * 16; };
    const Buckets b = buckets_of(vocab);
    const int size = chunk_size(rows);
    GradScratch s;
    s.runs = 0;
    s.places = up(((size_t)b.subs << b.log2) * sizeof(Run));
    s.total = s.places + (size_t)rows * sizeof(Place);
    s.part = s.total + 16;
    s.bytes = s.part + (size_t)((rows + size - 1) / size) * 2 * up((size_t)d * sizeof(float));
    return s;
}
size_t embed_grad_scratch_bytes(int rows, int d, int vocab) { return few_rows(rows, d) ? 0 : grad_scratch(rows, d, vocab).bytes; }

// Rows of the table that are cleared beside the grouping: 32 MB, 5 us of stores by themselves (8192 tokens: the grouping alone
// 8.8 us, with the zeros 11.3).
static int rows_cleared_first(size_t row_bytes, int rows, int vocab) {
    const size_t first = (32u << 20) / row_bytes;
    return rows > 0 && first < (size_t)vocab ? (int)first : vocab;
}

// The table's first rows, all to be cleared.  Rows behind each other in memory are cleared as rows of 4 KB, whatever their length
// (41617 rows of 51 bf16: 8.5 us by rows).
template <typename T> static Clear first_rows(const T* dtable, size_t ld, int d, int rows) {
    constexpr int L = 4096 / sizeof(T);
    const size_t elements = (size_t)rows * d, lines = (elements + L - 1) / L;
    const bool flat = ld == (size_t)d && lines <= 1 << 30;
    const Grid g = flat ? grid_of(dtable, L, L, 16 / sizeof(T), 1) : grid_of(dtable, ld, d, 16 / sizeof(T), 1);
    if (flat) return Clear{0, (int)lines, g.wide_log2, g.slices, L, L, elements};
    return Clear{0, rows, g.wide_log2, g.slices, d, ld, 0};
}

template <typename G, typename T, bool ACCUMULATE>
static hipError_t embed_grad(hipStream_t st, const G* dout, T* dtable, const int* tokens, GradArgs a, Place* places, Run* runs, int* total, int rows,
                             int vocab) {
    const int first = ACCUMULATE ? 0 : rows_cleared_first(a.d * sizeof(T), rows, vocab);
    if (rows > 0 && few_rows(rows, a.d)) {
        if (!ACCUMULATE) {
            const Clear whole = first_rows(dtable, a.ld_table, a.d, vocab);
            if (clear_blocks<1024>(whole) > kLaunchThreads / 1024) return hipErrorInvalidValue;
            k_group_and_clear<T><<<(unsigned)clear_blocks<1024>(whole), 1024, 0, st>>>(tokens, 0, vocab, a.b, places, runs, total, dtable, whole);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        const Grid g = grid_of((const T*)nullptr, 0, a.d, Shape<G, T>::C, Shape<G, T>::H, 6);
        k_few_rows_grad<G, T, ACCUMULATE><<<dim3(rows, g.slices), 256, 0, st>>>(dout, a.ld_dout, tokens, dtable, a.ld_table, a.scale, rows, a.d, vocab,
                                                                              g.wide_log2);
        return hipGetLastError();
    }
    const Clear beside = first_rows(dtable, a.ld_table, a.d, first);
    const Grid z = grid_of(dtable, a.ld_table, a.d, 16 / sizeof(T), 1);
    a.clear = Clear{first, ACCUMULATE ? first : vocab, z.wide_log2, z.slices, a.d, a.ld_table, 0};
    const int64_t group_blocks = (rows > 0 ? (int64_t)a.b.parts << a.b.log2 : 0) + clear_blocks<1024>(beside), clear = clear_blocks<256>(a.clear);
    const Grid g = grid_of((const T*)nullptr, 0, a.d, Shape<G, T>::C, Shape<G, T>::H);     // its pieces go by columns
    a.wide_log2 = g.wide_log2;
    a.slices = g.slices;
    const int64_t per = 256 >> g.wide_log2;
    // up to eight places (a place where no run begins costs little then), fewer where they would not fill the chip
    a.window = rows >= 8192 ? 8 : rows >= 1024 ? rows / 1024 : 1;
    const int64_t windows = (rows + a.window * per - 1) / (a.window * per);
    const int64_t table = ((a.c.count + per - 1) / per + (windows + 7) / 8 * 8) * g.slices;
    if (group_blocks > kLaunchThreads / 1024 || table + clear > kLaunchThreads / 256) return hipErrorInvalidValue;
    k_group_and_clear<T><<<(unsigned)group_blocks, 1024, group_lds_bytes(a.b), st>>>(tokens, rows, vocab, a.b, places, runs, total, dtable,
                                                                                    beside);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || rows <= 0) return e;
    a.table_blocks = (unsigned)table;
    a.clear_blocks = (unsigned)clear;
    k_table_grad<G, T, ACCUMULATE><<<(unsigned)(table + clear), 256, 0, st>>>(dout, dtable, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int groups = 1 << a.b.log2;
    if (a.d <= 1024) k_long_runs<T, ACCUMULATE, 16><<<dim3(groups, (a.d + 63) / 64), kJoinThreads, 0, st>>>(dtable, a);
    else k_long_runs<T, ACCUMULATE, 64><<<dim3(groups, (a.d + 255) / 256), kJoinThreads, 0, st>>>(dtable, a);
    return hipGetLastError();
}

hipError_t launch_embed_grad(hipStream_t st, int gdt, int tdt, const void* dout, size_t ld_dout, const int* tokens, float scale,
                             bool accumulate, void* dtable, size_t ld_table, void* scratch, int rows, int d, int vocab) {
    if (accumulate && rows <= 0) return hipSuccess;
    if (!sizes_fit(rows, d, vocab)) return hipErrorInvalidValue;
    const GradScratch g = grad_scratch(rows, d, vocab);
    Place* places = (Place*)((char*)scratch + g.places);
    int* total = (int*)((char*)scratch + g.total);
    Run* runs = (Run*)((char*)scratch + g.runs);
    GradArgs a;
    a.places = places; a.total = total; a.runs = runs;
    a.b = buckets_of(vocab);
    a.c = Chunks{(float*)((char*)scratch + g.part), ((size_t)d + 3) / 4 * 4, chunk_size(rows), 0};
    a.c.count = (rows + a.c.size - 1) / a.c.size;
    a.ld_dout = ld_dout; a.ld_table = ld_table; a.scale = scale; a.rows = rows; a.d = d;
    hipError_t e = hipSuccess;
    RLHF_TYPES2(gdt, tdt, (e = accumulate ? embed_grad<X, Y, true>(st, (const X*)dout, (Y*)dtable, tokens, a, places, runs, total, rows, vocab)
                                          : embed_grad<X, Y, false>(st, (const X*)dout, (Y*)dtable, tokens, a, places, runs, total, rows, vocab)));
    return e;
}

}  // namespace rlhf
