// Embedding lookup with scaling, and the gradient of its table.  Both are memory-bound: rows go through registers once.
#include "common.h"
#include "kernels.h"
#include "vec.h"

namespace rlhf {

// How threads lie over rows of d columns: a thread has eight columns of a row at a time, `wide` threads (a power of two, at most
// 256) lie side by side and 256 / wide rows share a workgroup; grid.y covers what is wider than 2048 columns.
struct RowShape { int wide_log2, slices; };
static RowShape row_shape(int d) {
    const int pieces = (d + 7 + 7) / 8;                  // a row that starts off a boundary has one more
    int lg = 3;
    while (lg < 8 && (1 << lg) < pieces) ++lg;
    return RowShape{lg, (pieces + (1 << lg) - 1) >> lg};
}
// Row and column numbers are ints.
static bool sizes_fit(int rows, int d, int vocab, const RowShape& s) { return rows <= 1 << 30 && d <= 1 << 30 && vocab <= 1 << 30 && s.slices <= 65535; }

// Columns [lo, hi) of piece c of a row at p: pieces meet where p + column reaches a 16-byte boundary.
template <typename T> __device__ __forceinline__ void piece_columns(const T* p, int c, int d, int& lo, int& hi) {
    const int shift = (int)((uintptr_t)p % 16 / sizeof(T));
    hi = min(d, c * 8 - shift + 8);
    lo = max(0, c * 8 - shift);
}

// The same columns of another row: eight at once, or the few there are.
template <bool ONCE, typename T> __device__ __forceinline__ void load_piece(const T* row, int lo, int hi, float (&x)[8]) {
    if (hi - lo == 8) return load8_any<ONCE, T>(row + lo, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = lo + e < hi ? to_f32<T>(row[lo + e]) : 0.f;
}
template <bool ONCE, typename T> __device__ __forceinline__ void store_piece(T* row, int lo, int hi, const float (&x)[8]) {
    if (hi - lo == 8) return store8_any<ONCE, T>(row + lo, x);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (lo + e < hi) row[lo + e] = from_f32<T>(x[e]);
}

template <typename T, typename O>
__global__ __launch_bounds__(256) void k_embed_rows(const T* __restrict__ table, size_t ld_table, const int* __restrict__ tokens,
                                                    O* __restrict__ out, size_t ld_out, float scale, int rows, int d, int vocab, int wide_log2) {
    const int r = blockIdx.x * (256 >> wide_log2) + (threadIdx.x >> wide_log2);
    if (r >= rows) return;
    const int v = tokens[r];
    O* o = out + (size_t)r * ld_out;
    int lo, hi;
    piece_columns(o, (blockIdx.y << wide_log2) + (threadIdx.x & ((1 << wide_log2) - 1)), d, lo, hi);
    if (lo >= hi) return;
    float x[8];
    if ((unsigned)v < (unsigned)vocab) {
        load_piece<false>(table + (size_t)v * ld_table, lo, hi, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= scale;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = v < 0 ? 0.f : NAN;
    }
    store_piece<false>(o, lo, hi, x);
}

// ---- gradient: rows grouped by token, then every token's rows summed in ascending order.
// The vocabulary is dealt to 2^log2 buckets by its low bits (frequent tokens have neighbouring ids), `subs` tokens each.  A
// workgroup per bucket looks through all tokens twice: the first time it counts its own, per wave (a wave has one contiguous share
// of the rows), and how many lie in earlier buckets; the second time each wave puts its rows behind those of the waves before
// it.  No sort passes over memory, no atomics whose order could show: 256 workgroups read the tokens out of the L2.
struct Buckets { int log2, subs; };
constexpr int kMaxSubs = 512;
static Buckets buckets_of(int vocab) {
    int lg = 8;
    while (((int64_t)vocab + (1ll << lg) - 1) >> lg > kMaxSubs) ++lg;
    return Buckets{lg, (int)(((int64_t)vocab + (1ll << lg) - 1) >> lg)};
}
struct Run { int start, count; };       // a token's rows: order[start .. start + count)

constexpr int kAhead = 8;               // tokens a lane has in flight
__device__ __forceinline__ void load_tokens(const int* tokens, int i, int end, int (&v)[kAhead]) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) v[j] = i + j * 64 < end ? tokens[i + j * 64] : -1;
}

__global__ __launch_bounds__(1024) void k_group_tokens(const int* __restrict__ tokens, int n, int vocab, Buckets b, int* __restrict__ order,
                                                       Run* __restrict__ runs, int* __restrict__ total) {
    extern __shared__ int next[];       // [16 waves][subs]
    __shared__ int s_part[16], s_before[16];
    const int t = threadIdx.x, w = t >> 6, lane = t & 63, mine = blockIdx.x, mask = (1 << b.log2) - 1;
    for (int i = t; i < 16 * b.subs; i += 1024) next[i] = 0;
    __syncthreads();
    const int share = ((n + 1023) >> 10) << 6;                     // rows of a wave
    const int first = min(n, w * share), end = min(n, first + share);
    int before = 0;
    for (int i0 = first; i0 < end; i0 += 64 * kAhead) {
        int v[kAhead];
        load_tokens(tokens, i0 + lane, end, v);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if ((unsigned)v[j] >= (unsigned)vocab) continue;
            const int k = v[j] & mask;
            if (k < mine) ++before;
            if (k == mine) atomicAdd(&next[w * b.subs + (v[j] >> b.log2)], 1);
        }
    }
    for (int o = 32; o > 0; o >>= 1) before += __shfl_xor(before, o, kWave);
    if (lane == 0) s_before[w] = before;
    __syncthreads();
    int base = 0, count = 0;
    for (int i = 0; i < 16; ++i) base += s_before[i];
    if (t < b.subs)
        for (int i = 0; i < 16; ++i) count += next[i * b.subs + t];
    int sum = count;                                               // inclusive over the tokens of the bucket
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(sum, o, kWave);
        if (lane >= o) sum += x;
    }
    if (lane == 63) s_part[w] = sum;
    __syncthreads();
    for (int i = 0; i < w; ++i) sum += s_part[i];
    int start = base + sum - count;
    if (t < b.subs) {
        runs[(size_t)mine * b.subs + t] = Run{start, count};
        for (int i = 0; i < 16; ++i) {
            const int c = next[i * b.subs + t];
            next[i * b.subs + t] = start;
            start += c;
        }
    }
    if (mine == mask && t == 1023) *total = base + sum;
    __syncthreads();
    for (int i0 = first; i0 < end; i0 += 64 * kAhead) {
        int v[kAhead];
        load_tokens(tokens, i0 + lane, end, v);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int sub = v[j] >> b.log2;
            bool left = (unsigned)v[j] < (unsigned)vocab && (v[j] & mask) == mine;
            for (uint64_t m = __ballot(left); m; m = __ballot(left)) {     // one token of the 64 rows at a time
                const int leader = __ffsll((unsigned long long)m) - 1;
                const bool same = left && sub == __shfl(sub, leader, kWave);
                const uint64_t all = __ballot(same);
                int at = 0;
                if (lane == leader) at = atomicAdd(&next[w * b.subs + sub], __popcll(all));
                at = __shfl(at, leader, kWave);
                if (same) order[at + __popcll(all & ((1ull << lane) - 1))] = i0 + j * 64 + lane;
                left = left && !same;
            }
        }
    }
}

// Rows [p, end) of the order, summed into x in that order; four rows in flight.
template <typename G>
__device__ __forceinline__ void sum_rows(const G* __restrict__ dout, size_t ld, const int* __restrict__ order, int p, int end, int lo, int hi,
                                         float (&x)[8]) {
    for (; p + 4 <= end; p += 4) {
        float y[4][8];
#pragma unroll
        for (int k = 0; k < 4; ++k) load_piece<true>(dout + (size_t)order[p + k] * ld, lo, hi, y[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += y[k][e];
    }
    for (; p < end; ++p) {
        float y[8];
        load_piece<true>(dout + (size_t)order[p] * ld, lo, hi, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += y[e];
    }
}

__device__ __forceinline__ Run run_of(const Run* runs, const Buckets& b, int v) {
    return runs[(size_t)(v & ((1 << b.log2) - 1)) * b.subs + (v >> b.log2)];
}

// A frequent token's run is cut into pieces of `chunk` places of the order, summed by workgroups of their own; a run of at most
// two chunks is not.
template <typename G>
__global__ __launch_bounds__(256) void k_run_chunks(const G* __restrict__ dout, size_t ld, const int* __restrict__ tokens,
                                                    const int* __restrict__ order, const int* __restrict__ total, const Run* __restrict__ runs,
                                                    Buckets b, float* __restrict__ part, size_t ld_part, int chunk, int d, int wide_log2) {
    const int k = blockIdx.x * (256 >> wide_log2) + (threadIdx.x >> wide_log2);
    const int64_t p = (int64_t)k * chunk;
    if (p + chunk > *total) return;
    const int v = tokens[order[p]];
    const Run run = run_of(runs, b, v);
    if (run.count <= 2 * chunk || p + chunk > (int64_t)run.start + run.count) return;
    const int lo = ((blockIdx.y << wide_log2) + (threadIdx.x & ((1 << wide_log2) - 1))) * 8, hi = min(d, lo + 8);
    if (lo >= hi) return;
    float x[8] = {};
    sum_rows(dout, ld, order, (int)p, (int)p + chunk, lo, hi, x);
    store_piece<false>(part + (size_t)k * ld_part, lo, hi, x);
}

// Rows of the table: all of them, or (accumulate) those whose token's first place in the order is the thread's.
template <typename G, typename T>
__global__ __launch_bounds__(256) void k_table_grad(const G* __restrict__ dout, size_t ld, const int* __restrict__ tokens,
                                                    const int* __restrict__ order, const int* __restrict__ total, const Run* __restrict__ runs,
                                                    Buckets b, const float* __restrict__ part, size_t ld_part, int chunk, T* __restrict__ dtable,
                                                    size_t ld_table, float scale, int accumulate, int n, int d, int vocab, int wide_log2) {
    const int i = blockIdx.x * (256 >> wide_log2) + (threadIdx.x >> wide_log2);
    int v = i;
    if (accumulate) {
        if (i >= *total) return;
        v = tokens[order[i]];
    }
    if (v >= vocab) return;
    const Run run = n > 0 ? run_of(runs, b, v) : Run{0, 0};
    if (accumulate && run.start != i) return;
    T* o = dtable + (size_t)v * ld_table;
    int lo, hi;
    piece_columns(o, (blockIdx.y << wide_log2) + (threadIdx.x & ((1 << wide_log2) - 1)), d, lo, hi);
    if (lo >= hi) return;
    float x[8] = {};
    const int end = run.start + run.count;
    if (run.count <= 2 * chunk) {
        sum_rows(dout, ld, order, run.start, end, lo, hi, x);
    } else {                                            // the rows before the first whole chunk, the chunks, the rest
        const int c0 = (run.start + chunk - 1) / chunk, c1 = end / chunk;
        sum_rows(dout, ld, order, run.start, c0 * chunk, lo, hi, x);
        for (int c = c0; c < c1; ++c) {
            float y[8];
            load_piece<false>(part + (size_t)c * ld_part, lo, hi, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += y[e];
        }
        sum_rows(dout, ld, order, c1 * chunk, end, lo, hi, x);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= scale;
    if (accumulate) {
        float y[8];
        load_piece<false>(o, lo, hi, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += y[e];
    }
    store_piece<false>(o, lo, hi, x);
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

hipError_t launch_embed_rows(hipStream_t st, int tdt, int odt, const void* table, size_t ld_table, const int* tokens, float scale,
                             void* out, size_t ld_out, int rows, int d, int vocab) {
    if (rows <= 0) return hipSuccess;
    const RowShape s = row_shape(d);
    if (!sizes_fit(rows, d, vocab, s)) return hipErrorInvalidValue;
    const int per = 256 >> s.wide_log2;
    const dim3 grid((rows + per - 1) / per, s.slices);
    RLHF_TYPES2(tdt, odt, (k_embed_rows<X, Y><<<grid, 256, 0, st>>>((const X*)table, ld_table, tokens, (Y*)out, ld_out, scale, rows, d, vocab,
                                                                    s.wide_log2)));
    return hipGetLastError();
}

// Places of the order a chunk has: a long run is then about as many chunks as a chunk has rows.
static int run_chunk(int n) {
    int c = 64;
    while ((int64_t)c * c < n / 2) c *= 2;
    return c;
}
struct GradScratch { size_t runs, order, total, part, bytes; };
static GradScratch grad_scratch(int rows, int d, int vocab) {
    const auto up = [](size_t x) { return (x + 15) / 16 * 16; };
    const Buckets b = buckets_of(vocab);
    const int chunk = run_chunk(rows);
    GradScratch s;
    s.runs = 0;
    s.order = up(((size_t)b.subs << b.log2) * sizeof(Run));
    s.total = s.order + up((size_t)rows * sizeof(int));
    s.part = s.total + 16;
    s.bytes = s.part + (rows > 2 * chunk ? (size_t)(rows / chunk) * up((size_t)d * sizeof(float)) : 0);
    return s;
}
size_t embed_grad_scratch_bytes(int rows, int d, int vocab) { return grad_scratch(rows, d, vocab).bytes; }

hipError_t launch_embed_grad(hipStream_t st, int gdt, int tdt, const void* dout, size_t ld_dout, const int* tokens, float scale,
                             bool accumulate, void* dtable, size_t ld_table, void* scratch, int rows, int d, int vocab) {
    if (accumulate && rows <= 0) return hipSuccess;
    const RowShape s = row_shape(d);
    if (!sizes_fit(rows, d, vocab, s)) return hipErrorInvalidValue;
    const int per = 256 >> s.wide_log2, chunk = run_chunk(rows);
    const GradScratch g = grad_scratch(rows, d, vocab);
    const Buckets b = buckets_of(vocab);
    Run* runs = (Run*)((char*)scratch + g.runs);
    int* order = (int*)((char*)scratch + g.order);
    int* total = (int*)((char*)scratch + g.total);
    float* part = (float*)((char*)scratch + g.part);
    const size_t ld_part = ((size_t)d + 3) / 4 * 4;
    hipError_t e = hipSuccess;
    if (rows > 0) {
        k_group_tokens<<<1 << b.log2, 1024, 16 * b.subs * sizeof(int), st>>>(tokens, rows, vocab, b, order, runs, total);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if (rows > 2 * chunk) {
            const dim3 grid((rows / chunk + per - 1) / per, s.slices);
            if (gdt == kBF16) k_run_chunks<bf16_t><<<grid, 256, 0, st>>>((const bf16_t*)dout, ld_dout, tokens, order, total, runs, b, part, ld_part, chunk, d, s.wide_log2);
            else if (gdt == kF16) k_run_chunks<f16_t><<<grid, 256, 0, st>>>((const f16_t*)dout, ld_dout, tokens, order, total, runs, b, part, ld_part, chunk, d, s.wide_log2);
            else k_run_chunks<float><<<grid, 256, 0, st>>>((const float*)dout, ld_dout, tokens, order, total, runs, b, part, ld_part, chunk, d, s.wide_log2);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    const dim3 grid(((accumulate ? rows : vocab) + per - 1) / per, s.slices);
    RLHF_TYPES2(gdt, tdt, (k_table_grad<X, Y><<<grid, 256, 0, st>>>((const X*)dout, ld_dout, tokens, order, total, runs, b, part, ld_part, chunk,
                                                                    (Y*)dtable, ld_table, scale, accumulate, rows, d, vocab, s.wide_log2)));
    return hipGetLastError();
}

}  // namespace rlhf
