// Global 2-norm of many gradients, and their scaling by it.  Both are a stream over memory, 2.1 GB of bf16 in 27 tensors 369 us =
// 5.8 TB/s and 800 us = 5.4 TB/s; what matters beside is that a model of hundreds of small tensors is not hundreds of launches
// (600 tensors of 700 floats: 18 and 16 us).  The factor is known only when all has been read, so gradients are read twice.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "vec.h"

namespace rlhf {

// Tensors travel as kernel arguments, kPackTensors to a launch: nothing has to be copied to the device first, and a captured graph
// holds all it needs.  Each is cut into chunks of vectors of 16 bytes, a workgroup a chunk.
constexpr int kPackTensors = 128;
struct PackTensor {
    const void* src;
    void* dst;
    // elements, the tensor's first chunk (at most 16384 of vectors_of and one more a tensor), type: 24 bytes in all, 3 KB a launch
    uint64_t n : 40, first : 22, dtype : 2;
};
struct Pack {
    PackTensor t[kPackTensors];
    int tensors, chunks, vectors;        // vectors: of a chunk
};

// Chunk c of the pack: its tensor, and the vectors [from, to) of it.  `head` elements come before the first vector, which begins where p
// reaches a 16-byte boundary; they and the few behind the last vector go to the tensor's first chunk, a thread each (odd < n).
struct Work { int i; size_t from, to, odd; int head; };
template <typename T, bool DST> __device__ __forceinline__ Work work_of(const Pack& pk, int i, int c) {
    constexpr int N = 16 / sizeof(T);
    const PackTensor& t = pk.t[i];
    const uintptr_t p = (uintptr_t)(DST ? t.dst : t.src);
    const int head = (int)min((size_t)((0 - p) % 16 / sizeof(T)), (size_t)t.n);
    const size_t all = (t.n - head) / N, from = (size_t)(c - (int)t.first) * pk.vectors, whole = all * N;
    Work w{i, from, min(all, from + pk.vectors), t.n, head};
    if (c == (int)t.first) w.odd = (int)threadIdx.x < head ? threadIdx.x : threadIdx.x + whole;
    return w;
}
__device__ __forceinline__ int tensor_of(const Pack& pk, int c) {
    int lo = 0, hi = pk.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if ((int)pk.t[mid].first <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ double block_sum_double(double v, double* red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double t = 0.;
    for (int i = 0; i < (int)blockDim.x >> 6; ++i) t += red[i];
    return t;
}

// Squares are summed in double: a float's square fits, whatever the float, and the two instructions an element are hidden behind
// the loads.
constexpr int kUnroll = 4;
template <typename T>
__device__ __forceinline__ double sum_squares(const Pack& pk, int i, int c) {
    constexpr int N = 16 / sizeof(T);
    const Work w = work_of<T, false>(pk, i, c);
    const T* x = (const T*)pk.t[i].src;
    double s = 0.;
    if (w.odd < pk.t[i].n) {
        const double v = to_f32<T>(x[w.odd]);
        s = v * v;
    }
    x += w.head;
    for (size_t k0 = w.from + threadIdx.x; k0 < w.to; k0 += 256 * kUnroll) {
        Vec<T> v[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (k0 + u * 256 < w.to) v[u].template load<false>(x + (k0 + u * 256) * N);
            else v[u].fill(0.f);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float f[N];
            v[u].get(f);
#pragma unroll
            for (int e = 0; e < N; ++e) s += (double)f[e] * (double)f[e];
        }
    }
    return s;
}

__global__ __launch_bounds__(256) void k_sum_squares(Pack pk, double* __restrict__ part) {
    __shared__ double red[4];
    const int c = blockIdx.x, i = tensor_of(pk, c), dt = pk.t[i].dtype;
    double s = dt == kBF16 ? sum_squares<bf16_t>(pk, i, c) : dt == kF16 ? sum_squares<f16_t>(pk, i, c) : sum_squares<float>(pk, i, c);
    s = block_sum_double(s, red);
    if (threadIdx.x == 0) part[c] = s;
}

__global__ __launch_bounds__(1024) void k_norm_finish(const double* __restrict__ part, int n, float* __restrict__ norm) {
    __shared__ double red[16];
    double s = 0.;
    for (int i = threadIdx.x; i < n; i += 1024 * 8) {
        double v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = i + k * 1024 < n ? part[i + k * 1024] : 0.;
#pragma unroll
        for (int k = 0; k < 8; ++k) s += v[k];
    }
    s = block_sum_double(s, red);
    if (threadIdx.x == 0) norm[0] = (float)sqrt(s);
}

template <typename T>
__device__ __forceinline__ void scale_chunk(const Pack& pk, int i, int c, float f) {
    constexpr int N = 16 / sizeof(T);
    const Work w = work_of<T, true>(pk, i, c);
    const T* x = (const T*)pk.t[i].src;
    T* y = (T*)pk.t[i].dst;
    if (w.odd < pk.t[i].n) y[w.odd] = round_to<T>(f * to_f32<T>(x[w.odd]));
    x += w.head;
    y += w.head;
    for (size_t k0 = w.from + threadIdx.x; k0 < w.to; k0 += 256 * kUnroll) {
        Vec<T> v[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (k0 + u * 256 < w.to) v[u].template load<true>(x + (k0 + u * 256) * N);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (k0 + u * 256 >= w.to) break;
            float a[N];
            v[u].get(a);
#pragma unroll
            for (int e = 0; e < N; ++e) a[e] *= f;
            v[u].set(a);
            v[u].template store<true>(y + (k0 + u * 256) * N);
        }
    }
}

// From the last chunk to the first: what the norm read last is still in the memory-side cache.
__global__ __launch_bounds__(256) void k_clip(Pack pk, const float* __restrict__ norm, float max_norm) {
    const int c = pk.chunks - 1 - blockIdx.x, i = tensor_of(pk, c), dt = pk.t[i].dtype;
    const float g = norm[0], f = g > max_norm && g < INFINITY ? max_norm / g : 1.f;
    if (f == 1.f && pk.t[i].src == pk.t[i].dst) return;
    if (dt == kBF16) scale_chunk<bf16_t>(pk, i, c, f);
    else if (dt == kF16) scale_chunk<f16_t>(pk, i, c, f);
    else scale_chunk<float>(pk, i, c, f);
}

// Vectors of a chunk: 16 KB, one round trip of a workgroup's threads, up to 32 MB; then up to 64 KB; more where that would be over
// 16384 chunks.
static size_t vectors_of(const GradTensor* t, int n) {
    size_t all = 0;
    for (int i = 0; i < n; ++i) all += t[i].n * (t[i].dtype == kF32 ? 4 : 2) / 16;
    const auto up = [](size_t x) { return std::max<size_t>(1, (x + 1023) / 1024) * 1024; };
    return std::max(std::min<size_t>(4096, up(all / 2048)), up(all / 16384));
}
static size_t chunks_of(const GradTensor& t, size_t vectors) {
    const size_t all = t.n * (t.dtype == kF32 ? 4 : 2) / 16;
    return std::max<size_t>(1, (all + vectors - 1) / vectors);
}

size_t grad_norm_scratch_doubles(const GradTensor* t, int n) {
    const size_t vectors = vectors_of(t, n);
    size_t c = 0;
    for (int i = 0; i < n; ++i) c += chunks_of(t[i], vectors);
    return c;
}

// launch(pack, chunks before it) for every pack of the list, from the front or from the back.
template <typename Launch>
static hipError_t each_pack(const GradTensor* t, int n, bool backwards, Launch launch) {
    const size_t vectors = vectors_of(t, n);
    const int packs = (n + kPackTensors - 1) / kPackTensors;
    if (vectors > 1 << 30) return hipErrorInvalidValue;
    size_t before = 0;
    for (int k = 0; k < packs; ++k) {
        const int at = (backwards ? packs - 1 - k : k) * kPackTensors;
        Pack pk;
        pk.tensors = std::min(kPackTensors, n - at);
        pk.vectors = (int)vectors;
        size_t chunks = 0;
        for (int i = 0; i < pk.tensors; ++i) {
            const GradTensor& g = t[at + i];
            pk.t[i] = PackTensor{g.src, g.dst, g.n, chunks, (uint64_t)g.dtype};
            chunks += chunks_of(g, vectors);
        }
        pk.chunks = (int)chunks;
        const hipError_t e = launch(pk, before);
        if (e != hipSuccess) return e;
        before += chunks;
    }
    return hipSuccess;
}

hipError_t launch_grad_norm(hipStream_t st, const GradTensor* t, int n, float* norm, double* scratch) {
    size_t all = 0;
    hipError_t e = each_pack(t, n, false, [&](const Pack& pk, size_t before) {
        k_sum_squares<<<pk.chunks, 256, 0, st>>>(pk, scratch + before);
        all = before + pk.chunks;
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    if (all > INT32_MAX) return hipErrorInvalidValue;
    k_norm_finish<<<1, 1024, 0, st>>>(scratch, (int)all, norm);
    return hipGetLastError();
}

hipError_t launch_clip_grads(hipStream_t st, const GradTensor* t, int n, const float* norm, float max_norm) {
    return each_pack(t, n, true, [&](const Pack& pk, size_t) {
        k_clip<<<pk.chunks, 256, 0, st>>>(pk, norm, max_norm);
        return hipGetLastError();
    });
}

}  // namespace rlhf
