// Global 2-norm of many gradients, and their scaling by it.
#include "common.h"
#include "kernels.h"

namespace rlhf {

constexpr int kNormBlocks = 256;

__device__ __forceinline__ double block_sum_double(double v, double* red) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double t = 0.;
    for (int i = 0; i < (int)blockDim.x >> 6; ++i) t += red[i];
    return t;
}

template <typename T>
__global__ __launch_bounds__(256) void k_sum_squares(const T* __restrict__ x, size_t n, double* __restrict__ part) {
    __shared__ double red[4];
    double s = 0.;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
        const double v = to_f32<T>(x[i]);
        s += v * v;
    }
    s = block_sum_double(s, red);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(256) void k_norm_finish(const double* __restrict__ part, int n, float* __restrict__ norm) {
    __shared__ double red[4];
    double s = 0.;
    for (int i = threadIdx.x; i < n; i += 256) s += part[i];
    s = block_sum_double(s, red);
    if (threadIdx.x == 0) norm[0] = (float)sqrt(s);
}

__device__ __forceinline__ float clip_factor(float norm, float max_norm) {
    return norm > max_norm && norm < INFINITY ? max_norm / norm : 1.f;
}

template <typename T>
__global__ __launch_bounds__(256) void k_scale(const T* x, T* y, size_t n, const float* __restrict__ norm, float max_norm) {
    const float f = clip_factor(norm[0], max_norm);
    if (f == 1.f) {
        if (x != y) for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) y[i] = x[i];
        return;
    }
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) y[i] = from_f32<T>(f * to_f32<T>(x[i]));
}

size_t grad_norm_scratch_doubles(const GradTensor* t, int n) { return (size_t)n * kNormBlocks; }

hipError_t launch_grad_norm(hipStream_t st, const GradTensor* t, int n, float* norm, double* scratch) {
    for (int i = 0; i < n; ++i) {
        double* p = scratch + (size_t)i * kNormBlocks;
        if (t[i].dtype == kBF16) k_sum_squares<bf16_t><<<kNormBlocks, 256, 0, st>>>((const bf16_t*)t[i].src, t[i].n, p);
        else if (t[i].dtype == kF16) k_sum_squares<f16_t><<<kNormBlocks, 256, 0, st>>>((const f16_t*)t[i].src, t[i].n, p);
        else k_sum_squares<float><<<kNormBlocks, 256, 0, st>>>((const float*)t[i].src, t[i].n, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    k_norm_finish<<<1, 256, 0, st>>>(scratch, n * kNormBlocks, norm);
    return hipGetLastError();
}

hipError_t launch_clip_grads(hipStream_t st, const GradTensor* t, int n, const float* norm, float max_norm) {
    for (int i = 0; i < n; ++i) {
        if (t[i].dtype == kBF16) k_scale<bf16_t><<<1024, 256, 0, st>>>((const bf16_t*)t[i].src, (bf16_t*)t[i].dst, t[i].n, norm, max_norm);
        else if (t[i].dtype == kF16) k_scale<f16_t><<<1024, 256, 0, st>>>((const f16_t*)t[i].src, (f16_t*)t[i].dst, t[i].n, norm, max_norm);
        else k_scale<float><<<1024, 256, 0, st>>>((const float*)t[i].src, (float*)t[i].dst, t[i].n, norm, max_norm);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace rlhf
