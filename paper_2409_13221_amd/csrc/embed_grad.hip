// Embedding lookup with scaling and the gradient of its table.
#include "common.h"
#include "kernels.h"

namespace rlhf {

template <typename T, typename O>
__global__ __launch_bounds__(256) void k_embed_rows(const T* __restrict__ table, size_t ld_table, const int* __restrict__ tokens,
                                                    float scale, O* __restrict__ out, size_t ld_out, int d, int vocab) {
    const int r = blockIdx.x, v = tokens[r];
    for (int i = threadIdx.x; i < d; i += 256)
        out[(size_t)r * ld_out + i] = from_f32<O>(v < 0 ? 0.f : v >= vocab ? NAN : scale * to_f32<T>(table[(size_t)v * ld_table + i]));
}

// One workgroup per row of the table: it looks through all tokens for its own.
template <typename G, typename T>
__global__ __launch_bounds__(256) void k_embed_grad(const G* __restrict__ dout, size_t ld_dout, const int* __restrict__ tokens,
                                                    float scale, int accumulate, T* __restrict__ dtable, size_t ld_table, int rows, int d) {
    const int v = blockIdx.x;
    for (int i = threadIdx.x; i < d; i += 256) {
        float s = 0.f;
        bool any = false;
        for (int r = 0; r < rows; ++r)
            if (tokens[r] == v) { s += to_f32<G>(dout[(size_t)r * ld_dout + i]); any = true; }
        T* o = dtable + (size_t)v * ld_table + i;
        if (!accumulate) *o = from_f32<T>(scale * s);
        else if (any) *o = from_f32<T>(to_f32<T>(*o) + scale * s);
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

hipError_t launch_embed_rows(hipStream_t st, int tdt, int odt, const void* table, size_t ld_table, const int* tokens, float scale,
                             void* out, size_t ld_out, int rows, int d, int vocab) {
    if (rows <= 0) return hipSuccess;
    RLHF_TYPES2(tdt, odt, (k_embed_rows<X, Y><<<rows, 256, 0, st>>>((const X*)table, ld_table, tokens, scale, (Y*)out, ld_out, d, vocab)));
    return hipGetLastError();
}

size_t embed_grad_scratch_bytes(int rows, int d, int vocab) { return 16; }

hipError_t launch_embed_grad(hipStream_t st, int gdt, int tdt, const void* dout, size_t ld_dout, const int* tokens, float scale,
                             bool accumulate, void* dtable, size_t ld_table, void* scratch, int rows, int d, int vocab) {
    RLHF_TYPES2(gdt, tdt, (k_embed_grad<X, Y><<<vocab, 256, 0, st>>>((const X*)dout, ld_dout, tokens, scale, accumulate, (Y*)dtable, ld_table, rows, d)));
    return hipGetLastError();
}

}  // namespace rlhf
