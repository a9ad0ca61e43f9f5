// Kernel-level C entry points (include/rlhf_ops.h): thin argument checks around the launchers.
#include "../../include/rlhf_ops.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <mutex>
#include <new>
#include <vector>

#include "../../include/rlhf.h"
#include "kernels.h"

using namespace rlhf;

// Split-KV partials of rlhf_op_paged_decode_attention_noalloc: per (row, query head, split) one
// float accumulator of up to 128 dims, then the (max, sum) pairs.  One copy per GPU, held until
// the process ends; its device address is looked up once per device.
constexpr size_t kNoAllocSlots = 16384;
constexpr size_t kNoAllocMaxHd = 128;
static __device__ __align__(256) float scratch[kNoAllocSlots * (kNoAllocMaxHd + 2)];

namespace {
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
float* g_scratch_ptr[kMaxDevices] = {};

// Device address of `scratch` on the current device (the array's name is only a host-side
// handle; every GPU has its own copy at its own address).
int scratch_of_current_device(float** out) {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) {
        set_global_error("rlhf_op_paged_decode_attention_noalloc: cannot identify the current device");
        return RLHF_EDEVICE;
    }
    std::lock_guard<std::mutex> lk(g_scratch_mu);
    if (!g_scratch_ptr[dev]) {
        void* p = nullptr;
        const hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess || !p) {
            set_global_error("rlhf_op_paged_decode_attention_noalloc: hipGetSymbolAddress failed");
            return RLHF_EDEVICE;
        }
        g_scratch_ptr[dev] = (float*)p;
    }
    *out = g_scratch_ptr[dev];
    return RLHF_OK;
}
}  // namespace

static int status_of(hipError_t e) {
    if (e == hipSuccess) return RLHF_OK;
    return e == hipErrorInvalidValue ? RLHF_EINVAL : RLHF_EDEVICE;
}

extern "C" int rlhf_op_gemm_nsplit(int dtype, int M, int N, int K, int max_split) {
    if (M <= 0 || N <= 0 || K <= 0 || max_split < 1) return 1;
    return gemm_choose_nsplit(dtype == RLHF_BF16 ? kBF16 : kF32, M, N, K, max_split);
}

extern "C" int rlhf_op_gemm(int dtype, int act_half, const void* A, const void* W, float* C, int M, int N,
                            int K, int nsplit, int variant, void* stream) {
    if (!A || !W || !C || M < 0 || N < 0 || K <= 0 || nsplit < 1) return RLHF_EINVAL;
    if (dtype == 2) {        // W is a half copy of a bf16 matrix (rlhf_op_bf16_to_half), A is half
        if (!act_half) return RLHF_EINVAL;
        return status_of(launch_gemm((hipStream_t)stream, kF16, kF16, A, W, C, M, N, K, nsplit, variant));
    }
    if (dtype != RLHF_BF16 && dtype != RLHF_FP32) return RLHF_EINVAL;
    if (act_half && dtype != RLHF_BF16) return RLHF_EINVAL;
    const int wdt = dtype == RLHF_BF16 ? kBF16 : kF32;
    return status_of(launch_gemm((hipStream_t)stream, wdt, act_half ? kF16 : wdt, A, W, C, M, N, K, nsplit, variant));
}

extern "C" int rlhf_op_paged_decode_attention(int dtype, const void* q, const void* pool,
                                              const int32_t* page_table, int pt_stride,
                                              const int32_t* row_sample, const int32_t* ctx_len, void* out,
                                              float* part_acc, float* part_ml, int rows, int layer, int nsplit,
                                              int n_layers, int n_q_heads, int n_kv_heads, int head_dim,
                                              void* stream) {
    if (!q || !pool || !page_table || !row_sample || !ctx_len || !out || rows < 0 || nsplit < 1 ||
        layer < 0 || layer >= n_layers || n_kv_heads <= 0 || n_q_heads % n_kv_heads)
        return RLHF_EINVAL;
    if (nsplit > 1 && (!part_acc || !part_ml)) return RLHF_EINVAL;
    Dims dm{n_layers, n_q_heads * head_dim, n_q_heads, n_kv_heads, head_dim, 0, 0, 16};
    const int dt = dtype == 2 ? kF16 : dtype == RLHF_BF16 ? kBF16 : kF32;
    return status_of(launch_decode_attn((hipStream_t)stream, dt, q, pool,
                                        page_table, pt_stride, row_sample, ctx_len, out, part_acc, part_ml,
                                        rows, layer, nsplit, dm));
}

extern "C" int rlhf_op_paged_decode_attention_noalloc(int dtype, const void* q, const void* pool,
                                                      const int32_t* page_table, int pt_stride,
                                                      const int32_t* row_sample, const int32_t* ctx_len,
                                                      void* out, int rows, int layer, int nsplit, int n_layers,
                                                      int n_q_heads, int n_kv_heads, int head_dim, void* stream) {
    if (!q || !pool || !page_table || !row_sample || !ctx_len || !out || rows < 0 || nsplit < 1 ||
        layer < 0 || layer >= n_layers || n_kv_heads <= 0 || n_q_heads <= 0 || n_q_heads % n_kv_heads) {
        set_global_error("rlhf_op_paged_decode_attention_noalloc: bad argument");
        return RLHF_EINVAL;
    }
    const size_t slots = (size_t)rows * n_q_heads * nsplit;
    if (head_dim <= 0 || (size_t)head_dim > kNoAllocMaxHd || slots > kNoAllocSlots) {
        set_global_error("rlhf_op_paged_decode_attention_noalloc: rows * n_q_heads * nsplit must not exceed 16384 "
                         "and head_dim must not exceed 128 (the size of the built-in scratch)");
        return RLHF_EINVAL;
    }
    float* sc = nullptr;
    const int rc = scratch_of_current_device(&sc);
    if (rc != RLHF_OK) return rc;
    float* part_acc = sc;                                   // [slots][head_dim]
    float* part_ml = sc + kNoAllocSlots * kNoAllocMaxHd;    // [slots][2]
    Dims dm{n_layers, n_q_heads * head_dim, n_q_heads, n_kv_heads, head_dim, 0, 0, 16};
    const int dt = dtype == 2 ? kF16 : dtype == RLHF_BF16 ? kBF16 : kF32;
    const hipError_t e = launch_decode_attn((hipStream_t)stream, dt, q, pool, page_table, pt_stride, row_sample,
                                            ctx_len, out, part_acc, part_ml, rows, layer, nsplit, dm);
    if (e != hipSuccess) set_global_error("rlhf_op_paged_decode_attention_noalloc: unsupported shape or launch failure");
    return status_of(e);
}

extern "C" int rlhf_op_varlen_attention(int out_half, const float* q, const float* k, const float* v,
                                        const int32_t* row_start, const int32_t* row_pos, void* out,
                                        int rows, int n_q_heads, int n_kv_heads, int head_dim, void* stream) {
    if (!q || !k || !v || !row_start || !row_pos || !out || rows < 0 || n_kv_heads <= 0 ||
        n_q_heads % n_kv_heads)
        return RLHF_EINVAL;
    Dims dm{1, n_q_heads * head_dim, n_q_heads, n_kv_heads, head_dim, 0, 0, 16};
    return status_of(launch_prefill_attn((hipStream_t)stream, out_half ? kF16 : kF32, q, k, v, row_start,
                                         row_pos, out, rows, dm));
}

extern "C" int rlhf_op_flash_attention(const void* q, const void* k, const void* v, const int32_t* tile_start,
                                       const int32_t* tile_q0, const int32_t* tile_len, void* out, int n_tiles,
                                       int rows, int n_q_heads, int n_kv_heads, int head_dim, void* stream) {
    if (!q || !k || !v || !tile_start || !tile_q0 || !tile_len || !out || n_tiles < 0 || rows <= 0 ||
        n_kv_heads <= 0 || n_q_heads % n_kv_heads)
        return RLHF_EINVAL;
    Dims dm{1, n_q_heads * head_dim, n_q_heads, n_kv_heads, head_dim, 0, 0, 16};
    return status_of(launch_flash_attn((hipStream_t)stream, q, k, v, tile_start, tile_q0, tile_len, out, n_tiles,
                                       rows, dm));
}

extern "C" int rlhf_op_gemm_swiglu(int act_half, const void* A, const void* W_gate_up, void* act, int M, int ffn,
                                   int K, void* stream) {
    if (!A || !W_gate_up || !act) return RLHF_EINVAL;
    const int adt = act_half ? kF16 : kBF16, wdt = act_half == 2 ? kF16 : kBF16;
    if (M >= 1 && M <= 16) {            // the few-row kernel of decode steps (no K split, SwiGLU in its epilogue)
        if (!gemm_stream_supported(wdt, adt, M, K) || K % 256 || ffn <= 0 || ffn % 8) return RLHF_EINVAL;
        RowsEpi ep;
        ep.act = act;
        ep.ffn = ffn;
        return status_of(launch_gemm_stream((hipStream_t)stream, wdt, adt, 1, A, W_gate_up, nullptr, M, 2 * ffn, K, ep));
    }
    if (M < 512 || !gemm_swiglu_supported(wdt, adt, M, ffn, K)) return RLHF_EINVAL;
    return status_of(launch_gemm_swiglu((hipStream_t)stream, wdt, adt, A, W_gate_up, act, M, ffn, K));
}

extern "C" int rlhf_op_gemm_rope(int act_half, const void* A, const void* W_qkv, const int32_t* pos,
                                 const int32_t* kv_dst, const float* table, void* q, void* k, void* v, void* pool,
                                 int M, int K, int layer, int n_layers, int n_q_heads, int n_kv_heads, int head_dim,
                                 void* stream) {
    if (!A || !W_qkv || !pos || !table || !q || (pool && !kv_dst) || n_q_heads <= 0 || n_kv_heads <= 0 ||
        n_q_heads % n_kv_heads || layer < 0 || layer >= n_layers)
        return RLHF_EINVAL;
    const int adt = act_half ? kF16 : kBF16, wdt = act_half == 2 ? kF16 : kBF16;
    Dims dm{n_layers, K, n_q_heads, n_kv_heads, head_dim, 0, 0, 16};
    RopeOut ro;
    ro.pos = pos; ro.kv_dst = kv_dst; ro.table = table;
    ro.q = q; ro.k = k; ro.v = v; ro.pool = pool;
    ro.layer = layer; ro.n_layers = n_layers;
    ro.n_q_heads = n_q_heads; ro.n_kv_heads = n_kv_heads; ro.head_dim = head_dim;
    if (M >= 1 && M <= 16) {            // the few-row kernel of decode steps (no K split, rotary in its epilogue)
        if (!gemm_stream_supported(wdt, adt, M, K) || K % 256 || (head_dim != 64 && head_dim != 128)) return RLHF_EINVAL;
        RowsEpi ep;
        ep.ro = ro;
        return status_of(launch_gemm_stream((hipStream_t)stream, wdt, adt, 2, A, W_qkv, nullptr, M,
                                            (n_q_heads + 2 * n_kv_heads) * head_dim, K, ep));
    }
    if (M < 512 || !gemm_rope_supported(wdt, adt, M, K, dm)) return RLHF_EINVAL;
    return status_of(launch_gemm_rope((hipStream_t)stream, wdt, adt, A, W_qkv, M, K, ro));
}

// ---- row-wise kernels

static int act_of(int act_dtype) { return act_dtype == 2 ? kF16 : act_dtype == RLHF_BF16 ? kBF16 : act_dtype == RLHF_FP32 ? kF32 : -1; }

extern "C" int rlhf_op_rmsnorm(int act_dtype, float* h, const float* part, int nsplit, int64_t sstride,
                               const int32_t* row_idx, const float* g, void* xn, int rows, int d, float eps,
                               void* stream) {
    const int adt = act_of(act_dtype);
    if (adt < 0 || !h || !g || !xn || rows < 0 || d <= 0 || nsplit < 0 || (nsplit > 0 && (!part || sstride < 0)))
        return RLHF_EINVAL;
    return status_of(launch_rmsnorm((hipStream_t)stream, adt, h, part, nsplit, (size_t)sstride, row_idx, g, xn, rows,
                                    d, eps));
}

extern "C" int rlhf_op_rope_kv(int act_dtype, const float* qkv, int nsplit, int64_t sstride, const int32_t* pos,
                               const int32_t* kv_dst, const float* table, void* q, void* k, void* v, void* pool,
                               int layer, int rows, int n_layers, int n_q_heads, int n_kv_heads, int head_dim,
                               void* stream) {
    const int adt = act_of(act_dtype);
    if (adt < 0 || !qkv || !pos || !table || !q || nsplit < 1 || sstride < 0 || rows < 0 || (pool && !kv_dst) ||
        n_q_heads <= 0 || n_kv_heads <= 0 || head_dim <= 0 || head_dim % 2 || layer < 0 || layer >= n_layers)
        return RLHF_EINVAL;
    Dims dm{n_layers, n_q_heads * head_dim, n_q_heads, n_kv_heads, head_dim, 0, 0, 16};
    return status_of(launch_rope_kv((hipStream_t)stream, adt, adt, qkv, nsplit, (size_t)sstride, pos, kv_dst, table,
                                    q, k, v, pool, layer, rows, dm));
}

extern "C" int rlhf_op_swiglu(int act_dtype, const float* gu, int nsplit, int64_t sstride, void* act, int rows,
                              int ffn, void* stream) {
    const int adt = act_of(act_dtype);
    if (adt < 0 || !gu || !act || nsplit < 1 || sstride < 0 || rows < 0 || ffn <= 0) return RLHF_EINVAL;
    return status_of(launch_swiglu((hipStream_t)stream, adt, gu, nsplit, (size_t)sstride, act, rows, ffn));
}

extern "C" int64_t rlhf_op_pick_scratch_floats(int rows) { return rows > 0 ? (int64_t)pick_scratch_floats(rows) : 0; }

extern "C" int rlhf_op_pick(const float* logits, int nsplit, int64_t sstride, int rows, int vocab,
                            const int32_t* forced, int32_t* tokens, const int32_t* tok_dst, float* lp,
                            const int32_t* lp_dst, int32_t* picked, float* scratch, void* stream) {
    if (!logits || !tokens || !tok_dst || !lp || !lp_dst || !scratch || nsplit < 1 || sstride < 0 || rows < 0 ||
        vocab < 1)
        return RLHF_EINVAL;
    return status_of(launch_pick((hipStream_t)stream, logits, nsplit, (size_t)sstride, rows, vocab, forced, tokens,
                                 tok_dst, lp, lp_dst, picked, scratch));
}

extern "C" int rlhf_op_gather_lp(const float* logits, int nsplit, int64_t sstride, int rows, int vocab,
                                 const int32_t* tokens, const int32_t* target_idx, float* out,
                                 const int32_t* out_dst, void* stream) {
    if (!logits || !tokens || !target_idx || !out || !out_dst || nsplit < 1 || sstride < 0 || rows < 0 || vocab < 1)
        return RLHF_EINVAL;
    return status_of(launch_gather_lp((hipStream_t)stream, logits, nsplit, (size_t)sstride, rows, vocab, tokens,
                                      target_idx, out, out_dst));
}

extern "C" int rlhf_op_head_dot(int act_dtype, int w_dtype, const void* xn, const void* w, int rows, int d,
                                float* out, const int32_t* out_dst, void* stream) {
    const int adt = act_of(act_dtype);
    if (adt < 0 || (w_dtype != RLHF_FP32 && w_dtype != RLHF_BF16) || !xn || !w || !out || !out_dst || rows < 0 ||
        d <= 0 || d % 8)
        return RLHF_EINVAL;
    return status_of(launch_head_dot((hipStream_t)stream, adt, w_dtype == RLHF_BF16 ? kBF16 : kF32, xn, w, rows, d,
                                     out, out_dst));
}

extern "C" int64_t rlhf_op_lm_head_logprob_scratch_floats(int M, int vocab) {
    if (M <= 0 || vocab <= 0) return 0;
    return (int64_t)M * (2 * gemm_lse_partials(vocab) + 1);
}

extern "C" int rlhf_op_lm_head_logprob(int act_half, const void* A, const void* W_head, const int32_t* tokens,
                                       const int32_t* target_idx, float* out, const int32_t* out_dst,
                                       float* scratch, int M, int vocab, int K, void* stream) {
    if (!A || !W_head || !tokens || !target_idx || !out || !out_dst || !scratch || M < 0 || vocab < 1 || K <= 0)
        return RLHF_EINVAL;
    const int adt = act_half ? kF16 : kBF16, wdt = act_half == 2 ? kF16 : kBF16;
    if (!gemm_lse_supported(wdt, adt, K)) return RLHF_EINVAL;
    LseOut lo;
    lo.n_part = gemm_lse_partials(vocab);
    lo.tokens = tokens;
    lo.target_idx = target_idx;
    lo.part_max = scratch;
    lo.part_sum = scratch + (size_t)M * lo.n_part;
    lo.tgt = scratch + (size_t)2 * M * lo.n_part;
    hipError_t e = launch_gemm_lse((hipStream_t)stream, wdt, adt, A, W_head, M, vocab, K, lo);
    if (e == hipSuccess)
        e = launch_lse_merge((hipStream_t)stream, lo.part_max, lo.part_sum, lo.tgt, lo.n_part, M, out, out_dst);
    return status_of(e);
}

extern "C" int rlhf_op_bf16_to_half(const void* src, void* dst, int64_t n, void* stream) {
    if (!src || !dst || n < 0 || n % 2) return RLHF_EINVAL;
    return status_of(launch_bf16_to_half((hipStream_t)stream, src, dst, (size_t)n));
}

// ---- the Actor's update

static size_t elem_bytes(int dt) { return dt == kF32 ? 4 : 2; }
// A matrix that an operator reads or writes: its elements lie in `rows` pieces of `width` bytes, `step` bytes apart.
struct Matrix { uintptr_t at; size_t rows, width, step; };
static Matrix matrix(const void* p, int rows, int cols, int64_t ld, int dt) {
    return Matrix{(uintptr_t)p, (size_t)rows, (size_t)cols * elem_bytes(dt), (size_t)ld * elem_bytes(dt)};
}
// Matrices that share an element, or might (of different steps, and interleaved).
static bool overlap(const Matrix& a, const Matrix& b) {
    if (a.rows == 0 || b.rows == 0) return false;
    if (a.at >= b.at + (b.rows - 1) * b.step + b.width || b.at >= a.at + (a.rows - 1) * a.step + a.width) return false;
    if (a.step != b.step) return true;
    const size_t behind = a.at <= b.at ? (b.at - a.at) % a.step : (a.step - (a.at - b.at) % a.step) % a.step;     // b's columns, behind a's
    return behind < a.width || behind + b.width > a.step;
}
static bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

extern "C" int64_t rlhf_op_policy_loss_scratch_floats(int rows, int vocab) {
    return rows > 0 && vocab > 0 ? (int64_t)policy_scratch_floats(rows, vocab) : 0;
}

extern "C" int rlhf_op_policy_loss(int logit_dtype, const void* logits, int64_t ld, const int32_t* tokens,
                                   const float* lp_old, const float* lp_ref, const float* adv, const float* weight,
                                   float clip_low, float clip_high, float kl_coef, float grad_scale, float* lp, float* stats,
                                   void* dlogits, int64_t ld_grad, float* scratch, int rows, int vocab, void* stream) {
    const int dt = act_of(logit_dtype);
    if (dt < 0 || rows < 0 || vocab < 1 || ld < vocab || !stats || (dlogits && ld_grad < vocab)) return RLHF_EINVAL;
    if (rows > 0 && (!logits || !tokens || !lp_old || !adv || !lp || !scratch)) return RLHF_EINVAL;
    // written so that a NaN is refused
    if (!(clip_low >= 0.f && clip_low <= 1.f) || !(clip_high >= 0.f) || !(kl_coef >= 0.f && kl_coef < INFINITY) ||
        !(grad_scale > -INFINITY && grad_scale < INFINITY) || (!lp_ref && kl_coef != 0.f))
        return RLHF_EINVAL;
    if (!aligned(logits, elem_bytes(dt)) || !aligned(dlogits, elem_bytes(dt))) return RLHF_EINVAL;
    if (dlogits && !(dlogits == logits && ld_grad == ld) &&
        overlap(matrix(logits, rows, vocab, ld, dt), matrix(dlogits, rows, vocab, ld_grad, dt)))
        return RLHF_EINVAL;
    PolicyArgs a;
    a.logits = logits; a.ld = (size_t)ld; a.tokens = tokens;
    a.weight = weight; a.lp_old = lp_old; a.lp_ref = lp_ref; a.adv = adv;
    a.grad = dlogits; a.ld_grad = (size_t)ld_grad; a.lp = lp; a.terms = scratch; a.terms_ld = (size_t)rows;
    a.rows = rows; a.vocab = vocab;
    a.lo = 1.f - clip_low; a.hi = 1.f + clip_high; a.kl_coef = kl_coef; a.grad_scale = grad_scale;
    return status_of(launch_policy_loss((hipStream_t)stream, dt, a, stats));
}

extern "C" int rlhf_op_embed(int table_dtype, int out_dtype, const void* table, int64_t ld_table, const int32_t* tokens,
                             float scale, void* out, int64_t ld_out, int rows, int d, int vocab, void* stream) {
    const int tdt = act_of(table_dtype), odt = act_of(out_dtype);
    if (tdt < 0 || odt < 0 || rows < 0 || d < 1 || vocab < 1 || ld_table < d || ld_out < d) return RLHF_EINVAL;
    if (rows == 0) return RLHF_OK;
    if (!table || !tokens || !out || !aligned(table, elem_bytes(tdt)) || !aligned(out, elem_bytes(odt)) ||
        overlap(matrix(table, vocab, d, ld_table, tdt), matrix(out, rows, d, ld_out, odt)))
        return RLHF_EINVAL;
    return status_of(launch_embed_rows((hipStream_t)stream, tdt, odt, table, (size_t)ld_table, tokens, scale, out,
                                       (size_t)ld_out, rows, d, vocab));
}

extern "C" int64_t rlhf_op_embed_grad_scratch_bytes(int rows, int d, int vocab) {
    return rows > 0 && d > 0 && vocab > 0 ? (int64_t)embed_grad_scratch_bytes(rows, d, vocab) : 0;
}

extern "C" int rlhf_op_embed_grad(int dout_dtype, int table_dtype, const void* dout, int64_t ld_dout, const int32_t* tokens,
                                  float scale, int accumulate, void* dtable, int64_t ld_table, void* scratch, int rows,
                                  int d, int vocab, void* stream) {
    const int gdt = act_of(dout_dtype), tdt = act_of(table_dtype);
    if (gdt < 0 || tdt < 0 || rows < 0 || d < 1 || vocab < 1 || ld_dout < d || ld_table < d || !dtable ||
        !aligned(dtable, elem_bytes(tdt)))
        return RLHF_EINVAL;
    if (rows > 0 && (!dout || !tokens || (!scratch && embed_grad_scratch_bytes(rows, d, vocab) > 0) || !aligned(dout, elem_bytes(gdt)) || !aligned(scratch, 16) ||
                     overlap(matrix(dout, rows, d, ld_dout, gdt), matrix(dtable, vocab, d, ld_table, tdt))))
        return RLHF_EINVAL;
    return status_of(launch_embed_grad((hipStream_t)stream, gdt, tdt, dout, (size_t)ld_dout, tokens, scale, accumulate != 0,
                                       dtable, (size_t)ld_table, scratch, rows, d, vocab));
}

// The caller's list in the launchers' form; empty tensors are dropped.  false: an entry that cannot be used.
static bool grad_tensors(const rlhf_tensor* t, int n, bool write, std::vector<GradTensor>* out) {
    if (n < 0 || (n > 0 && !t)) return false;
    out->reserve((size_t)n);
    for (int i = 0; i < n; ++i) {
        const int dt = act_of(t[i].dtype);
        if (dt < 0 || t[i].n < 0 || t[i].n >= kMaxGradElements) return false;
        if (t[i].n == 0) continue;
        if (!t[i].src || !aligned(t[i].src, elem_bytes(dt)) || (write && !t[i].dst) || !aligned(t[i].dst, elem_bytes(dt)))
            return false;
        out->push_back(GradTensor{t[i].src, t[i].dst, (size_t)t[i].n, dt});
    }
    return true;
}

// Whether every dst is memory of its own: shared with no other entry, and with its own src only as a whole.  Where two entries
// write the same memory, or one writes what another reads, the workgroups' order would decide what is scaled, and how often.
static bool apart(const std::vector<GradTensor>& v) {
    struct Range { uintptr_t from, to; bool write; };
    std::vector<Range> r;
    r.reserve(2 * v.size());
    for (const GradTensor& t : v) {
        const size_t bytes = t.n * elem_bytes(t.dtype);
        r.push_back({(uintptr_t)t.dst, (uintptr_t)t.dst + bytes, true});
        if (t.src != t.dst) r.push_back({(uintptr_t)t.src, (uintptr_t)t.src + bytes, false});
    }
    const auto before = [](const Range& a, const Range& b) { return a.from < b.from; };
    if (!std::is_sorted(r.begin(), r.end(), before)) std::sort(r.begin(), r.end(), before);
    uintptr_t end = 0, written = 0;               // of all ranges so far, and of those that are written
    for (const Range& x : r) {
        if (x.from < (x.write ? end : written)) return false;
        end = std::max(end, x.to);
        if (x.write) written = std::max(written, x.to);
    }
    return true;
}

extern "C" int64_t rlhf_op_grad_norm_scratch_doubles(const rlhf_tensor* tensors, int n_tensors) try {
    std::vector<GradTensor> v;
    return grad_tensors(tensors, n_tensors, false, &v) ? (int64_t)grad_norm_scratch_doubles(v.data(), (int)v.size()) : 0;
} catch (const std::bad_alloc&) {
    return 0;
}

extern "C" int rlhf_op_grad_norm(const rlhf_tensor* tensors, int n_tensors, float* norm, double* scratch, void* stream) try {
    std::vector<GradTensor> v;
    if (!norm || !grad_tensors(tensors, n_tensors, false, &v) || (!v.empty() && (!scratch || !aligned(scratch, 8)))) return RLHF_EINVAL;
    return status_of(launch_grad_norm((hipStream_t)stream, v.data(), (int)v.size(), norm, scratch));
} catch (const std::bad_alloc&) {
    return RLHF_ENOMEM;
}

extern "C" int rlhf_op_clip_grads(const rlhf_tensor* tensors, int n_tensors, const float* norm, float max_norm, void* stream) try {
    std::vector<GradTensor> v;
    if (!norm || !(max_norm > 0.f) || !grad_tensors(tensors, n_tensors, true, &v) || !apart(v)) return RLHF_EINVAL;
    return status_of(launch_clip_grads((hipStream_t)stream, v.data(), (int)v.size(), norm, max_norm));
} catch (const std::bad_alloc&) {
    return RLHF_ENOMEM;
}

// ---- attention that reads less of its cache

// Addresses and row strides of matrices of whole 16-byte pieces.
static bool in_pieces(const void* p, int64_t ld, int dt) { return p && aligned(p, 16) && (size_t)ld * elem_bytes(dt) % 16 == 0; }
static bool heads_ok(int hq, int hkv, int hd) {
    return hkv > 0 && hq > 0 && hq % hkv == 0 && hq <= 1 << 16 && (hd == 64 || hd == 128);
}
constexpr size_t kMaxPoolBytes = (size_t)1 << 47;       // beyond any address space
static Matrix bytes_of(const void* p, size_t n) { return Matrix{(uintptr_t)p, n > 0 ? 1u : 0u, n, n}; }

extern "C" int rlhf_op_window_attention(int act_dtype, const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                                        const int32_t* tile_start, const int32_t* tile_q0, const int32_t* tile_len, void* out,
                                        int64_t ld_out, int n_tiles, int rows, int window, int sinks, int n_q_heads, int n_kv_heads,
                                        int head_dim, void* stream) {
    const int dt = act_of(act_dtype);
    if (dt < 0 || n_tiles < 0 || n_tiles > 1 << 30 || rows < 0 || rows > 1 << 30 || window < 1 || sinks < 0 || !heads_ok(n_q_heads, n_kv_heads, head_dim))
        return RLHF_EINVAL;
    const int qc = n_q_heads * head_dim, kc = n_kv_heads * head_dim;
    if (ld_q < qc || ld_out < qc || ld_k < kc || ld_v < kc || ld_k >= 1 << 25 || ld_v >= 1 << 25) return RLHF_EINVAL;     // the rows of a tile of keys in 32 bits
    if (n_tiles == 0 || rows == 0) return RLHF_OK;
    if (!tile_start || !tile_q0 || !tile_len || !in_pieces(q, ld_q, dt) || !in_pieces(k, ld_k, dt) || !in_pieces(v, ld_v, dt) || !in_pieces(out, ld_out, dt))
        return RLHF_EINVAL;
    const Matrix o = matrix(out, rows, qc, ld_out, dt);
    if (overlap(o, matrix(q, rows, qc, ld_q, dt)) || overlap(o, matrix(k, rows, kc, ld_k, dt)) || overlap(o, matrix(v, rows, kc, ld_v, dt)))
        return RLHF_EINVAL;
    WindowArgs a;
    a.q = q; a.k = k; a.v = v; a.ld_q = (size_t)ld_q; a.ld_k = (size_t)ld_k; a.ld_v = (size_t)ld_v;
    a.tile_start = tile_start; a.tile_q0 = tile_q0; a.tile_len = tile_len;
    a.out = out; a.ld_out = (size_t)ld_out; a.n_tiles = n_tiles; a.rows = rows;
    a.window = window; a.sinks = sinks; a.n_q_heads = n_q_heads; a.n_kv_heads = n_kv_heads;
    return status_of(launch_window_attention((hipStream_t)stream, dt, head_dim, a));
}

extern "C" int rlhf_op_window_decode_nsplit(int rows, int n_q_heads, int n_kv_heads, int max_ctx, int window, int sinks) {
    if (rows < 1 || n_kv_heads < 1 || n_q_heads < n_kv_heads || max_ctx < 1 || window < 1 || sinks < 0) return 1;
    return window_decode_nsplit(rows, n_q_heads, n_kv_heads, max_ctx, window, sinks);
}

extern "C" int64_t rlhf_op_window_decode_scratch_floats(int rows, int n_q_heads, int head_dim, int nsplit) {
    return rows > 0 && n_q_heads > 0 && head_dim > 0 && nsplit > 1 ? (int64_t)window_decode_scratch_floats(rows, n_q_heads, head_dim, nsplit) : 0;
}

static int window_decode(bool four_bits, int act_dtype, const void* q, int64_t ld_q, const void* pool, int n_pages, const int32_t* page_table,
                         int pt_stride, int n_samples, const int32_t* row_sample, const int32_t* ctx_len, void* out, int64_t ld_out,
                         float* scratch, int rows, int layer, int nsplit, int window, int sinks, int n_layers, int n_q_heads,
                         int n_kv_heads, int head_dim, void* stream) {
    const int dt = act_of(act_dtype);
    if (dt < 0 || rows < 0 || rows > 1 << 24 || nsplit < 1 || nsplit > 64 || window < 1 || sinks < 0 || layer < 0 || layer >= n_layers || n_layers > 1 << 16 ||
        n_pages < 0 || n_pages >= 1 << 27 || n_samples < 0 || pt_stride < 0 || pt_stride >= 1 << 27 || !heads_ok(n_q_heads, n_kv_heads, head_dim))
        return RLHF_EINVAL;
    const int qc = n_q_heads * head_dim;
    if (ld_q < qc || ld_out < qc) return RLHF_EINVAL;
    if (rows == 0) return RLHF_OK;
    if (n_pages < 1 || n_samples < 1 || pt_stride < 1 || !pool || !aligned(pool, 16) || !page_table || !row_sample || !ctx_len || !in_pieces(q, ld_q, dt) || !in_pieces(out, ld_out, dt) ||
        (nsplit > 1 && (!scratch || !aligned(scratch, 16))))
        return RLHF_EINVAL;
    const size_t page = four_bits ? (size_t)rlhf_op_kv4_page_bytes(n_layers, n_kv_heads, head_dim)
                                  : (size_t)n_layers * 2 * n_kv_heads * 16 * head_dim * elem_bytes(dt);
    const Matrix o = matrix(out, rows, qc, ld_out, dt);
    if (page > kMaxPoolBytes / n_pages || overlap(o, matrix(q, rows, qc, ld_q, dt)) || overlap(o, bytes_of(pool, page * n_pages))) return RLHF_EINVAL;
    WindowDecodeArgs a;
    a.q = q; a.pool = pool; a.page_table = page_table; a.row_sample = row_sample; a.ctx_len = ctx_len; a.out = out; a.part = scratch;
    a.ld_q = (size_t)ld_q; a.ld_out = (size_t)ld_out; a.rows = rows; a.layer = layer; a.n_layers = n_layers;
    a.n_q_heads = n_q_heads; a.n_kv_heads = n_kv_heads; a.nsplit = nsplit; a.window = window; a.sinks = sinks;
    a.n_pages = n_pages; a.n_samples = n_samples; a.pt_stride = pt_stride;
    return status_of(launch_window_decode((hipStream_t)stream, dt, four_bits, head_dim, a));
}

extern "C" int rlhf_op_window_decode_attention(int act_dtype, const void* q, int64_t ld_q, const void* pool, int n_pages,
                                               const int32_t* page_table, int pt_stride, int n_samples, const int32_t* row_sample,
                                               const int32_t* ctx_len, void* out, int64_t ld_out, float* scratch, int rows, int layer,
                                               int nsplit, int window, int sinks, int n_layers, int n_q_heads, int n_kv_heads,
                                               int head_dim, void* stream) {
    return window_decode(false, act_dtype, q, ld_q, pool, n_pages, page_table, pt_stride, n_samples, row_sample, ctx_len, out, ld_out, scratch, rows,
                         layer, nsplit, window, sinks, n_layers, n_q_heads, n_kv_heads, head_dim, stream);
}

extern "C" int rlhf_op_kv4_decode_attention(int act_dtype, const void* q, int64_t ld_q, const void* pool, int n_pages,
                                            const int32_t* page_table, int pt_stride, int n_samples, const int32_t* row_sample,
                                            const int32_t* ctx_len, void* out, int64_t ld_out, float* scratch, int rows, int layer,
                                            int nsplit, int window, int sinks, int n_layers, int n_q_heads, int n_kv_heads,
                                            int head_dim, void* stream) {
    return window_decode(true, act_dtype, q, ld_q, pool, n_pages, page_table, pt_stride, n_samples, row_sample, ctx_len, out, ld_out, scratch, rows,
                         layer, nsplit, window, sinks, n_layers, n_q_heads, n_kv_heads, head_dim, stream);
}

extern "C" int64_t rlhf_op_kv4_page_bytes(int n_layers, int n_kv_heads, int head_dim) {
    return n_layers > 0 && n_kv_heads > 0 && (head_dim == 64 || head_dim == 128)
               ? (int64_t)n_layers * n_kv_heads * (int64_t)kv4_block_bytes(head_dim) : 0;
}

// Checks what append and read share; a row is n_kv_heads * head_dim elements.
static bool kv4_args(int dt, const void* k, int64_t ld_k, const void* v, int64_t ld_v, const int32_t* slot, const void* pool, int n_pages,
                     int rows, int layer, int n_layers, int n_kv_heads, int head_dim, bool writes_rows, Kv4Args* a) {
    if (dt < 0 || rows < 0 || rows > 1 << 30 || n_pages < 0 || n_pages >= 1 << 27 || layer < 0 || layer >= n_layers || n_layers > 1 << 16 ||
        !heads_ok(n_kv_heads, n_kv_heads, head_dim) || ld_k < (int64_t)n_kv_heads * head_dim || ld_v < (int64_t)n_kv_heads * head_dim)
        return false;
    if (rows > 0) {
        const int cols = n_kv_heads * head_dim;
        const Matrix mk = matrix(k, rows, cols, ld_k, dt), mv = matrix(v, rows, cols, ld_v, dt);
        const size_t page = (size_t)rlhf_op_kv4_page_bytes(n_layers, n_kv_heads, head_dim);
        const Matrix mp = bytes_of(pool, page * n_pages);
        if (n_pages < 1 || page > kMaxPoolBytes / n_pages || !slot || !pool || !aligned(pool, 16) || !in_pieces(k, ld_k, dt) || !in_pieces(v, ld_v, dt) || overlap(mk, mp) || overlap(mv, mp) ||
            (writes_rows && overlap(mk, mv)))
            return false;
    }
    *a = Kv4Args{(void*)k, (void*)v, (size_t)ld_k, (size_t)ld_v, slot, (void*)pool, n_pages, rows, layer, n_layers, n_kv_heads};
    return true;
}

extern "C" int rlhf_op_kv4_append(int act_dtype, const void* k, int64_t ld_k, const void* v, int64_t ld_v, const int32_t* kv_dst, void* pool,
                                  int n_pages, int rows, int layer, int n_layers, int n_kv_heads, int head_dim, void* stream) {
    const int dt = act_of(act_dtype);
    Kv4Args a;
    if (!kv4_args(dt, k, ld_k, v, ld_v, kv_dst, pool, n_pages, rows, layer, n_layers, n_kv_heads, head_dim, false, &a)) return RLHF_EINVAL;
    return rows == 0 ? RLHF_OK : status_of(launch_kv4_append((hipStream_t)stream, dt, head_dim, a));
}

extern "C" int rlhf_op_kv4_read(int act_dtype, const void* pool, int n_pages, const int32_t* kv_src, void* k, int64_t ld_k, void* v, int64_t ld_v,
                                int rows, int layer, int n_layers, int n_kv_heads, int head_dim, void* stream) {
    const int dt = act_of(act_dtype);
    Kv4Args a;
    if (!kv4_args(dt, k, ld_k, v, ld_v, kv_src, pool, n_pages, rows, layer, n_layers, n_kv_heads, head_dim, true, &a)) return RLHF_EINVAL;
    return rows == 0 ? RLHF_OK : status_of(launch_kv4_read((hipStream_t)stream, dt, head_dim, a));
}

extern "C" int rlhf_op_gemm_tall_grid(int tiles_m, int tiles_n) {
    return tiles_m > 0 && tiles_n > 0 ? gemm_tall_grid(tiles_m, tiles_n) : 0;
}

extern "C" int rlhf_op_gemm_tall_tile(int bid, int tiles_m, int tiles_n, int* tm, int* tn) {
    if (bid < 0 || tiles_m <= 0 || tiles_n <= 0 || !tm || !tn) return RLHF_EINVAL;
    return gemm_tall_tile(bid, tiles_m, tiles_n, tm, tn) ? 1 : 0;
}
