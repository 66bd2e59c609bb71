// Attention of a batch's new rows over a paged cache: s2d2_paged_attention.
#include <math.h>

#include "paged_attention.cuh"

namespace s2d2 {
namespace {

int check_shape(const char* op, const s2d2_rows* rows, const s2d2_paged_kv* kv, int n_q_heads) {
    if (int rc = ops::check_rows(op, rows)) return rc;
    if (int rc = ops::check_kv(op, kv)) return rc;
    if (kv->head_dim > 128) return ops::fail(S2D2_ERR_UNSUPPORTED, "%s: head_dim must be at most 128", op);
    if (n_q_heads < 1 || n_q_heads > S2D2_MAX_HEADS || n_q_heads % kv->n_kv_heads)
        return ops::fail(S2D2_ERR_INVALID, "%s: n_q_heads must be a multiple of n_kv_heads, at most %d", op, S2D2_MAX_HEADS);
    return S2D2_OK;
}

}  // namespace

namespace ops {
cudaError_t load_attention_kernels() { return load(patt::rows_kernel); }
}  // namespace ops
}  // namespace s2d2

using namespace s2d2;

extern "C" int s2d2_paged_attention_workspace(const s2d2_rows* rows, const s2d2_paged_kv* kv, int32_t n_q_heads, int64_t* bytes) {
    ops::clear_error();
    const char* op = "paged_attention_workspace";
    if (!bytes) return ops::fail(S2D2_ERR_INVALID, "%s: bytes: null pointer", op);
    if (int rc = check_shape(op, rows, kv, n_q_heads)) return rc;
    *bytes = 0;
    return S2D2_OK;
}

extern "C" int s2d2_paged_attention(const void* d_q, int64_t q_stride, void* d_out, int64_t out_stride, float* d_lse, int32_t n_q_heads,
                                    const s2d2_rows* rows, const s2d2_paged_kv* kv, int32_t mask_block, const uint64_t* d_row_mask,
                                    float scale, void* d_ws, int64_t ws_bytes, void* cuda_stream) {
    ops::clear_error();
    const char* op = "paged_attention";
    if (int rc = check_shape(op, rows, kv, n_q_heads)) return rc;
    const long long width = (long long)n_q_heads * kv->head_dim;
    if (q_stride < width || q_stride % 8 || q_stride > (1LL << 40)) return ops::fail(S2D2_ERR_INVALID, "%s: q_stride must be a multiple of 8 in heads * head_dim..2^40", op);
    if (out_stride < width || out_stride % 8 || out_stride > (1LL << 40)) return ops::fail(S2D2_ERR_INVALID, "%s: out_stride must be a multiple of 8 in heads * head_dim..2^40", op);
    if (mask_block < 0) return ops::fail(S2D2_ERR_INVALID, "%s: mask_block must not be negative", op);
    if (d_row_mask && mask_block) return ops::fail(S2D2_ERR_INVALID, "%s: mask_block must be 0 with row masks", op);
    if (!(scale > 0.f) || !isfinite(scale)) return ops::fail(S2D2_ERR_INVALID, "%s: scale must be positive", op);
    const ops::Device* dev;
    if (int rc = ops::device(&dev)) return rc;
    if (rows->n_rows == 0 || rows->n_seqs == 0) return S2D2_OK;
    patt::Params p = {};
    if (int rc = ops::device_rows(dev, op, rows, kv, &p.b)) return rc;
    if (int rc = ops::device_kv(dev, op, kv, &p.c)) return rc;
    if (int rc = ops::check_ptr(dev, d_q, 16, "q")) return rc;
    if (int rc = ops::check_ptr(dev, d_out, 16, "out")) return rc;
    if (d_lse)
        if (int rc = ops::check_ptr(dev, d_lse, 4, "lse")) return rc;
    if (d_row_mask)
        if (int rc = ops::check_ptr(dev, d_row_mask, 8, "row_mask")) return rc;
    p.q = (const bf16*)d_q;
    p.out = (bf16*)d_out;
    p.lse = d_lse;
    p.q_ld = q_stride;
    p.out_ld = out_stride;
    p.row_mask = (const unsigned long long*)d_row_mask;
    p.mask_block = mask_block;
    p.heads = n_q_heads;
    p.kv_heads = kv->n_kv_heads;
    p.group = n_q_heads / kv->n_kv_heads;
    p.head_dim = kv->head_dim;
    p.scale_log2 = scale * 1.4426950408889634f;
    const long long tasks = (long long)p.b.n_rows * n_q_heads;
    const cudaError_t e = ops::launch(patt::rows_kernel, dim3((unsigned)std::min<long long>((tasks + 3) / 4, 1 << 20)), 128, 0, 1, (cudaStream_t)cuda_stream, p);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return ops::fail(S2D2_ERR_CUDA, "%s: %s", op, cudaGetErrorString(e));
    }
    return S2D2_OK;
}
