// Attention of a batch's new rows over a paged cache: s2d2_paged_attention.
#include <math.h>

#include "paged_attention_tc.cuh"

namespace s2d2 {
namespace {

constexpr int MAX_ROWS = 1 << 22;
constexpr long long MAX_LEN = 1 << 30;      // tokens of a sequence, and query vectors of a kv head

thread_local uint32_t g_wait_limit = tc::WAIT_LIMIT;
thread_local int g_withhold = 0;

int check_shape(const char* op, const s2d2_rows* rows, const s2d2_paged_kv* kv, int n_q_heads) {
    if (int rc = ops::check_rows(op, rows)) return rc;
    if (int rc = ops::check_kv(op, kv)) return rc;
    if (kv->head_dim > 128) return ops::fail(S2D2_ERR_UNSUPPORTED, "%s: head_dim must be at most 128", op);
    if (n_q_heads < 1 || n_q_heads > S2D2_MAX_HEADS || n_q_heads % kv->n_kv_heads)
        return ops::fail(S2D2_ERR_INVALID, "%s: n_q_heads must be a multiple of n_kv_heads, at most %d", op, S2D2_MAX_HEADS);
    if ((long long)rows->n_rows * (n_q_heads / kv->n_kv_heads) > MAX_LEN)
        return ops::fail(S2D2_ERR_UNSUPPORTED, "%s: n_rows * n_q_heads / n_kv_heads must be at most 2^30", op);
    if (rows->n_rows > MAX_ROWS) return ops::fail(S2D2_ERR_UNSUPPORTED, "%s: n_rows must be at most 2^22", op);
    if ((long long)rows->max_pages * kv->page_tokens > MAX_LEN) return ops::fail(S2D2_ERR_UNSUPPORTED, "%s: max_pages * page_tokens must be at most 2^30", op);
    return S2D2_OK;
}

// How the work is cut, from what the host knows.
struct Plan {
    int hdp, nh, gs, rows_half, ctas, stages, smem, control_at;
    bool joins;                      // an item may be cut
    long long ml_at, o_at, bytes;    // of the workspace
    double costs;                    // units, at most
};
Plan make_plan(const s2d2_rows* rows, const s2d2_paged_kv* kv, int n_q_heads) {
    Plan n;
    n.hdp = kv->head_dim > 64 ? 128 : 64;
    const int group = n_q_heads / kv->n_kv_heads;
    n.gs = std::min(group, patt::QTILE);
    while (group % n.gs) --n.gs;
    n.rows_half = patt::QTILE / n.gs;
    // items of one tile where no sequence has more rows, as far as the host knows
    n.nh = rows->max_rows <= n.rows_half ? 1 : 2;
    const long long most = std::max(1LL, ((long long)rows->max_pages * kv->page_tokens + patt::KEYS - 1) / patt::KEYS), per = n.nh * n.rows_half;
    const long long items = (rows->n_rows + per - 1) / per + std::min(rows->n_seqs, rows->n_rows);
    n.costs = (double)items * (double)(most + 1) * (n_q_heads / n.gs);
    n.ctas = (int)std::min<double>(patt::MAX_CTAS, std::max(1., (double)items * (double)most * (n_q_heads / n.gs)));
    n.joins = most > 1;
    const int stage = patt::KEYS * n.hdp * 2, q = n.nh * patt::QTILE * n.hdp * 2, most_smem = 227 * 1024 - 1024 - (int)sizeof(patt::Control);
    n.stages = std::min(patt::MAX_STAGES, (most_smem - q) / stage);
    n.control_at = q + n.stages * stage;
    // (at least 200 KB: no other CTA that takes tensor memory is on the SM, so taking all of it does not wait)
    n.smem = std::max(200 * 1024, 1024 + n.control_at + (int)sizeof(patt::Control));
    n.ml_at = n.ctas * 32LL;
    n.o_at = n.ml_at + (n.joins ? 2LL * n.ctas * patt::QTILE * n.nh * 8 : 0);      // (a multiple of 32)
    n.bytes = n.o_at + (n.joins ? 2LL * n.ctas * patt::QTILE * n.nh * n.hdp * 4 : 0);
    return n;
}

// Keys or values of a layer as [page][head][token][element] in boxes of up to 128 tokens x 64 elements; elements behind the head's read as zero.
int encode(const ops::Device* dev, CUtensorMap* map, const void* base, const s2d2_paged_kv* kv) {
    cuuint64_t dims[4] = {(cuuint64_t)kv->head_dim, (cuuint64_t)kv->page_tokens, (cuuint64_t)kv->n_kv_heads, (cuuint64_t)kv->n_pages};
    cuuint64_t strides[3] = {(cuuint64_t)kv->token_stride * 2, (cuuint64_t)kv->head_stride * 2, (cuuint64_t)kv->page_stride * 2};
    cuuint32_t box[4] = {64, (cuuint32_t)std::min(kv->page_tokens, patt::KEYS), 1, 1}, step[4] = {1, 1, 1, 1};
    const CUresult r = dev->encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, step,
                                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? S2D2_OK : ops::fail(S2D2_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}

// Queries as [row][head][element] in boxes of a tile's rows x heads x 64 elements.
int encode_q(const ops::Device* dev, CUtensorMap* map, const void* q, long long q_stride, int n_rows, int heads, int head_dim, const Plan& n) {
    cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)heads, (cuuint64_t)n_rows};
    cuuint64_t strides[2] = {(cuuint64_t)head_dim * 2, (cuuint64_t)q_stride * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)n.gs, (cuuint32_t)n.rows_half}, step[3] = {1, 1, 1};
    const CUresult r = dev->encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(q), dims, strides, box, step,
                                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? S2D2_OK : ops::fail(S2D2_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}

template <int HDP, int NH>
cudaError_t launch_tiles(const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v, const patt::TileParams& t, const Plan& n, cudaStream_t st) {
    cudaError_t e = ops::launch(patt::tile_kernel<HDP, NH>, dim3(n.ctas), patt::threads(NH), n.smem, 1, st, map_q, map_k, map_v, t);
    if (!e && n.joins) e = ops::launch(patt::join_kernel<HDP, NH>, dim3(n.ctas, 128 * NH / (patt::JOIN_WARPS * patt::join_vectors(NH))), 32 * patt::JOIN_WARPS, 0, 1, st, t);
    return e;
}

}  // namespace

namespace ops {
cudaError_t load_attention_kernels() {
    constexpr int most = 227 * 1024;
    cudaError_t e = load(patt::tile_kernel<64, 1>, most);
    if (!e) e = load(patt::tile_kernel<64, 2>, most);
    if (!e) e = load(patt::tile_kernel<128, 1>, most);
    if (!e) e = load(patt::tile_kernel<128, 2>, most);
    if (!e) e = load(patt::join_kernel<64, 1>);
    if (!e) e = load(patt::join_kernel<64, 2>);
    if (!e) e = load(patt::join_kernel<128, 1>);
    return e ? e : load(patt::join_kernel<128, 2>);
}
}  // namespace ops
}  // namespace s2d2

using namespace s2d2;

extern "C" int s2d2_paged_attention_workspace(const s2d2_rows* rows, const s2d2_paged_kv* kv, int32_t n_q_heads, int64_t* bytes) {
    ops::clear_error();
    const char* op = "paged_attention_workspace";
    if (!bytes) return ops::fail(S2D2_ERR_INVALID, "%s: bytes: null pointer", op);
    if (int rc = check_shape(op, rows, kv, n_q_heads)) return rc;
    *bytes = make_plan(rows, kv, n_q_heads).bytes;
    return S2D2_OK;
}

extern "C" int s2d2_paged_attention(const void* d_q, int64_t q_stride, void* d_out, int64_t out_stride, float* d_lse, int32_t n_q_heads,
                                    const s2d2_rows* rows, const s2d2_paged_kv* kv, int32_t mask_block, const uint64_t* d_row_mask,
                                    float scale, void* d_ws, int64_t ws_bytes, void* cuda_stream) {
    ops::clear_error();
    const char* op = "paged_attention";
    if (int rc = check_shape(op, rows, kv, n_q_heads)) return rc;
    const long long width = (long long)n_q_heads * kv->head_dim;
    if (q_stride < width || q_stride % 8 || q_stride >= (1LL << 39)) return ops::fail(S2D2_ERR_INVALID, "%s: q_stride must be a multiple of 8 from heads * head_dim on, below 2^39", op);
    if (out_stride < width || out_stride % 8 || out_stride > (1LL << 40)) return ops::fail(S2D2_ERR_INVALID, "%s: out_stride must be a multiple of 8 in heads * head_dim..2^40", op);
    if (mask_block < 0) return ops::fail(S2D2_ERR_INVALID, "%s: mask_block must not be negative", op);
    if (d_row_mask && mask_block) return ops::fail(S2D2_ERR_INVALID, "%s: mask_block must be 0 with row masks", op);
    if (!(scale > 0.f) || !isfinite(scale)) return ops::fail(S2D2_ERR_INVALID, "%s: scale must be positive", op);
    const Plan n = make_plan(rows, kv, n_q_heads);
    const bool work = rows->n_rows && rows->n_seqs;
    if (n.costs > 2e9) return ops::fail(S2D2_ERR_UNSUPPORTED, "%s: rows x max_pages: too much for one call", op);
    if (work && ws_bytes < n.bytes) return ops::fail(S2D2_ERR_INVALID, "%s: workspace of %lld bytes, needs %lld", op, (long long)ws_bytes, n.bytes);
    const ops::Device* dev;
    if (int rc = ops::device(&dev)) return rc;
    if (!work) return S2D2_OK;
    patt::TileParams t = {};
    patt::Params& p = t.a;
    if (int rc = ops::device_rows(dev, rows, kv, &p.b)) return rc;
    if (int rc = ops::device_kv(dev, kv, &p.c)) return rc;
    if (int rc = ops::check_ptr(dev, d_q, 16, "q")) return rc;
    if (int rc = ops::check_ptr(dev, d_out, 16, "out")) return rc;
    if (int rc = ops::check_ptr(dev, d_ws, 32, "workspace")) return rc;
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
    CUtensorMap map_q, map_k, map_v;
    if (int rc = encode_q(dev, &map_q, d_q, q_stride, rows->n_rows, n_q_heads, kv->head_dim, n)) return rc;
    if (int rc = encode(dev, &map_k, kv->d_k, kv)) return rc;
    if (int rc = encode(dev, &map_v, kv->d_v, kv)) return rc;
    t.ctas = n.ctas;
    t.stages = n.stages;
    t.control_at = n.control_at;
    t.gs = n.gs;
    t.vsub = p.group / n.gs;
    t.rows_half = n.rows_half;
    const uint32_t per = n.rows_half * n.nh;
    t.items_magic = per == 1 ? 0u : (uint32_t)((0x100000000ULL + per - 1) / per);
    // lanes per sequence when units are counted: as many as it may have items, as long as one round takes all sequences
    t.seq_lanes = 1;
    while (t.seq_lanes < 32 && (long long)t.seq_lanes * per < rows->max_rows && (long long)rows->n_seqs * t.seq_lanes * 2 <= 32) t.seq_lanes *= 2;
    t.split = (int4*)d_ws;
    t.part_ml = (float2*)((char*)d_ws + n.ml_at);
    t.part_o = (float*)((char*)d_ws + n.o_at);
    t.out_32 = ((uintptr_t)d_out & 31) == 0 && out_stride % 16 == 0 && kv->head_dim % 16 == 0;
    t.timeouts = dev->timeouts;
    t.wait_limit = g_wait_limit;
    t.withhold = g_withhold;
    g_wait_limit = tc::WAIT_LIMIT;
    g_withhold = 0;
    const auto launch = n.hdp == 128 ? (n.nh == 1 ? launch_tiles<128, 1> : launch_tiles<128, 2>) : (n.nh == 1 ? launch_tiles<64, 1> : launch_tiles<64, 2>);
    const cudaError_t e = launch(map_q, map_k, map_v, t, n, (cudaStream_t)cuda_stream);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return ops::fail(S2D2_ERR_CUDA, "%s: %s", op, cudaGetErrorString(e));
    }
    return S2D2_OK;
}

extern "C" int s2d2_debug_attention_wait(uint32_t limit_polls, int32_t withhold) {
    ops::clear_error();
    if (limit_polls < 1 || limit_polls > 1u << 20) return ops::fail(S2D2_ERR_INVALID, "debug_attention_wait: limit_polls must be in 1..2^20");
    g_wait_limit = limit_polls;
    g_withhold = withhold != 0;
    return S2D2_OK;
}
