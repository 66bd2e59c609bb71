// MXFP4: quantisation, its inverse, and the host side of the products (kernels in mxfp4_tc.cuh).
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "mxfp4_tc.cuh"
#include "ops_host.h"

namespace s2d2 {
namespace {

constexpr int QT = 256;              // threads of the element-wise kernels
constexpr int QUAD = 128;            // elements under one 32-bit word of scale bytes: 4 blocks, 16 threads x 8 elements
constexpr int QROWS = QT / 32;       // rows of a block

struct QuantParams {
    const void* x;                   // quantise: input;  dequantise: output
    long long ld;
    long long rows;
    int cols;
    int quads;                       // words of scale bytes per row
    long long code_ld;               // bytes of codes per row
    uint8_t* codes;
    uint8_t* scales;
    int vec;                         // rows of x are 16-byte aligned
};

__host__ __device__ __forceinline__ size_t scale_word(long long row, int quad, int quads) {      // byte offset of 4 scale bytes
    return ((size_t)(row / 128) * quads + quad) * 512 + (size_t)(row % 32) * 16 + (size_t)(row % 128) / 32 * 4;
}

// Eight elements as they stand in memory, 16-byte aligned.
template <typename T>
struct Eight {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load_stream(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = __ldcs((const uint4*)p + i);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void load_shared(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = *((const uint4*)p + i);
    }
    __device__ __forceinline__ void values(float* v) const {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (sizeof(T) == 4) {
                    v[4 * i + e] = __uint_as_float(u[e]);
                } else {
                    v[2 * e] = __uint_as_float(u[e] << 16);
                    v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
                }
            }
        }
    }
};

__device__ __forceinline__ float load_stream_one(const float* p) { return __ldcs(p); }
// (as a whole number: the load of a bf16 itself is no volatile one, and may be moved in front of pdl_wait)
__device__ __forceinline__ bf16 load_stream_one(const bf16* p) { return __ushort_as_bfloat16(__ldcs((const unsigned short*)p)); }

// The larger magnitude; a NaN if there is one.
__device__ __forceinline__ float max_magnitude(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(fabsf(a)), "f"(fabsf(b)), "f"(fabsf(c)));
    return d;
}
__device__ __forceinline__ void mul2(float& a, float& b, float c) {      // two products in one instruction
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(a), "+f"(b)
        : "f"(c));
}
// Eight e2m1 codes, element 0 in the lowest nibble: round to nearest, ties to even, saturating.
__device__ __forceinline__ uint32_t e2m1x8(const float* v) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// and back, as four pairs of fp16 (exact)
__device__ __forceinline__ void e2m1x8_values(uint32_t codes, float* v) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// A warp takes STEPS x 256 elements of a row, all of its loads in flight at once, 16 threads per 128 elements: four threads share
// a block.  Scale and quotient are exact: the scale is a power of two.  Should be memory bound; what it has to watch is the
// number of instructions (15 per element took 31 us for 12288 x 4096 bf16, about 7 take the time of the copy).  Rows that are not
// aligned to 16 bytes, and a row's end, go through shared memory: 32 consecutive elements per load (loads of each thread's own eight
// took three times as long).  Rows that pad the last scale tile get zeros.
// WHOLE: every warp's elements are whole and aligned (the other path costs registers: 42 us both ways instead of 38).
template <typename T, int STEPS, bool WHOLE>
__global__ void __launch_bounds__(QT) quantize_kernel(const QuantParams p) {
    __shared__ alignas(16) T staged[WHOLE ? 1 : QROWS][2 * QUAD];
    pdl_wait();
    pdl_launch();
    const int lane = threadIdx.x & 31, sub = lane & 15;
    const long long row = (long long)blockIdx.x * QROWS + (threadIdx.x >> 5);
    const int quad0 = (int)blockIdx.y * (2 * STEPS) + (lane >> 4), c0 = quad0 * QUAD + sub * 8;
    const bool inside = row < p.rows;
    const int left = inside ? p.cols - c0 : -(1 << 24);                 // elements from c0 on; none in a row that pads the tile
    const int w0 = (int)blockIdx.y * (2 * STEPS) * QUAD;            // first element of the warp
    const T* x = (const T*)p.x + (inside ? row * p.ld : 0) + w0;
    const int n = inside ? p.cols - w0 : 0;                         // elements of the row from there on
    // whole and aligned, or element by element: lane, lane + 32, ...
    const bool direct = WHOLE || (p.vec && n >= STEPS * 2 * QUAD);
    Eight<T> in[STEPS];
    T one[STEPS][8];
    if (direct) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            if (inside) in[i].load_stream(x + i * (2 * QUAD) + lane * 8);
            else in[i].clear();
        }
    } else {
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int e = i * (2 * QUAD) + j * 32 + lane;
                one[i][j] = e < n ? load_stream_one(x + e) : from_f32<T>(0.f);
            }
    }
    uint32_t* codes = (uint32_t*)(p.codes + (inside ? row * p.code_ld : 0) + c0 / 2);
    uint32_t* scales = (uint32_t*)(p.scales + scale_word(row, quad0, p.quads));
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        if (!direct) {
            T* stage = (T*)staged[threadIdx.x >> 5];
#pragma unroll
            for (int j = 0; j < 8; ++j) stage[j * 32 + lane] = one[i][j];
            __syncwarp();
            in[i].load_shared(stage + lane * 8);
            __syncwarp();
        }
        float v[8];
        in[i].values(v);
        float m = max_magnitude(v[0], v[1], v[2]);
        m = max_magnitude(m, v[3], v[4]);
        m = max_magnitude(m, v[5], v[6]);
        uint32_t a = __float_as_uint(max_magnitude(m, v[7], v[7]));     // infinities and NaN stay on top as integers
        a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
        a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
        const int exponent = (int)(a >> 23);                       // biased; 0 for zero and for subnormals
        const bool bad = exponent == 255;
        const int byte = bad ? 255 : max(exponent - 2, 0);
        const float inverse = __uint_as_float((uint32_t)(254 - (bad ? 127 : byte)) << 23);       // 2^(127 - byte)
#pragma unroll
        for (int e = 0; e < 8; e += 2) mul2(v[e], v[e + 1], inverse);
        // (a row ends with a whole block: behind the last element its threads store zeros)
        if (left - i * (2 * QUAD) > -(int)(c0 & 31)) codes[i * QUAD / 4] = bad ? 0u : e2m1x8(v);
        uint32_t word = (uint32_t)byte << (8 * (sub >> 2));
        if (left - i * (2 * QUAD) <= -(int)(c0 & 31)) word = 0;
        word |= __shfl_xor_sync(0xffffffffu, word, 4);
        word |= __shfl_xor_sync(0xffffffffu, word, 8);
        if (sub == 0 && quad0 + 2 * i < p.quads) scales[i * 2 * 128] = word;
    }
}

template <typename T, int STEPS>
__global__ void __launch_bounds__(QT) dequantize_kernel(const QuantParams p) {
    __shared__ alignas(16) T staged[QROWS][2 * QUAD];
    pdl_wait();
    pdl_launch();
    const int lane = threadIdx.x & 31, sub = lane & 15;
    const long long row = (long long)blockIdx.x * QROWS + (threadIdx.x >> 5);
    const int quad0 = (int)blockIdx.y * (2 * STEPS) + (lane >> 4), c0 = quad0 * QUAD + sub * 8, left = p.cols - c0;
    if (row >= p.rows) return;
    const uint32_t* in = (const uint32_t*)(p.codes + row * p.code_ld + c0 / 2);
    const uint8_t* scales = p.scales + scale_word(row, quad0, p.quads) + (sub >> 2);
    uint32_t codes[STEPS], byte[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const bool some = left > i * (2 * QUAD);
        codes[i] = some ? __ldcs(in + i * QUAD / 4) : 0u;
        byte[i] = some ? scales[i * 2 * 512] : 0u;      // (not through the read-only path: the kernel in front may write them while this one begins)
    }
    const int w0 = (int)blockIdx.y * (2 * STEPS) * QUAD, n = p.cols - w0;
    const bool direct = p.vec && n >= STEPS * 2 * QUAD;             // whole and aligned; else through shared memory, 32 elements per store
    T* y = (T*)const_cast<void*>(p.x) + row * p.ld + w0;
#pragma unroll
    for (int i = 0; i < STEPS; ++i, y += 2 * QUAD) {
        const float scale = __uint_as_float(byte[i] == 255 ? 0x7fffffffu : byte[i] ? byte[i] << 23 : 0x00400000u);
        float v[8];
        e2m1x8_values(codes[i], v);
#pragma unroll
        for (int e = 0; e < 8; e += 2) mul2(v[e], v[e + 1], scale);
        uint4 w[sizeof(T) / 2];
        if (sizeof(T) == 4) {
            w[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
            w[sizeof(T) / 2 - 1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
        } else {
            uint32_t h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
                h[e] = *reinterpret_cast<const uint32_t*>(&b);
            }
            w[0] = make_uint4(h[0], h[1], h[2], h[3]);
        }
        if (direct) {
#pragma unroll
            for (int j = 0; j < (int)sizeof(T) / 2; ++j) __stcs((uint4*)(y + lane * 8) + j, w[j]);
        } else {
            T* stage = (T*)staged[threadIdx.x >> 5];
#pragma unroll
            for (int j = 0; j < (int)sizeof(T) / 2; ++j) *((uint4*)(stage + lane * 8) + j) = w[j];
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i * (2 * QUAD) + j * 32 + lane < n) __stcs(y + j * 32 + lane, stage[j * 32 + lane]);
            __syncwarp();
        }
    }
}

constexpr long long MAX_COLS = 1 << 20;

int check_shape(const char* op, long long rows, long long cols) {
    if (rows < 0 || rows > S2D2_MXFP4_MAX_DIM) return ops::fail(S2D2_ERR_INVALID, "%s: rows must be in 0..%d", op, S2D2_MXFP4_MAX_DIM);
    if (cols < 1 || cols > MAX_COLS) return ops::fail(S2D2_ERR_INVALID, "%s: columns must be in 1..%lld", op, MAX_COLS);
    return S2D2_OK;
}

int elementwise(const char* op, bool inverse, const void* x, int dtype, long long rows, long long cols, long long ld, const void* codes,
                const void* scales, cudaStream_t st) {
    ops::clear_error();
    if (dtype != S2D2_DTYPE_F32 && dtype != S2D2_DTYPE_BF16) return ops::fail(S2D2_ERR_INVALID, "%s: dtype", op);
    if (int rc = check_shape(op, rows, cols)) return rc;
    if (ld < cols || ld > (1LL << 40)) return ops::fail(S2D2_ERR_INVALID, "%s: row_stride must be in cols..2^40", op);
    const ops::Device* dev;
    if (int rc = ops::device(&dev)) return rc;
    if (rows == 0) return S2D2_OK;
    const size_t size = dtype == S2D2_DTYPE_F32 ? 4 : 2;
    if (int rc = ops::check_ptr(dev, x, size, inverse ? "y" : "x")) return rc;
    if (int rc = ops::check_ptr(dev, codes, 16, "codes")) return rc;
    if (int rc = ops::check_ptr(dev, scales, 16, "scales")) return rc;
    QuantParams p;
    p.x = x;
    p.ld = ld;
    p.rows = rows;
    p.cols = (int)cols;
    const long long blocks = (cols + 31) / 32;
    p.quads = (int)((blocks + 3) / 4);
    p.code_ld = blocks * 16;
    p.codes = (uint8_t*)const_cast<void*>(codes);
    p.scales = (uint8_t*)const_cast<void*>(scales);
    p.vec = ((uintptr_t)x & 15) == 0 && (ld * size) % 16 == 0;
    const long long row_blocks = ((inverse ? rows : (rows + 127) / 128 * 128) + QROWS - 1) / QROWS;      // at most 2^19
    // four steps per warp once that many blocks fill the GPU (12288 x 4096 bf16, both ways: 38 us, 57 with one);
    // one step for small matrices (333 x 2049 fp32, both ways: 3.4 us, 4.8 with four)
    const int steps = row_blocks * ((p.quads + 7) / 8) >= 8LL * dev->n_sms ? 4 : 1;
    const dim3 grid((unsigned)row_blocks, (unsigned)((p.quads + 2 * steps - 1) / (2 * steps)));           // at most 2^12 along y
    const bool whole = p.vec && cols % (steps * 2 * QUAD) == 0;
    void (*kernel)(QuantParams);
    if (dtype == S2D2_DTYPE_F32)
        kernel = inverse      ? (steps == 4 ? dequantize_kernel<float, 4> : dequantize_kernel<float, 1>)
                 : steps == 4 ? (whole ? quantize_kernel<float, 4, true> : quantize_kernel<float, 4, false>)
                              : (whole ? quantize_kernel<float, 1, true> : quantize_kernel<float, 1, false>);
    else
        kernel = inverse      ? (steps == 4 ? dequantize_kernel<bf16, 4> : dequantize_kernel<bf16, 1>)
                 : steps == 4 ? (whole ? quantize_kernel<bf16, 4, true> : quantize_kernel<bf16, 4, false>)
                              : (whole ? quantize_kernel<bf16, 1, true> : quantize_kernel<bf16, 1, false>);
    const cudaError_t e = ops::launch(kernel, grid, QT, 0, 1, st, p);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return ops::fail(S2D2_ERR_CUDA, "%s: %s", op, cudaGetErrorString(e));
    }
    return S2D2_OK;
}

// Codes of a [rows, K] matrix in boxes of box_rows rows x 256 elements; what lies outside the matrix reads as zero.
int encode_codes(const ops::Device* dev, CUtensorMap* map, const void* codes, int rows, int K, int box_rows) {
    const cuuint64_t row_bytes = (cuuint64_t)((K + 31) / 32) * 16;
    cuuint64_t dims[2] = {row_bytes, (cuuint64_t)rows}, strides[1] = {row_bytes};
    cuuint32_t box[2] = {(cuuint32_t)mx::KBYTES, (cuuint32_t)box_rows}, step[2] = {1, 1};
    const CUresult r = dev->encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(codes), dims, strides, box, step,
                                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? S2D2_OK : ops::fail(S2D2_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}

constexpr int MAX_SMEM = 224 * 1024;     // 3 KB of an SM are left to kernels without tensor memory

int check_operands(const ops::Device* dev, const void* xc, const void* xs, const void* wc, const void* ws) {
    if (int rc = ops::check_ptr(dev, xc, 16, "x_codes")) return rc;
    if (int rc = ops::check_ptr(dev, xs, 16, "x_scales")) return rc;
    if (int rc = ops::check_ptr(dev, wc, 16, "w_codes")) return rc;
    return ops::check_ptr(dev, ws, 16, "w_scales");
}
int check_product_shape(const char* op, int M, int N, int K) {
    if (M < 0 || M > S2D2_MXFP4_MAX_DIM) return ops::fail(S2D2_ERR_INVALID, "%s: M must be in 0..%d", op, S2D2_MXFP4_MAX_DIM);
    if (N < 1 || N > S2D2_MXFP4_MAX_DIM) return ops::fail(S2D2_ERR_INVALID, "%s: N must be in 1..%d", op, S2D2_MXFP4_MAX_DIM);
    if (K < 1 || K > MAX_COLS) return ops::fail(S2D2_ERR_INVALID, "%s: K must be in 1..%lld", op, MAX_COLS);
    return S2D2_OK;
}

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

// Scale tiles of a [rows, K] matrix as rows of 512 bytes, two at a time (one k-block).
int encode_scales(const ops::Device* dev, CUtensorMap* map, const void* scales, int rows, int K) {
    cuuint64_t dims[2] = {mx::SF_TILE / 4, (cuuint64_t)ceil_div(rows, 128) * ceil_div(ceil_div(K, 32), 4)}, strides[1] = {mx::SF_TILE};
    cuuint32_t box[2] = {mx::SF_TILE / 4, 2}, step[2] = {1, 1};
    const CUresult r = dev->encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(scales), dims, strides, box, step,
                                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? S2D2_OK : ops::fail(S2D2_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", (int)r);
}

struct Plan {
    mx::Params p = {};
    int cg = 1, grid = 0, smem = 0;
};

bool two_accumulators(int T, int sf_tiles) { return mx::used_columns(T, sf_tiles, 2) <= 512; }

// Accumulators, tensor-memory columns, shared memory and ring depth once tiles, T, sf_tiles and splits are known.
void finish_plan(Plan& plan, long long tiles_per_cluster, int stages_wanted) {
    mx::Params& p = plan.p;
    p.n_acc = tiles_per_cluster > 1 && two_accumulators(p.T, p.sf_tiles) ? 2 : 1;
    const int used = mx::used_columns(p.T, p.sf_tiles, p.n_acc);
    p.tmem_cols = 32;
    while ((int)p.tmem_cols < used) p.tmem_cols *= 2;
    const int sbytes = mx::stage_bytes(plan.cg, p.a_box, p.T, p.sf_tiles), fixed = 1024 + (int)sizeof(mx::Control),
              pad = mx::ring_bytes(plan.cg, 0, p.a_box, p.T, p.sf_tiles);
    // clusters keep to half an SM's memory, so that the set-up of the next kernel may overlap
    const int room = (p.splits > 1 ? 113 * 1024 : MAX_SMEM) - fixed;
    p.stages = std::max(2, std::min(std::min(mx::MAX_STAGES, (room - pad) / sbytes), stages_wanted));
    p.control_at = std::max(mx::ring_bytes(plan.cg, p.stages, p.a_box, p.T, p.sf_tiles), p.splits > 1 ? p.T * mx::ROWS * 4 : 0);
    plan.smem = std::max(fixed + p.control_at, mx::min_smem(p.tmem_cols));
}

// Clock cycles of a tile, for choosing T.  A k-block costs the larger of what the SM takes in (64 bytes a cycle) and what its tensor
// core multiplies (2 T cycles for 128 x T x 256); without a second accumulator the next tile waits for the read of this one.
double tile_cycles(int cg, int a_box, int T, int kb_total) {
    const int sf_tiles = T > 128 ? 2 : 1;
    const double in = mx::stage_bytes(cg, a_box, T, sf_tiles) / 64.0;
    return kb_total * std::max(in, 2.0 * T) + 400 + (two_accumulators(T, sf_tiles) ? 0 : 600);
}

void plan_product(Plan& plan, int n_sms, int M, int N, int K) {
    mx::Params& p = plan.p;
    p.a_rows = N;
    p.b_rows = M;
    p.K = K;
    p.kb_total = ceil_div(K, mx::KBLOCK);
    p.quads = ceil_div(ceil_div(K, 32), 4);
    p.splits = 1;
    p.a_box = mx::ROWS;
    if (M > 128) {
        // Pairs of CTAs, if the tiles occupy at least half of them: T by the number of waves times a tile's length.
        const int pairs = n_sms / 2, a_tiles = ceil_div(N, 256);
        double best = 1e30;
        for (int T = 128; T <= 256; T += 64) {
            const int width = M < T ? (M + 31) / 32 * 32 : T;                                  // one tile: any width
            const double cost = (double)ceil_div((long long)a_tiles * ceil_div(M, T), pairs) * tile_cycles(2, mx::ROWS, width, p.kb_total);
            if (cost < best) best = cost, p.T = width;
        }
        p.a_tiles = a_tiles;
        p.b_tiles = ceil_div(M, p.T);
        if ((long long)p.a_tiles * p.b_tiles * 2 >= pairs) {
            plan.cg = 2;
            p.sf_tiles = p.T > 128 ? 2 : 1;        // tiles start at multiples of 128, or of 64 with T = 192
            const long long tiles = (long long)p.a_tiles * p.b_tiles;
            const int clusters = (int)std::min<long long>(tiles, pairs);
            plan.grid = clusters * 2;
            finish_plan(plan, (tiles + clusters - 1) / clusters, mx::MAX_STAGES);
            return;
        }
    }
    plan.cg = 1;
    p.T = std::min(128, (M + 15) / 16 * 16);
    p.a_tiles = ceil_div(N, mx::ROWS);
    p.b_tiles = ceil_div(M, p.T);
    p.sf_tiles = 1;                            // T = 128, or one tile
    const long long tiles = (long long)p.a_tiles * p.b_tiles;
    // Few tiles: the CTAs of a cluster share a tile's k-blocks.  Measured: 0.27 us per k-block in a CTA, and 0.6 us plus 7 ns per
    // token row (12 ns with eight CTAs) for the sum over the cluster.  (M 1, N 4096, K 4096: 7.7 us unsplit, 5.6 us with four;
    // M 64: 8.2 and 7.7; M 128, N 1024: 8.8 and 6.8; M 64, N 4096, K 2048 stays unsplit.)  Every cluster has to be at work at once;
    // eight CTAs of a whole SM each do not fit everywhere.
    double best = 1e30;
    for (int s = 1; s <= 8 && s <= p.kb_total; s *= 2) {
        if (s > 1 && tiles * s * (s == 8 && p.T > 64 ? 4 : 3) > 3 * n_sms) break;
        const double cost = 0.27 * ceil_div(p.kb_total, s) + (s > 1 ? 0.6 + p.T * (s == 8 ? 0.012 : 0.007) : 0.0);
        if (cost < best) best = cost, p.splits = s;
    }
    const int clusters = (int)std::min<long long>(tiles, p.splits > 1 ? tiles : n_sms);
    plan.grid = clusters * p.splits;
    const long long per_cluster = (tiles + clusters - 1) / clusters;
    finish_plan(plan, per_cluster, (int)std::min<long long>(mx::MAX_STAGES, per_cluster * ceil_div(p.kb_total, p.splits)));
}

constexpr int SCORE_MAX_ITEMS = 320;       // (A tile, range) items, unless there are more A tiles

int score_cg(int M) { return M > 128 ? 2 : 1; }
int score_max_ranges(int a_tiles, int N) { return std::max(1, std::min(ceil_div(N, 64), SCORE_MAX_ITEMS / a_tiles)); }

void plan_score(Plan& plan, int n_sms, int M, int N, int K) {
    mx::Params& p = plan.p;
    p.a_rows = M;
    p.b_rows = N;
    p.K = K;
    p.kb_total = ceil_div(K, mx::KBLOCK);
    p.quads = ceil_div(ceil_div(K, 32), 4);
    p.splits = 1;
    plan.cg = score_cg(M);
    p.a_tiles = ceil_div(M, mx::ROWS * plan.cg);
    p.a_box = std::min(mx::ROWS, (M + 7) / 8 * 8);
    // Ranges of the head's rows per A tile, and the tile's T, by the time of the busiest cluster.
    const int slots = n_sms / plan.cg;
    double best = 1e30;
    for (int T = 64; T <= 256; T += 64) {
        const int unit = T % 128 ? 64 : 128, units = ceil_div(N, unit);
        if (plan.cg == 1 && T > 192) break;
        const double full = tile_cycles(plan.cg, p.a_box, T, p.kb_total);
        // as many ranges as fill one to four waves of clusters
        for (int w = ceil_div(p.a_tiles, slots), last = w + 3; w <= last; ++w) {
            const int r = std::max(1, std::min({(int)((long long)slots * w / p.a_tiles), units, score_max_ranges(p.a_tiles, N)}));
            const int waves = ceil_div((long long)p.a_tiles * r, slots), len = ceil_div(units, r) * unit;
            // a single CTA loads no more of its last tile than the range holds
            const int rest = plan.cg == 1 && len % T ? len % T : T;
            const double cost = waves * ((ceil_div(len, T) - 1) * full + tile_cycles(plan.cg, p.a_box, rest, p.kb_total) + 1000);
            if (cost < best) best = cost, p.ranges = r, p.T = T, p.unit = unit;
        }
    }
    p.sf_tiles = p.T > 128 ? 2 : 1;            // T = 64 and 192 start at multiples of 64, T = 128 and 256 at multiples of 128
    p.b_tiles = 0;
    const long long items = (long long)p.a_tiles * p.ranges;
    const int clusters = (int)std::min<long long>(items, slots);
    plan.grid = clusters * plan.cg;
    finish_plan(plan, 2, mx::MAX_STAGES);
}

template <int CG, bool SCORE, int NQ>
int launch_product(const Plan& plan, const CUtensorMap* maps, cudaStream_t st) {
    const cudaError_t e = ops::launch(mx::product_kernel<CG, SCORE, NQ>, dim3((unsigned)plan.grid), mx::THREADS, plan.smem,
                                      CG * plan.p.splits, st, maps[0], maps[1], maps[2], maps[3], maps[4], plan.p);
    if (e == cudaSuccess) return S2D2_OK;
    cudaGetLastError();
    return ops::fail(S2D2_ERR_CUDA, "mxfp4 product: %s", cudaGetErrorString(e));
}

// Test tap: waits of this host thread's next product (0: as they are), and whether its codes are held back.
thread_local uint32_t g_wait_limit;
thread_local int g_withhold;

template <bool SCORE>
int run_product(const ops::Device* dev, Plan& plan, const void* ac, const void* as, const void* bc, const void* bs, cudaStream_t st) {
    mx::Params& p = plan.p;
    p.wait_limit = g_wait_limit ? g_wait_limit : tc::WAIT_LIMIT;
    p.withhold = g_withhold;
    g_wait_limit = 0;
    g_withhold = 0;
    CUtensorMap maps[5];
    if (int rc = encode_codes(dev, &maps[0], ac, p.a_rows, p.K, p.a_box)) return rc;
    if (int rc = encode_codes(dev, &maps[1], bc, p.b_rows, p.K, p.T / plan.cg)) return rc;
    if (SCORE && plan.cg == 1) {
        if (int rc = encode_codes(dev, &maps[2], bc, p.b_rows, p.K, mx::CUT)) return rc;
    } else {
        maps[2] = maps[1];
    }
    if (int rc = encode_scales(dev, &maps[3], as, p.a_rows, p.K)) return rc;
    if (int rc = encode_scales(dev, &maps[4], bs, p.b_rows, p.K)) return rc;
    if (plan.cg == 1) return p.T <= 64 ? launch_product<1, SCORE, 1>(plan, maps, st) : launch_product<1, SCORE, 3>(plan, maps, st);
    return p.T <= 192 ? launch_product<2, SCORE, 3>(plan, maps, st) : launch_product<2, SCORE, 4>(plan, maps, st);
}

}  // namespace

cudaError_t ops::load_mxfp4_kernels() {
    const cudaError_t all[] = {load(quantize_kernel<float, 1, false>), load(quantize_kernel<float, 4, false>), load(quantize_kernel<bf16, 1, false>),
                               load(quantize_kernel<bf16, 4, false>), load(quantize_kernel<float, 1, true>), load(quantize_kernel<float, 4, true>),
                               load(quantize_kernel<bf16, 1, true>), load(quantize_kernel<bf16, 4, true>), load(dequantize_kernel<float, 1>), load(dequantize_kernel<float, 4>),
                               load(dequantize_kernel<bf16, 1>), load(dequantize_kernel<bf16, 4>),
                               load(mx::product_kernel<1, false, 1>, MAX_SMEM), load(mx::product_kernel<1, false, 3>, MAX_SMEM),
                               load(mx::product_kernel<2, false, 3>, MAX_SMEM), load(mx::product_kernel<2, false, 4>, MAX_SMEM),
                               load(mx::product_kernel<1, true, 1>, MAX_SMEM), load(mx::product_kernel<1, true, 3>, MAX_SMEM),
                               load(mx::product_kernel<2, true, 3>, MAX_SMEM), load(mx::product_kernel<2, true, 4>, MAX_SMEM),
                               load(mx::score_parts_kernel)};
    for (cudaError_t e : all)
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}
}  // namespace s2d2

using namespace s2d2;

extern "C" int s2d2_mxfp4_sizes(int64_t rows, int64_t cols, int64_t* codes_bytes, int64_t* scales_bytes) {
    ops::clear_error();
    if (!codes_bytes || !scales_bytes) return ops::fail(S2D2_ERR_INVALID, "mxfp4_sizes: null pointer");
    if (int rc = check_shape("mxfp4_sizes", rows, cols)) return rc;
    const int64_t blocks = (cols + 31) / 32;
    *codes_bytes = rows * blocks * 16;
    *scales_bytes = (rows + 127) / 128 * ((blocks + 3) / 4) * 512;
    return S2D2_OK;
}

extern "C" int s2d2_mxfp4_quantize(const void* d_x, int32_t dtype, int64_t rows, int64_t cols, int64_t row_stride, void* d_codes,
                                   void* d_scales, void* cuda_stream) {
    return elementwise("mxfp4_quantize", false, d_x, dtype, rows, cols, row_stride, d_codes, d_scales, (cudaStream_t)cuda_stream);
}

extern "C" int s2d2_mxfp4_dequantize(const void* d_codes, const void* d_scales, int64_t rows, int64_t cols, void* d_y, int32_t dtype,
                                     int64_t row_stride, void* cuda_stream) {
    return elementwise("mxfp4_dequantize", true, d_y, dtype, rows, cols, row_stride, d_codes, d_scales, (cudaStream_t)cuda_stream);
}

extern "C" int s2d2_mxfp4_gemm(const void* d_x_codes, const void* d_x_scales, const void* d_w_codes, const void* d_w_scales, void* d_y,
                               int32_t y_dtype, int32_t M, int32_t N, int32_t K, int64_t y_stride, float scale, void* cuda_stream) {
    ops::clear_error();
    if (y_dtype != S2D2_DTYPE_F32 && y_dtype != S2D2_DTYPE_BF16) return ops::fail(S2D2_ERR_INVALID, "mxfp4_gemm: y_dtype");
    if (int rc = check_product_shape("mxfp4_gemm", M, N, K)) return rc;
    if (y_stride < N || y_stride > (1LL << 40)) return ops::fail(S2D2_ERR_INVALID, "mxfp4_gemm: y_stride must be in N..2^40");
    const ops::Device* dev;
    if (int rc = ops::device(&dev)) return rc;
    if (M == 0) return S2D2_OK;
    if (int rc = check_operands(dev, d_x_codes, d_x_scales, d_w_codes, d_w_scales)) return rc;
    if (int rc = ops::check_ptr(dev, d_y, y_dtype == S2D2_DTYPE_F32 ? 4 : 2, "y")) return rc;
    Plan plan;
    plan_product(plan, dev->n_sms, M, N, K);
    plan.p.y = d_y;
    plan.p.y_bf16 = y_dtype == S2D2_DTYPE_BF16;
    plan.p.ldy = y_stride;
    plan.p.scale = scale;
    plan.p.timeouts = dev->timeouts;
    return run_product<false>(dev, plan, d_w_codes, d_w_scales, d_x_codes, d_x_scales, (cudaStream_t)cuda_stream);
}

extern "C" int s2d2_mxfp4_score_workspace(int32_t M, int32_t N, int32_t K, int64_t* bytes) {
    ops::clear_error();
    if (!bytes) return ops::fail(S2D2_ERR_INVALID, "mxfp4_score_workspace: null pointer");
    if (int rc = check_product_shape("mxfp4_score_workspace", M, N, K)) return rc;
    const int rows = mx::ROWS * score_cg(M), a_tiles = ceil_div(M, rows);
    *bytes = M ? (int64_t)a_tiles * score_max_ranges(a_tiles, N) * 2 * rows * 16 : 0;
    return S2D2_OK;
}

extern "C" int s2d2_mxfp4_score(const void* d_x_codes, const void* d_x_scales, const void* d_w_codes, const void* d_w_scales, int32_t M,
                                int32_t N, int32_t K, float scale, const int32_t* d_tokens, float* d_logprob, float* d_lse,
                                float* d_entropy, void* d_ws, int64_t ws_bytes, void* cuda_stream) {
    ops::clear_error();
    if (int rc = check_product_shape("mxfp4_score", M, N, K)) return rc;
    if (!d_logprob && !d_lse && !d_entropy) return ops::fail(S2D2_ERR_INVALID, "mxfp4_score: no output");
    if (d_logprob && !d_tokens) return ops::fail(S2D2_ERR_INVALID, "mxfp4_score: log probability needs tokens");
    int64_t need = 0;
    if (int rc = s2d2_mxfp4_score_workspace(M, N, K, &need)) return rc;
    if (ws_bytes < need) return ops::fail(S2D2_ERR_INVALID, "mxfp4_score: the workspace needs %lld bytes", (long long)need);
    const ops::Device* dev;
    if (int rc = ops::device(&dev)) return rc;
    if (M == 0) return S2D2_OK;
    if (int rc = check_operands(dev, d_x_codes, d_x_scales, d_w_codes, d_w_scales)) return rc;
    const void* words[] = {d_tokens, d_logprob, d_lse, d_entropy};
    const char* names[] = {"tokens", "logprob", "lse", "entropy"};
    for (int i = 0; i < 4; ++i)
        if (words[i])
            if (int rc = ops::check_ptr(dev, words[i], 4, names[i])) return rc;
    if (int rc = ops::check_ptr(dev, d_ws, 16, "workspace")) return rc;
    Plan plan;
    plan_score(plan, dev->n_sms, M, N, K);
    plan.p.scale = scale;
    plan.p.timeouts = dev->timeouts;
    plan.p.tokens = d_tokens;
    plan.p.parts = (float4*)d_ws;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    if (int rc = run_product<true>(dev, plan, d_x_codes, d_x_scales, d_w_codes, d_w_scales, st)) return rc;
    const cudaError_t e = ops::launch(mx::score_parts_kernel, dim3((unsigned)M), 128, 0, 1, st, plan.p, mx::ROWS * plan.cg,
                                      d_logprob, d_lse, d_entropy);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return ops::fail(S2D2_ERR_CUDA, "mxfp4_score: %s", cudaGetErrorString(e));
    }
    return S2D2_OK;
}

extern "C" int s2d2_debug_mxfp4_wait(uint32_t limit_polls, int32_t withhold) {
    ops::clear_error();
    if (limit_polls < 1 || limit_polls > (1u << 20)) return ops::fail(S2D2_ERR_INVALID, "debug_mxfp4_wait: limit_polls must be in 1..2^20");
    g_wait_limit = limit_polls;
    g_withhold = withhold != 0;
    return S2D2_OK;
}
