// Tensor-core products of MXFP4 operands (sm_100a, tcgen05 kind::mxf4).
//
//   Y[m, n] = scale * sum_k X[m, k] W[n, k],   X and W in blocks of 32 elements with one power-of-two scale each
//
// The tensor core multiplies e2m1 codes, applies both scales and sums in fp32, so nothing is widened on the way: a
// weight costs 17/32 byte of HBM instead of 2.  As in the bf16 kernels the weights are the MMA's "M" operand (128 rows)
// and the tokens its "N" operand (16..128 rows): the accumulator's lanes are output features, so an epilogue warp
// stores 32 consecutive elements of one output row, whatever that row's alignment.
//
// One k-block of a stage is 256 elements = 128 bytes of codes per row (one 128-byte swizzle row, four MMAs of 64) and
// 8 scales per row = two 512-byte scale tiles.  Scales go from shared memory to tensor memory by tcgen05.cp (32 lanes x 16
// bytes, repeated for the four lane quarters): column c + r / 32 of lane r % 32 then holds the four scales of row r of that
// tile, and an MMA of 64 elements takes the lower or the upper two of them (scale id 0 or 2).
#pragma once
#include "ops_host.h"
#include "tc_ptx.cuh"

namespace s2d2 {
namespace mx {

using namespace tc;

constexpr int ROWS = 128;            // weight rows of a tile (MMA M of one CTA)
constexpr int KBLOCK = 256;          // elements of a stage's k-block
constexpr int KBYTES = KBLOCK / 2;
constexpr int MMA_K = 64;
constexpr int SF_TILE = 512;         // bytes of one scale tile: 128 rows x 4 blocks
constexpr int THREADS = 128;

struct GemmParams {
    void* y;
    int y_bf16;
    int M, N, K;
    long long ldy;
    float scale;
    int T;                           // token rows per tile (multiple of 16; of 32 if there are several tiles)
    int x_tiles;                     // scale tiles that the token rows of a tile touch (1 or 2)
    int stages;
    int splits;                      // k splits = CTAs per cluster
    int kb_total;                    // k-blocks
    int quads;                       // scale tiles along k
    int m_tiles;
    int control_at;                  // byte offset of the barriers behind the ring
    const uint8_t* w_scales;
    const uint8_t* x_scales;
    int* status;
};

__host__ __device__ __forceinline__ int stage_bytes(int T, int x_tiles) {
    return ROWS * KBYTES + T * KBYTES + (1 + x_tiles) * 2 * SF_TILE;
}

__device__ __forceinline__ uint64_t desc_sw128(uint32_t smem_addr) {      // K-major rows of 128 bytes, 128-byte swizzle
    return (uint64_t)((smem_addr & 0x3FFFF) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t desc_scales(uint32_t smem_addr) {     // 8 rows of 16 bytes are contiguous, no swizzle
    return (uint64_t)((smem_addr & 0x3FFFF) >> 4) | ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
}
// D fp32, A and B e2m1 (K-major), scales ue8m0; M = rows, N = T; scale ids are added per MMA
__host__ __device__ __forceinline__ uint32_t instr_desc(int rows, int T) {
    return (1u << 7) | (1u << 10) | ((uint32_t)(T >> 3) << 17) | (1u << 23) | ((uint32_t)(rows >> 7) << 27);
}
__device__ __forceinline__ uint32_t scale_ids(int id) { return ((uint32_t)id << 4) | ((uint32_t)id << 29); }

__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void scales_to_tmem(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(src), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void store_y(void* y, int y_bf16, size_t at, float v) {
    if (y_bf16) reinterpret_cast<bf16*>(y)[at] = __float2bfloat16_rn(v);
    else reinterpret_cast<float*>(y)[at] = v;
}

// ---------------------------------------------------------------------------------------------------------------------
// The weight stream: up to 128 token rows per tile, one output tile per CTA, or per cluster whose CTAs share its k-blocks.
//   warp 0 / lane 0  producer: codes by TMA, scale tiles by bulk copies, into a ring of stages
//   warp 1 / lane 0  scales to tensor memory (two buffers), four MMAs per stage
//   warps 0..3       epilogue
// Two CTAs fit on an SM, so the set-up and the epilogue of one overlap the stream of the other.  With a cluster the partial
// tiles meet in distributed shared memory: every CTA sums its share of the token rows over the cluster in rank order
// (deterministic, no workspace, no tickets: nothing that two launches could share).
// ---------------------------------------------------------------------------------------------------------------------
struct StreamControl {
    uint64_t full[8], empty[8], acc_ready;
    uint32_t tmem_slot;
    int abort_flag, issued, consumed;
};
// Tensor memory is taken with an instruction that waits until enough columns are free.  A CTA of a cluster that waited there for
// a CTA of another cluster, which waits for its own cluster, could wait for good.  So shared memory is asked for in
// proportion (57 KB of an SM's 228 KB, 1 KB of it reserved per CTA, for every 128 of its 512 columns): the CTAs
// that fit on an SM by their shared memory also fit by their columns, and nobody ever waits.
__host__ __device__ __forceinline__ uint32_t stream_columns(int T) { return T <= 64 ? 128 : 256; }
__host__ __device__ __forceinline__ int stream_min_smem(int T) { return (T <= 64 ? 56 : 113) * 1024; }
constexpr int STREAM_MAX_SMEM = 113 * 1024;      // two CTAs per SM

static __global__ void __launch_bounds__(THREADS)
stream_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const GemmParams p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    StreamControl& ctl = *(StreamControl*)(ring + p.control_at);
    uint64_t *full = ctl.full, *empty = ctl.empty, &acc_ready = ctl.acc_ready;
    uint32_t& tmem_slot = ctl.tmem_slot;
    volatile int &abort_flag = ctl.abort_flag, &issued = ctl.issued, &consumed = ctl.consumed;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = p.stages, T = p.T, sbytes = stage_bytes(T, p.x_tiles);
    const int split = p.splits > 1 ? (int)cluster_rank() : 0;
    const int tile = blockIdx.x / (unsigned)p.splits;
    const int m0 = (tile % p.m_tiles) * T, n_tile = tile / p.m_tiles;
    const int kb0 = (int)((long long)p.kb_total * split / p.splits), kb1 = (int)((long long)p.kb_total * (split + 1) / p.splits);
    constexpr uint32_t D_COL = 64;                                  // columns 0..47: two scale buffers of up to 24
    const uint32_t tmem_cols = stream_columns(T);

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        mbar_init(&acc_ready, 1);
        abort_flag = 0;
        issued = 0;
        consumed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_w) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_x) : "memory");
    }
    if (warp == 0) {
        tmem_alloc(&tmem_slot, tmem_cols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    pdl_launch();

    if (warp == 0 && lane == 0) {
        pdl_wait();
        const int x_group = m0 / ROWS, x_groups = (p.M + ROWS - 1) / ROWS;
        for (int kb = kb0; kb < kb1; ++kb) {
            const int i = kb - kb0, s = i % S;
            if (i >= S && !mbar_wait(&empty[s], ((i / S) - 1) & 1, &abort_flag)) {
                abort_flag = 1;
                break;
            }
            if (abort_flag) break;
            uint8_t* w = ring + (size_t)s * sbytes;
            uint8_t* x = w + ROWS * KBYTES;
            uint8_t* sf = x + T * KBYTES;
            const uint32_t sf_bytes = (uint32_t)min(2, p.quads - 2 * kb) * SF_TILE;
            const int xt = min(p.x_tiles, x_groups - x_group);
            mbar_expect_tx(&full[s], (uint32_t)(ROWS + T) * KBYTES + (1 + xt) * sf_bytes);
            tma_load_2d(w, &map_w, kb * KBYTES, n_tile * ROWS, &full[s]);
            tma_load_2d(x, &map_x, kb * KBYTES, m0, &full[s]);
            bulk_load(sf, p.w_scales + ((size_t)n_tile * p.quads + 2 * kb) * SF_TILE, sf_bytes, &full[s]);
            for (int a = 0; a < xt; ++a)
                bulk_load(sf + (1 + a) * 2 * SF_TILE, p.x_scales + ((size_t)(x_group + a) * p.quads + 2 * kb) * SF_TILE, sf_bytes,
                          &full[s]);
            issued = i + 1;
        }
    } else if (warp == 1 && lane == 0) {
        const uint32_t idesc = instr_desc(ROWS, T);
        const int sf_cols = 8 + 8 * p.x_tiles;                      // per buffer: weights 2 x 4, tokens 2 x x_tiles x 4
        const uint32_t x_col = (uint32_t)(m0 % ROWS) / 32;
        for (int kb = kb0; kb < kb1; ++kb) {
            const int i = kb - kb0, s = i % S;
            if (!mbar_wait(&full[s], (i / S) & 1, &abort_flag)) {
                abort_flag = 1;
                break;
            }
            tc_fence_after();
            const uint32_t w_addr = smem_u32(ring + (size_t)s * sbytes), x_addr = w_addr + ROWS * KBYTES, sf_addr = x_addr + T * KBYTES;
            const uint32_t sfw = tmem + (i & 1) * sf_cols, sfx = sfw + 8;
            const int steps = min(KBLOCK / MMA_K, (p.K - kb * KBLOCK + MMA_K - 1) / MMA_K), quads = (steps + 1) / 2;
            for (int g = 0; g < quads; ++g) {
                scales_to_tmem(sfw + g * 4, desc_scales(sf_addr + g * SF_TILE));
                for (int a = 0; a < p.x_tiles; ++a)
                    scales_to_tmem(sfx + (g * p.x_tiles + a) * 4, desc_scales(sf_addr + ((1 + a) * 2 + g) * SF_TILE));
            }
            const uint64_t wd = desc_sw128(w_addr), xd = desc_sw128(x_addr);
            for (int k = 0; k < steps; ++k)                         // 64 elements are 32 bytes: +2 in the descriptors' address fields
                mma_mxf4(tmem + D_COL, wd + 2 * k, xd + 2 * k, idesc | scale_ids((k & 1) * 2), sfw + (k >> 1) * 4,
                         sfx + (k >> 1) * 4 * p.x_tiles + x_col, (i > 0 || k > 0) ? 1u : 0u);
            umma_commit(&empty[s]);
            consumed = i + 1;
        }
        umma_commit(&acc_ready);
    }
    __syncwarp();
    if (!mbar_wait(&acc_ready, 0)) abort_flag = 1;
    tc_fence_after();
    __syncthreads();
    const bool aborted = abort_flag != 0;
    if (aborted && threadIdx.x == 0) {
        atomicExch(p.status, 1);
        for (int i = consumed; i < issued; ++i) mbar_wait(&full[i % S], (i / S) & 1);      // copies in flight land first
    }
    const float nan = __int_as_float(0x7fffffff);
    const uint32_t taddr = tmem + D_COL + ((uint32_t)(warp * 32) << 16);
    const int n_local = warp * 32 + lane, n = n_tile * ROWS + n_local, rows = min(T, p.M - m0);
    if (p.splits == 1) {
        for (int c = 0; c < rows; c += 16) {
            float v[16];
            tmem_ld16(taddr + c, v);
            if (n < p.N) {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (c + j < rows) store_y(p.y, p.y_bf16, (size_t)(m0 + c + j) * p.ldy + n, aborted ? nan : p.scale * v[j]);
            }
        }
    } else {
        float* part = reinterpret_cast<float*>(ring);               // [T][128]; the ring is idle
        __syncthreads();                                            // ... once thread 0 has seen the last copies land
        for (int c = 0; c < rows; c += 16) {
            float v[16];
            tmem_ld16(taddr + c, v);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c + j < rows) part[(c + j) * ROWS + n_local] = aborted ? nan : v[j];
        }
        cluster_arrive();
        cluster_wait();
        const uint32_t mine = smem_u32(part) + 4 * n_local;
        for (int t = split; t < rows; t += p.splits) {
            float sum = 0.f;
            for (int q = 0; q < p.splits; ++q) {
                float v;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_map(mine + t * ROWS * 4, q)) : "memory");
                sum += v;
            }
            if (n < p.N) store_y(p.y, p.y_bf16, (size_t)(m0 + t) * p.ldy + n, p.scale * sum);
        }
        cluster_arrive();                                           // nobody leaves while others read its partial tile
        cluster_wait();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, tmem_cols);
}

}  // namespace mx
}  // namespace s2d2
