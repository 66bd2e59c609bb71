// Tensor-core products of MXFP4 operands (sm_100a, tcgen05 kind::mxf4).
//
//   Y[m, n] = scale * sum_k X[m, k] W[n, k],   X and W in blocks of 32 elements with one power-of-two scale each
//
// The tensor core multiplies e2m1 codes, applies both scales and sums in fp32, so nothing is widened on the way: a
// weight costs 17/32 byte of HBM instead of 2.
//
// One k-block of a stage is 256 elements = 128 bytes of codes per row (one 128-byte swizzle row, four MMAs of 64) and
// 8 scales per row = two 512-byte scale tiles.  Scales go from shared memory to tensor memory by tcgen05.cp (32 lanes x 16
// bytes, repeated for the four lane quarters): column c + r / 32 of lane r % 32 then holds the four scales of row r of that
// tile, and an MMA of 64 elements takes the lower or the upper two of them (scale id 0 or 2).  A tile of B that starts in
// the middle of a scale tile reads its scales from column 2 on.  The column must be even (an odd one is a misaligned address),
// so tiles start at multiples of 64 rows.
#pragma once
#include "ops_host.h"
#include "tc_ptx.cuh"

namespace s2d2 {
namespace mx {

using namespace tc;

constexpr int ROWS = 128;            // A rows of a CTA's tile (MMA M)
constexpr int KBLOCK = 256;          // elements of a stage's k-block
constexpr int KBYTES = KBLOCK / 2;
constexpr int MMA_K = 64;
constexpr int SF_TILE = 512;         // bytes of one scale tile: 128 rows x 4 blocks
constexpr int THREADS = 352;         // warps: codes, MMA, eight of the epilogue, scales
constexpr int MAX_STAGES = 12;
constexpr int CUT = 64;              // B rows of a load of a tile that is cut short

// D = A B^T; which matrix is A and which is B depends on the operator (see product_kernel).
struct Params {
    int a_rows, b_rows, K;           // rows of the two matrices, elements along k
    int T;                           // B rows of a tile (multiple of 16 CG; of 64 if there are several tiles)
    int a_box;                       // A rows that a CTA loads per tile: 128, or fewer (a multiple of 8) where A has fewer
    int sf_tiles;                    // scale tiles that the B rows of a tile touch (1 or 2)
    int stages;
    int n_acc;                       // accumulator buffers (2: the epilogue of a tile overlaps the next tile's MMAs)
    int kb_total;                    // k-blocks
    int quads;                       // scale tiles along k
    int splits;                      // CTAs of a cluster that share a tile's k-blocks (1 with CTA pairs)
    int a_tiles, b_tiles;
    uint32_t tmem_cols;
    int control_at;                  // byte offset of Control behind the ring
    float scale;
    int* timeouts;
    uint32_t wait_limit;             // polls of a barrier before a wait is given up
    int withhold;                    // test tap: the codes are not loaded, so that nothing ever completes a stage
    // product
    void* y;                         // [b_rows, a_rows], rows ldy elements apart
    long long ldy;
    int y_bf16;
    // scores
    const int* tokens;
    float4* parts;                   // [a_tile][range][column half][A rows of a tile]: reference, sum, moment (in units of log 2), the token's logit or 0
    int ranges;                      // ranges of B per A tile, in units of `unit` rows
    int unit;
};

struct Control {
    uint64_t full[MAX_STAGES], empty[MAX_STAGES], acc_full[2], acc_empty[2];
    uint32_t tmem_slot;
    int abort_flag;
};

// Bytes of a CTA's stage: its A rows, its share of the B rows, scales of both.
__host__ __device__ __forceinline__ int stage_bytes(int cg, int a_box, int T, int sf_tiles) {
    return a_box * KBYTES + T / cg * KBYTES + (1 + sf_tiles) * 2 * SF_TILE;
}
// An MMA reads 128 rows of A.  Where fewer are loaded, the others are whatever follows in the ring (any bits are e2m1 codes); they
// end up in lanes that nobody reads.  Behind the last stage as many bytes are kept free.
__host__ __device__ __forceinline__ int ring_bytes(int cg, int stages, int a_box, int T, int sf_tiles) {
    return stages * stage_bytes(cg, a_box, T, sf_tiles) + (ROWS - a_box) * KBYTES;
}
__host__ __device__ __forceinline__ int scale_columns(int sf_tiles) { return 8 + 8 * sf_tiles; }      // of one of two buffers
// Accumulators are read 32 columns at a time.
__host__ __device__ __forceinline__ int acc_columns(int T) { return (T + 31) / 32 * 32; }
__host__ __device__ __forceinline__ int used_columns(int T, int sf_tiles, int n_acc) { return 2 * scale_columns(sf_tiles) + n_acc * acc_columns(T); }
// Tensor memory is taken with an instruction that waits until enough columns are free.  A CTA of a cluster that waited there for
// a CTA of another cluster, which waits for its own cluster, could wait for good.  So shared memory is asked for in
// proportion (57 KB of an SM's 228 KB, 1 KB of it reserved per CTA, for every 128 of its 512 columns; with all columns so much
// that no other CTA of these kernels fits): CTAs that fit on an SM by their shared memory also fit by their columns, and
// nobody ever waits.
__host__ __device__ __forceinline__ int min_smem(uint32_t cols) { return cols <= 64 ? 28 * 1024 : cols <= 128 ? 56 * 1024 : cols <= 256 ? 113 * 1024 : 200 * 1024; }

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

// The instructions come in a form for one CTA and one for a pair of CTAs (an even and an odd one of a cluster) that share
// an MMA of 256 rows: each holds 128 rows of A, half of the rows of B, all scales of B, and 128 lanes of the accumulator.
template <int CG>
__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         uint32_t accumulate) {
    if (CG == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
            : "memory");
}
template <int CG>
__device__ __forceinline__ void scales_to_tmem(uint32_t taddr, uint64_t desc) {
    if (CG == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// Arrives on the barrier (of both CTAs of a pair) when the MMAs issued so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint64_t* bar) {
    if (CG == 1) umma_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                         smem_u32(bar)),
                     "h"((uint16_t)3)
                     : "memory");
}
template <int CG>
__device__ __forceinline__ void alloc(uint32_t* slot, uint32_t cols) {
    if (CG == 1) {
        tmem_alloc(slot, cols);
        tmem_relinquish();
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int CG>
__device__ __forceinline__ void dealloc(uint32_t addr, uint32_t cols) {
    if (CG == 1) tmem_dealloc(addr, cols);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
// TMA tile load into this CTA that reports to a barrier of this CTA, or (pair) of the pair's first CTA
template <int CG>
__device__ __forceinline__ void load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
                dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
                dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
}
// 32 columns of this warp's 32 lanes; several loads may be in flight before load_wait()
__device__ __forceinline__ void tmem_ld32_issue(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// Release at CTA scope: what it orders are the reads of tensor memory in front of the fence.  At cluster scope it would wait for all
// stores of the warp (the output of the tile before), too.
__device__ __forceinline__ void arrive_remote(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void set_remote(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void store_y(void* y, int y_bf16, size_t at, float v) {
    if (y_bf16) reinterpret_cast<bf16*>(y)[at] = __float2bfloat16_rn(v);
    else reinterpret_cast<float*>(y)[at] = v;
}
// A thread's column of the accumulator: `cols` elements, one in each row of y from `y` on.
template <typename T, int NQ>
__device__ __forceinline__ void store_columns(T* y, long long ldy, const uint32_t (&v)[NQ][32], int cols, float scale) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        if (q * 32 + 32 <= cols) {
#pragma unroll
            for (int j = 0; j < 32; ++j, y += ldy) *y = from_f32<T>(scale * __uint_as_float(v[q][j]));
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j, y += ldy)
                if (q * 32 + j < cols) *y = from_f32<T>(scale * __uint_as_float(v[q][j]));
        }
    }
}
__device__ __forceinline__ float exp2_fast(float x) {      // relative error 2^-22; below 2^-126 zero
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

constexpr float LOG2E = 1.4426950408889634f;
constexpr float NEAR = 1048576.f;      // logits of up to this magnitude take the short form of fold()

// Sum of e^(x - m) and moment sum of u 2^u, u = (x - m) / log 2, over a token's logits; each with what its additions rounded off, since
// one thread may add up millions of terms. m is the largest logit or up to 1 less: it rises in steps of more than 1, so
// that the errors of the factors of its rises do not add up (each is weighted by the e^-1 of those behind it).
struct Sums {
    float m, s, s_low, mo, mo_low;
};
// a + low += b, low taking the rounding error of the addition exactly
__device__ __forceinline__ void add_exact(float& a, float& low, float b) {
    const float t = a + b, c = t - a;
    low += (a - (t - c)) + (b - c);
    a = t;
}
__device__ __forceinline__ void raise(Sums& a, float top) {
    if (top > a.m + 1.f) {
        const float d = fmaxf((a.m - top) * LOG2E, -300.f), f = exp2_fast(d);
        a.mo = f * fmaf(d, a.s, a.mo);
        a.mo_low = f * fmaf(d, a.s_low, a.mo_low);
        a.s *= f;
        a.s_low *= f;
        a.m = top;
    }
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {      // two operations in one instruction
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
// The largest and the smallest of the first n of 32 accumulators (NaN is passed over).
__device__ __forceinline__ void extremes(const uint32_t (&v)[32], int n, float& high, float& low) {
    high = low = __uint_as_float(v[0]);
    if (n >= 32) {
#pragma unroll
        for (int j = 1; j < 31; j += 2) {
            asm("max.f32 %0, %0, %1, %2;" : "+f"(high) : "f"(__uint_as_float(v[j])), "f"(__uint_as_float(v[j + 1])));
            asm("min.f32 %0, %0, %1, %2;" : "+f"(low) : "f"(__uint_as_float(v[j])), "f"(__uint_as_float(v[j + 1])));
        }
        high = fmaxf(high, __uint_as_float(v[31]));
        low = fminf(low, __uint_as_float(v[31]));
    } else {
#pragma unroll
        for (int j = 1; j < 32; ++j)
            if (j < n) high = fmaxf(high, __uint_as_float(v[j])), low = fminf(low, __uint_as_float(v[j]));
    }
}
// Adds n logits (accumulators times scale) to the sums: at most 16 terms one after the other, even and odd columns apart, then exactly.
// NEAR_ALL: 32 logits, all of at most NEAR in magnitude, as is the reference. x - m is one operation then: against a reference that is
// rounded the unrounded logit is up to 2^-24 NEAR larger, which is nothing. Otherwise the logit is rounded first and differences are cut off
// where their exponential is zero: that of -3e38 and 3e38 is infinite.
template <bool NEAR_ALL>
__device__ __forceinline__ void fold(const uint32_t (&v)[32], int n, float scale, Sums& a) {
    float2 s = make_float2(0.f, 0.f), mo = s;
    const float m = a.m;
    const float2 cc = make_float2(scale, scale), minus_m = make_float2(-m, -m), log2e = make_float2(LOG2E, LOG2E);
    if (NEAR_ALL) {
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            const float2 u = mul2(fma2(make_float2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), cc, minus_m), log2e);
            const float2 e = make_float2(exp2_fast(u.x), exp2_fast(u.y));
            s = add2(s, e);
            mo = fma2(u, e, mo);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < n) {
                // NaN for a NaN, and for infinity (m is infinite then): such a row is undefined
                const float u = (__fmul_rn(__uint_as_float(v[j]), scale) - m) * LOG2E, e = exp2_fast(u);
                if (j & 1) s.y += e, mo.y = fmaf(fmaxf(u, -300.f), e, mo.y);
                else s.x += e, mo.x = fmaf(fmaxf(u, -300.f), e, mo.x);
            }
    }
    add_exact(a.s, a.s_low, s.x + s.y);
    add_exact(a.mo, a.mo_low, mo.x + mo.y);
}

// Rows split, split + S, ... of a tile's sum over the S CTAs of a cluster, each with a partial tile [T][128] at `part`.  A warp takes
// a row at a time, a lane four of its elements, and has eight loads in flight: distant shared memory answers late.
template <int S>
__device__ __forceinline__ void sum_parts(const Params& p, uint32_t part, int split, int rows, int b0, int a) {
    constexpr int AT_ONCE = 8 / S, WARPS = THREADS / 32;
    const int warp = threadIdx.x >> 5;
    for (int j0 = warp * AT_ONCE; j0 * S + split < rows; j0 += WARPS * AT_ONCE) {
        float4 v[AT_ONCE][S];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
            for (int q = 0; q < S; ++q) {
                const int b = (j0 + j) * S + split;
                v[j][q] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (b < rows)
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                 : "=f"(v[j][q].x), "=f"(v[j][q].y), "=f"(v[j][q].z), "=f"(v[j][q].w)
                                 : "r"(cluster_map(part + b * ROWS * 4 + 16 * (threadIdx.x & 31), q))
                                 : "memory");
            }
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int b = (j0 + j) * S + split;
            if (b >= rows) break;
            float4 sum = v[j][0];
#pragma unroll
            for (int q = 1; q < S; ++q) {
                sum.x += v[j][q].x;
                sum.y += v[j][q].y;
                sum.z += v[j][q].z;
                sum.w += v[j][q].w;
            }
            const float x[4] = {sum.x, sum.y, sum.z, sum.w};
            const size_t at = (size_t)(b0 + b) * p.ldy + a;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (a + e < p.a_rows) store_y(p.y, p.y_bf16, at + e, p.scale * x[e]);
        }
    }
}

// One lane of a converged warp.  The warps that feed the tensor core and the copy engine run their loops with all lanes, so
// that addresses and descriptors stay in uniform registers; only the instruction itself is left to one lane.
__device__ __forceinline__ bool elect() {
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e != 0;
}
// After a time-out: copies in flight land before anything else uses their shared memory.
__device__ __forceinline__ void settle() {
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
}
__device__ __forceinline__ bool poll(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done;
}
// Bounded wait for the phase with the given parity; false when it has run out or another role of the CTA has given up. The limit is
// looked at every 32 polls of about 4 us, beside a constant bound: as the loop's own bound it made every stage 4 % longer.
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, uint32_t limit, volatile int* abort_flag) {
    const uint32_t addr = smem_u32(bar);
    for (uint32_t it = 0; it < WAIT_LIMIT; ++it) {
        if ((it & 31u) == 31u && (it >= limit || *abort_flag)) return false;
        if (poll(addr, parity)) return true;
    }
    return false;
}
// Position in the ring: stage and the parity of its current use.
struct Ring {
    int s = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next(int stages) {
        if (++s == stages) s = 0, parity ^= 1;
    }
};

// The tiles that a cluster works on, in order.
//   product: tile number = cluster + i * clusters; B tiles vary fastest, so that the clusters at work share the A tiles
//   scores:  a cluster takes (A tile, range) items; inside an item the B tiles of its range
struct Tiles {
    int item, b, b_end;              // scores: first B row of the next tile, end of the range
    int a0, b0, rows;                // current tile: A tile number, first B row, B rows
    int first, last;                 // scores: first / last tile of an item
};
template <bool SCORE>
__device__ __forceinline__ Tiles first_tile(int cluster) {
    Tiles t;
    t.item = cluster;
    t.b = t.b_end = 0;
    t.last = 1;
    return t;
}
template <bool SCORE>
__device__ __forceinline__ bool next_tile(const Params& p, Tiles& t, int clusters) {
    if (!SCORE) {
        if (t.item >= p.a_tiles * p.b_tiles) return false;
        t.a0 = t.item / p.b_tiles;
        t.b0 = (t.item % p.b_tiles) * p.T;
        t.rows = p.T;
        t.item += clusters;
        return true;
    }
    t.first = t.last;
    if (t.first) {
        if (t.item >= p.a_tiles * p.ranges) return false;
        t.a0 = t.item % p.a_tiles;                 // clusters next to each other read the same range of B
        const int range = t.item / p.a_tiles;
        const long long units = (p.b_rows + p.unit - 1) / p.unit;
        t.b = (int)(units * range / p.ranges) * p.unit;
        t.b_end = (int)(units * (range + 1) / p.ranges) * p.unit;
        t.item += clusters;
    }
    t.b0 = t.b;
    t.rows = min(p.T, t.b_end - t.b);
    t.b += t.rows;
    t.last = t.b >= t.b_end;
    return true;
}

// After a time-out: NaN in all outputs of the cluster's tiles, those that were finished included.
template <int CG, bool SCORE>
__device__ __forceinline__ void all_nan(const Params& p, int cluster, int clusters, int pair_rank) {
    const float nan = __int_as_float(0x7fffffff);
    Tiles t = first_tile<SCORE>(cluster);
    while (next_tile<SCORE>(p, t, clusters)) {
        const int row0 = pair_rank * ROWS, a0 = t.a0 * CG * ROWS + row0;
        if (SCORE) {
            const int range = (t.item - clusters) / p.a_tiles;
            for (int i = threadIdx.x; t.last && i < 2 * ROWS; i += THREADS)
                if (a0 + i % ROWS < p.a_rows)
                    p.parts[(((size_t)t.a0 * p.ranges + range) * 2 + i / ROWS) * (ROWS * CG) + row0 + i % ROWS] = make_float4(0.f, nan, nan, nan);
        } else {
            const int rows = min(t.rows, p.b_rows - t.b0);
            for (int i = threadIdx.x; i < rows * ROWS; i += THREADS)
                if (a0 + i % ROWS < p.a_rows) store_y(p.y, p.y_bf16, (size_t)(t.b0 + i / ROWS) * p.ldy + a0 + i % ROWS, nan);
        }
    }
}

// One kernel for both operators and for one CTA or a pair of CTAs per tile.
//   product (SCORE = false): A = weights, B = tokens.  The accumulator's lanes are output features, so an epilogue warp stores 32
//     consecutive elements of an output row, whatever that row's alignment.
//   scores (SCORE = true): A = tokens, B = head.  A lane is one token's row of logits: each thread folds the logits of
//     its token into a running reference, sum and moment; nothing is exchanged between threads and no logit leaves the SM.
//   warp 0     producer of the codes: TMA into a ring of stages that runs on from tile to tile
//   warp 10    producer of the scale tiles of the same stages
//   warp 1     scales to tensor memory (two buffers), four MMAs of 64 elements per stage; tensor memory
//   warps 2-9  epilogue: four lane quarters, two warps for the halves of the columns.  A warp takes its part of the
//              accumulator (up to 128 columns) into registers at once and gives tensor memory back before it computes
//              and stores, so the next tile's MMAs wait for a short read only, even with one accumulator.
// With few tiles the CTAs of a cluster (p.splits) share the k-blocks of one tile; the partial tiles meet in distributed
// shared memory, where every CTA sums its share of the rows over the cluster in rank order: deterministic, no
// workspace, no tickets, nothing that two launches could share.
// Measured (B200): a head of 151936 x 4096 against 8 rows 57 us (330 MB at 5.8 TB/s); 1024 x 24576 x 4096, with the quantisation of the
// rows, 46 us (52 with T = 192, 65 with T = 128; 55 in a long loop); scores of 1024 rows against the head 225 us (5.7 PFLOP/s; 4.8 in
// a long loop, at the power limit; its MMAs alone 194 us).
// Every wait on a barrier is bounded; after a time-out all outputs of the cluster are NaN and it is counted.
// NQ: groups of 32 columns that an epilogue warp holds; with one (T <= 64) two CTAs fit on an SM by their registers.
template <int CG, bool SCORE, int NQ>
__global__ void __launch_bounds__(THREADS, NQ == 1 ? 2 : 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ CUtensorMap map_cut, const __grid_constant__ CUtensorMap map_sfa,
               const __grid_constant__ CUtensorMap map_sfb, const Params p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* ring = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Control& ctl = *(Control*)(ring + p.control_at);
    volatile int* abort_flag = &ctl.abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = p.stages, sbytes = stage_bytes(CG, p.a_box, p.T, p.sf_tiles);
    const int cluster_size = CG * p.splits;
    const uint32_t rank = cluster_size > 1 ? cluster_rank() : 0;
    const int cluster = blockIdx.x / (unsigned)cluster_size, clusters = gridDim.x / (unsigned)cluster_size;
    const int split = CG == 1 ? (int)rank : 0;
    const int kb0 = (int)((long long)p.kb_total * split / p.splits), kb1 = (int)((long long)p.kb_total * (split + 1) / p.splits);
    const uint32_t d_col = 2 * scale_columns(p.sf_tiles);

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(&ctl.full[s], 1);
            mbar_init(&ctl.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&ctl.acc_full[b], 1);
            mbar_init(&ctl.acc_empty[b], 8 * CG);
        }
        ctl.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_sfa) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_sfb) : "memory");
    }
    if (warp == 1) alloc<CG>(&ctl.tmem_slot, p.tmem_cols);
    tc_fence_before();
    if (cluster_size > 1) {
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
    tc_fence_after();
    const uint32_t tmem = ctl.tmem_slot;
    pdl_launch();
    // All warps: none reads or writes memory that the kernels in front still use, and the bounded waits begin behind them.
    pdl_wait();

    Tiles t = first_tile<SCORE>(cluster);
    const int b_half = p.T / CG, a_bytes = p.a_box * KBYTES, b_bytes = b_half * KBYTES;
    if (warp == 0 || warp == 10) {
        // Producers: codes (warp 0) and scales (warp 10) of the same stage, reported to one barrier.
        const uint32_t fixed_bytes = (uint32_t)CG * (a_bytes + (1 + p.sf_tiles) * 2 * SF_TILE);
        Ring r;
        r.parity = 1;                                        // a fresh barrier passes a wait for the phase before its first
        bool ok = true;
        if (p.withhold && warp == 0) t.item = 0x7fffffff;
        while (ok && next_tile<SCORE>(p, t, clusters)) {
            const int a_row = (t.a0 * CG + (CG == 2 ? (int)rank : 0)) * ROWS;
            const int b_row = t.b0 + (CG == 2 ? (int)rank * b_half : 0);
            const int sfa_row = a_row / ROWS * p.quads, sfb_row = t.b0 / ROWS * p.quads;
            const bool cut = SCORE && CG == 1 && t.rows < p.T;          // a single CTA loads no more of it than the range holds
            const uint32_t bytes = fixed_bytes + (uint32_t)CG * (cut ? (t.rows + CUT - 1) / CUT * CUT : b_half) * KBYTES;
            for (int kb = kb0; kb < kb1; ++kb, r.next(S)) {
                ok = __all_sync(0xffffffffu, wait(&ctl.empty[r.s], r.parity, p.wait_limit, abort_flag));
                if (!ok) break;
                const uint32_t a = smem_u32(ring) + r.s * sbytes;
                uint32_t bar = smem_u32(&ctl.full[r.s]);
                if (CG == 2) bar = cluster_map(bar, 0);
                if (elect()) {
                    if (warp == 0) {
                        if (CG == 1 || rank == 0) mbar_expect_tx(&ctl.full[r.s], bytes);
                        load_2d<CG>(a, &map_a, kb * KBYTES, a_row, bar);
                        if (!cut) load_2d<CG>(a + a_bytes, &map_b, kb * KBYTES, b_row, bar);
                        else
                            for (int i = 0; i < t.rows; i += CUT) load_2d<CG>(a + a_bytes + i * KBYTES, &map_cut, kb * KBYTES, b_row + i, bar);
                    } else {
                        const uint32_t sf = a + a_bytes + b_bytes;
                        load_2d<CG>(sf, &map_sfa, 0, sfa_row + 2 * kb, bar);
                        load_2d<CG>(sf + 2 * SF_TILE, &map_sfb, 0, sfb_row + 2 * kb, bar);
                        if (p.sf_tiles > 1) load_2d<CG>(sf + 4 * SF_TILE, &map_sfb, 0, sfb_row + p.quads + 2 * kb, bar);
                    }
                }
                __syncwarp();
            }
        }
        if (!ok) *abort_flag = 1;
    } else if (warp == 1) {
        if (CG == 1 || rank == 0) {
            const uint32_t idesc = instr_desc(ROWS * CG, p.T);      // of a tile cut short at the end of a range, the last columns go unread
            const int sf_cols = scale_columns(p.sf_tiles), sfb_step = 4 * p.sf_tiles;
            Ring r;
            int acc = 0, odd = 0;
            uint32_t acc_parity = 1;
            bool ok = true;
            while (ok && next_tile<SCORE>(p, t, clusters)) {
                ok = __all_sync(0xffffffffu, wait(&ctl.acc_empty[acc], acc_parity, p.wait_limit, abort_flag));
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem + d_col + acc * acc_columns(p.T);
                const uint32_t b_col = (uint32_t)(t.b0 % ROWS) / 32;
                for (int kb = kb0; kb < kb1; ++kb, r.next(S), odd ^= 1) {
                    ok = __all_sync(0xffffffffu, wait(&ctl.full[r.s], r.parity, p.wait_limit, abort_flag));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t a_addr = smem_u32(ring) + r.s * sbytes, sf_addr = a_addr + a_bytes + b_bytes;
                    const uint32_t sfa = tmem + odd * sf_cols, sfb = sfa + 8;
                    const uint64_t ad = desc_sw128(a_addr), bd = desc_sw128(a_addr + a_bytes), sd = desc_scales(sf_addr);
                    const int left = p.K - kb * KBLOCK;
                    if (elect()) {
                        // a scale tile is 512 bytes: +32 in a descriptor's address field; 64 elements are 32 bytes: +2
                        auto scales = [&](int q) {
                            scales_to_tmem<CG>(sfa + q * 4, sd + q * 32);
                            scales_to_tmem<CG>(sfb + q * sfb_step, sd + 64 + q * 32);
                            if (p.sf_tiles > 1) scales_to_tmem<CG>(sfb + q * sfb_step + 4, sd + 128 + q * 32);
                        };
                        auto multiply = [&](int k) {
                            mma_mxf4<CG>(d, ad + 2 * k, bd + 2 * k, idesc | scale_ids((k & 1) * 2), sfa + (k >> 1) * 4,
                                         sfb + (k >> 1) * sfb_step + b_col, (kb > kb0 || k > 0) ? 1u : 0u);
                        };
                        scales(0);
                        if (left > KBLOCK / 2) scales(1);
                        if (left > KBLOCK - MMA_K) {
#pragma unroll
                            for (int k = 0; k < KBLOCK / MMA_K; ++k) multiply(k);
                        } else {
                            for (int k = 0; k * MMA_K < left; ++k) multiply(k);
                        }
                        commit<CG>(&ctl.empty[r.s]);
                        if (kb == kb1 - 1) commit<CG>(&ctl.acc_full[acc]);
                    }
                    __syncwarp();
                }
                if (++acc == p.n_acc) acc = 0, acc_parity ^= 1;
            }
            if (!ok) *abort_flag = 1;
        }
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;      // the lanes of tensor memory that this warp may read; its columns
        const int row = quarter * 32 + lane, row0 = (CG == 2 ? (int)rank * ROWS : 0) + row;
        const int half_cols = (p.T / 2 + 31) / 32 * 32;
        const int col0 = half * half_cols, col1 = half ? p.T : min(half_cols, p.T);
        const float nan = __int_as_float(0x7fffffff);
        int acc = 0;
        uint32_t parity = 0;
        // scores
        Sums sums = {};
        float x_t = 0.f;
        int token = -1;
        while (next_tile<SCORE>(p, t, clusters)) {
            if (!__all_sync(0xffffffffu, !*abort_flag && wait(&ctl.acc_full[acc], parity, p.wait_limit, abort_flag))) {
                *abort_flag = 1;
                break;
            }
            tc_fence_after();
            const uint32_t taddr = tmem + d_col + acc * acc_columns(p.T) + col0 + ((uint32_t)(quarter * 32) << 16);
            const int a = t.a0 * CG * ROWS + row0;
            // columns of the tile that are rows of B; lanes that are rows of A
            const int cols = min(col1, min(t.rows, p.b_rows - t.b0)) - col0;
            const bool any = a - lane < p.a_rows && cols > 0;
            uint32_t v[NQ][32];
            if (any) {
#pragma unroll
                for (int q = 0; q < NQ; ++q)
                    if (q * 32 < cols) tmem_ld32_issue(taddr + q * 32, v[q]);
                tmem_ld_wait();
            }
            // the accumulator may be overwritten (by the pair's first CTA, which issues the MMAs)
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG == 1) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(&ctl.acc_empty[acc])) : "memory");
                else arrive_remote(cluster_map(smem_u32(&ctl.acc_empty[acc]), 0));
            }
            if (++acc == p.n_acc) acc = 0, parity ^= 1;
            if (!SCORE) {
                if (!any) continue;
                const int b = t.b0 + col0;
                if (p.splits > 1) {
                    // the ring is idle: a cluster that shares a tile has no other, and all its loads have been multiplied
                    float* part = reinterpret_cast<float*>(ring) + (size_t)col0 * ROWS + row;
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (q * 32 + j < cols) part[(q * 32 + j) * ROWS] = __uint_as_float(v[q][j]);
                } else if (a < p.a_rows) {
                    if (p.y_bf16) store_columns(reinterpret_cast<bf16*>(p.y) + (size_t)b * p.ldy + a, p.ldy, v, cols, p.scale);
                    else store_columns(reinterpret_cast<float*>(p.y) + (size_t)b * p.ldy + a, p.ldy, v, cols, p.scale);
                }
            } else {
                if (t.first) {
                    sums = Sums{-3.402823466e38f, 0.f, 0.f, 0.f, 0.f};
                    x_t = 0.f;
                    token = p.tokens && a < p.a_rows ? p.tokens[a] : -1;
                }
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    if (!any || q * 32 >= cols) break;
                    const int n = cols - q * 32;
                    float high, low;
                    extremes(v[q], n, high, low);
                    // the largest product comes from the largest accumulator, or with a negative factor from the smallest
                    const float x0 = high * p.scale, x1 = low * p.scale, bottom = fminf(x0, x1);
                    raise(sums, fmaxf(x0, x1));
                    if (n >= 32 && fmaxf(fabsf(sums.m), -bottom) <= NEAR) fold<true>(v[q], 32, p.scale, sums);
                    else fold<false>(v[q], n, p.scale, sums);
                    if (bottom == -INFINITY) sums.s = nan;            // its exponential is zero: nothing else shows it
                    const int at = token - (t.b0 + col0 + q * 32);
                    if (at >= 0 && at < 32) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (j == at) x_t = __fmul_rn(__uint_as_float(v[q][j]), p.scale);
                    }
                }
                if (t.last && a < p.a_rows) {
                    const int range = (t.item - clusters) / p.a_tiles;
                    p.parts[(((size_t)t.a0 * p.ranges + range) * 2 + half) * (ROWS * CG) + row0] = make_float4(sums.m, sums.s + sums.s_low, sums.mo + sums.mo_low, x_t);
                }
            }
        }
    }
    __syncwarp();
    if (CG == 1 && p.splits > 1) {
        // sum of the partial tiles over the cluster
        cluster_arrive();
        cluster_wait();
        Tiles u = first_tile<SCORE>(cluster);
        next_tile<SCORE>(p, u, clusters);
        const int rows = min(u.rows, p.b_rows - u.b0), a = u.a0 * ROWS + 4 * lane;
        if (p.splits == 2) sum_parts<2>(p, smem_u32(ring), split, rows, u.b0, a);
        else if (p.splits == 4) sum_parts<4>(p, smem_u32(ring), split, rows, u.b0, a);
        else sum_parts<8>(p, smem_u32(ring), split, rows, u.b0, a);
    }
    __syncthreads();
    if (*abort_flag) {
        settle();
        // the CTAs of a cluster fail together: what one of them missed is in the others' outputs, too
        if (threadIdx.x < cluster_size) set_remote(cluster_size > 1 ? cluster_map(smem_u32(&ctl.abort_flag), threadIdx.x) : smem_u32(&ctl.abort_flag), 1);
    }
    tc_fence_before();
    if (cluster_size > 1) {
        // nobody leaves while others read its shared memory, signal its barriers or multiply into its tensor memory
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
    if (warp == 1) dealloc<CG>(tmem, p.tmem_cols);
    if (*abort_flag) {
        // behind the barrier, so that these are the last values of the cluster's outputs
        if (threadIdx.x == 0) atomicAdd(p.timeouts, 1);
        all_nan<CG, SCORE>(p, cluster, clusters, CG == 2 ? (int)rank : 0);
    }
}

// Scores from the partial results of a row: one block per row, a thread per part (or several), merged in a fixed order.
// Few registers and little shared memory: it waits on the SMs while the product still runs.
static __global__ void __launch_bounds__(128, 10)
score_parts_kernel(const Params p, int rows_per_tile, float* logprob, float* lse, float* entropy) {
    __shared__ float4 sh[4];
    pdl_wait();
    pdl_launch();
    const int r = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float4* parts = p.parts + (size_t)(r / rows_per_tile) * p.ranges * 2 * rows_per_tile + r % rows_per_tile;
    const int token = p.tokens ? p.tokens[r] : -1;
    const bool has_token = token >= 0 && token < p.b_rows;
    float4 a = make_float4(-3.402823466e38f, 0.f, 0.f, 0.f);      // reference, sum, moment; logit of the token (zero in all parts but one)
    auto add = [&](const float4 b) {
        const float M = fmaxf(a.x, b.x), d1 = fmaxf((a.x - M) * LOG2E, -300.f), d2 = fmaxf((b.x - M) * LOG2E, -300.f);
        const float f1 = exp2_fast(d1), f2 = exp2_fast(d2);
        a = make_float4(M, f1 * a.y + f2 * b.y, f1 * (a.z + d1 * a.y) + f2 * (b.z + d2 * b.y), a.w + b.w);
    };
#pragma unroll 4
    for (int i = threadIdx.x; i < 2 * p.ranges; i += 128) {
        add(parts[(size_t)i * rows_per_tile]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        add(make_float4(__shfl_xor_sync(0xffffffffu, a.x, o), __shfl_xor_sync(0xffffffffu, a.y, o), __shfl_xor_sync(0xffffffffu, a.z, o),
                        __shfl_xor_sync(0xffffffffu, a.w, o)));
    if (lane == 0) sh[warp] = a;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < 4; ++w) add(sh[w]);
    const float log_s = logf(a.y), nan = __int_as_float(0x7fffffff);
    const bool undefined = !(a.y > 0.f) || isinf(a.x);
    if (lse) lse[r] = undefined ? nan : a.x + log_s;
    // (of a certain token: a difference of equal numbers, rounded)
    if (entropy) entropy[r] = undefined ? nan : fmaxf(log_s - a.z * 0.6931471805599453f / a.y, 0.f);
    if (logprob) logprob[r] = undefined || !has_token ? nan : (a.w - a.x) - log_s;
}

}  // namespace mx
}  // namespace s2d2
