// Attention of new rows over a paged cache: parameters, and one row by a warp.
#pragma once
#include <algorithm>

#include "paged.cuh"

namespace s2d2 {
namespace patt {

struct Params {
    paged::Batch b;
    paged::Cache c;
    const bf16* q;
    bf16* out;
    float* lse;                      // may be null
    long long q_ld, out_ld;
    const unsigned long long* row_mask;
    int mask_block, heads, kv_heads, group, head_dim;
    float scale_log2;                // scale / ln 2: exponentials are powers of two
};

__device__ __forceinline__ float exp2_fast(float x) {      // relative error 2^-22; below 2^-126 zero
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float dot8(uint4 a, uint4 b, float s) {
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), s);
        s = fmaf(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), s);
    }
    return s;
}

// Maximum (times scale_log2), sum and weighted values of one (row, head) over the keys [k0, k1), by a warp: a lane takes a key's
// score, then every lane takes the elements lane, lane + 32, .. of the values.  Keys that are not seen are not read; a value that
// is seen counts even if its probability is zero: NaN and infinities are not lost.  `progress` (shared memory) goes up by one per 32 keys.
struct RowSum {
    float m, l, o[4];
};
__device__ __forceinline__ RowSum row_sum(const Params& p, int seq, int kv, int kvh, const bf16* q, const paged::View& view, int k0, int k1,
                                          int* progress) {
    const int lane = threadIdx.x & 31;
    RowSum a;
    a.m = -INFINITY;
    a.l = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) a.o[i] = 0.f;
    const long long head = (long long)kvh * p.c.head_stride;
    for (int j0 = k0; j0 < k1; j0 += 32) {
        if (lane == 0) atomicAdd(progress, 1);
        const int j = j0 + lane;
        const bool seen = j < min(k1, kv) && view.sees(j);
        long long at = -1;
        float s = -INFINITY;
        if (seen) {
            const int page = paged::page_of(p.b, seq, j);
            if (page >= 0) {
                at = page * p.c.page_stride + head + (j & p.c.page_mask) * p.c.token_stride;
                s = 0.f;
                for (int e = 0; e < p.head_dim; e += 8)
                    s = dot8(*reinterpret_cast<const uint4*>(q + e), *reinterpret_cast<const uint4*>(p.c.k + at + e), s);
                s *= p.scale_log2;
            } else {
                s = __int_as_float(0x7fffffff);
            }
        }
        const float m = fmaxf(a.m, warp_max(s));         // passes NaN over
        const float ref = m == -INFINITY ? 0.f : m;
        const float shrink = exp2_fast(a.m - ref), e = exp2_fast(s - ref);      // (infinity - infinity: NaN, as it should be)
        a.l = a.l * shrink + warp_sum(e);
        a.m = m;
#pragma unroll
        for (int i = 0; i < 4; ++i) a.o[i] *= shrink;
        // four keys' values on their way together (with eight, 164 registers leave the join's blocks no room beside the tiles); for a key that is not seen (weight 0) or has no page (weight NaN) those of one that is there
        const unsigned there = __ballot_sync(0xffffffffu, at >= 0);
        if (!there) continue;
        const long long other = __shfl_sync(0xffffffffu, at, __ffs(there) - 1);
#pragma unroll 1
        for (int t0 = 0; t0 < 32; t0 += 4) {
            float x[4][4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const long long from = __shfl_sync(0xffffffffu, at, t0 + t);
                const bf16* v = p.c.v + (from < 0 ? other : from);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float y = to_f32(v[min(lane + 32 * i, p.head_dim - 1)]);
                    x[t][i] = from < 0 ? 0.f : y;
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const float w = __shfl_sync(0xffffffffu, e, t0 + t);
#pragma unroll
                for (int i = 0; i < 4; ++i) a.o[i] = fmaf(w, x[t][i], a.o[i]);
            }
        }
    }
    if (a.l == 0.f) {                                    // scores of -inf only
#pragma unroll
        for (int i = 0; i < 4; ++i) a.o[i] = 0.f;
    }
    return a;
}

}  // namespace patt
}  // namespace s2d2
