// Scores of caller-supplied logits: log probability and rank of a given token, log-sum-exp, entropy, top alternatives.
//
// With m = max_j x_j and s = sum_j e^(x_j - m) over one row of logits:
//   lse = m + log s        logprob = (x_t - m) - log s        entropy = log s - (1/s) sum_j (x_j - m) e^(x_j - m)
//   rank = #{j : x_j > x_t} + #{j < t : x_j = x_t}            top: value descending, lowest id first among equals
//
// One pass over the row with a running maximum (per thread, one rescale per 16 elements).  Maxima, sums and moments are fp32
// per thread over at most a few thousand terms and are merged in a fixed order.  The moment uses x - m instead of x:
// log s - t/s then adds two non-negative terms, where lse - sum x p subtracts numbers of the size of the logits.
//
// The top alternatives cost nothing per element: the loop keeps the maximum of every (thread, 16 elements) tile in shared memory.
// If every one of the eight warps has at least ceil(k / 8) threads whose maximum is t or more, t is a lower bound of the k-th
// largest element.  So only tiles whose maximum reaches the least of the warps' ceil(k / 8)-th largest thread maxima are read
// again (two to three tiles of 16 elements per alternative), and only elements that reach it are ordered.
//
// Bound by HBM for the sums (1024 x 157184 fp32: 100 us, 6.4 TB/s; 117 us with five alternatives and ranks); for 16-bit logits
// instructions weigh as much (256 x 151936: 20 us of which 12 are the bytes'). One row of 151936 takes 4 us, 9 with 20 alternatives.
//
// A row is shared by a cluster of 1, 2, 4 or 8 CTAs, so that a few rows fill the GPU; partial results meet in the shared memory
// of the cluster's first CTA.  Nothing is kept in global memory, no atomics on it, no workspace.
#include <float.h>
#include <math.h>


#include "common.cuh"
#include "ops_host.h"

namespace s2d2 {
namespace {

constexpr int NT = 256;            // threads
constexpr int NW = NT / 32;
constexpr int TILE = 16;           // elements of one thread between two rescales
constexpr int CAP = 1024;          // candidates held in shared memory
constexpr int MANY_EQUAL = 128;    // threads whose maximum equals the bound: more, and equal elements are taken in id order instead
constexpr int TILES = 768;         // tiles that may be read again
constexpr int MAX_CLUSTER = 8;
constexpr int MAX_TILES = 64;      // tiles of a CTA with alternatives: one bit each when they are marked
static_assert(S2D2_SCORE_MAX_VOCAB + 64 <= MAX_CLUSTER * MAX_TILES * NT * TILE, "a vocabulary fits a cluster's tiles");
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int MAX_SMEM = MAX_TILES * NT * 4;   // tile maxima

struct ScoreParams {
    const void* x;
    long long ld;
    int V;
    int cluster;
    int seg_vec;                   // 16-byte vectors of a row per CTA
    int n_tiles;                   // tiles per CTA
    const int* tokens;
    int top;
    float* logprob;
    int* rank;
    float* lse;
    float* entropy;
    int* top_ids;
    float* top_lp;
};

// Relative error 2^-22; 0 for -inf, NaN for NaN.  Results below 2^-126 become zero (they are next to sums of at least one), which
// saves the scaling of subnormal results: three instructions of about ten per element.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two fp32 operations per instruction, each rounded as the scalar one.
struct Pair {
    unsigned long long v;
};
__device__ __forceinline__ Pair pair(float a, float b) {
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p.v) : "f"(a), "f"(b));
    return p;
}
__device__ __forceinline__ float lo(Pair p) {
    return __uint_as_float((uint32_t)p.v);
}
__device__ __forceinline__ float hi(Pair p) {
    return __uint_as_float((uint32_t)(p.v >> 32));
}
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
    Pair p;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(p.v) : "l"(a.v), "l"(b.v));
    return p;
}
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
    Pair p;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(p.v) : "l"(a.v), "l"(b.v));
    return p;
}
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c) {
    Pair p;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(p.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return p;
}
// Larger key = earlier in the order (value descending, id ascending).  -0 counts as +0.
__device__ __forceinline__ unsigned long long order_key(float v, int id) {
    const uint32_t b = __float_as_uint(v + 0.f);
    const uint32_t o = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
    return ((unsigned long long)o << 32) | (uint32_t)~(uint32_t)id;
}
__device__ __forceinline__ float key_value(unsigned long long k) {
    const uint32_t o = (uint32_t)(k >> 32);
    return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ int key_id(unsigned long long k) { return (int)~(uint32_t)k; }

// The row as 16-byte vectors counted from the aligned address at or before its first element; `lead` elements in front
// of the row belong to vector 0.  Elements outside the row read as -inf and are not touched in memory.
template <typename T>
struct Row {
    static constexpr int E = 16 / (int)sizeof(T);
    const T* p;
    int lead, V;
    __device__ __forceinline__ Row(const T* row, int V) : p(row), V(V) {
        lead = (int)(((uintptr_t)row & 15) / sizeof(T));
    }
    __device__ __forceinline__ int first_id(int vec) const { return vec * E - lead; }
    static __device__ __forceinline__ void widen(const uint4 w, float* x) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
        if (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(u[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[2 * e] = __uint_as_float(u[e] << 16);
                x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
            }
        }
    }
    // a vector as it stands in memory; `inside`: all of it lies in the row. Not through the read-only path: the logits may be written
    // by the kernel in front after this one has begun.
    __device__ __forceinline__ uint4 raw(int vec, bool inside) const {
        const int i0 = first_id(vec);
        if (inside || (i0 >= 0 && i0 + E <= V)) return *reinterpret_cast<const uint4*>(p + i0);
        uint32_t u[4];
#pragma unroll
        for (int e = 0; e < E; e += 4 / (int)sizeof(T)) {
            uint32_t w = 0;
#pragma unroll
            for (int h = 0; h < 4 / (int)sizeof(T); ++h) {
                const float f = (i0 + e + h >= 0 && i0 + e + h < V) ? to_f32(p[i0 + e + h]) : -INFINITY;
                w |= sizeof(T) == 4 ? __float_as_uint(f) : (__float_as_uint(f) >> 16) << (16 * h);
            }
            u[e * (int)sizeof(T) / 4] = w;
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
    __device__ __forceinline__ void load(int vec, float* x) const { widen(raw(vec, false), x); }
};

struct alignas(16) Partial {       // one CTA's share of a row
    float m, s, t;
    int before;
};

struct Shared {
    unsigned long long cand[CAP + 8];
    unsigned long long top[MAX_CLUSTER][32];     // in the cluster's first CTA: every CTA's best, in order, 0 = none
    unsigned long long best[32];                 // this CTA's best, in order
    Partial part[MAX_CLUSTER * NW];              // in the cluster's first CTA: every warp's sums
    float bound[NW];
    int warp_count[NW];
    int tile[TILES];                             // tiles that are read again
    int n_cand, n_tile;
    float m, log_s;
};

// Position of `key` among the n keys of `list`, which is padded to a multiple of eight with zeros.
__device__ __forceinline__ int count_above(const unsigned long long* list, int n, unsigned long long key) {
    int pos = 0;
    for (int j = 0; j < n; j += 8) {
#pragma unroll
        for (int h = 0; h < 8; h += 2) {
            const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(list + j + h);
            pos += w.x > key;
            pos += w.y > key;
        }
    }
    return pos;
}

// Places for `n` entries of every lane behind *count, taken by the warp at once; the first of this lane's.  Converged warp.
__device__ __forceinline__ int warp_places(int n, int* count) {
    const int lane = threadIdx.x & 31;
    int end = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int w = __shfl_up_sync(0xffffffffu, end, o);
        if (lane >= o) end += w;
    }
    int base = 0;
    if (lane == 31) base = atomicAdd(count, end);
    return __shfl_sync(0xffffffffu, base, 31) + end - n;
}

// Appends, in id order, elements equal to `v` of the vectors [v0, v1) to best[n..], until `k` are there.  Whole CTA.
template <typename T>
__device__ int append_equal(const Row<T>& row, int v0, int v1, float v, unsigned long long* best, int n, int k, Shared& sh) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int b = v0; b < v1 && n < k; b += NT) {
        const int vec = b + (int)threadIdx.x;
        float x[Row<T>::E];
        int c = 0;
        if (vec < v1) {
            row.load(vec, x);
#pragma unroll
            for (int e = 0; e < Row<T>::E; ++e) c += x[e] == v;
        }
        int inc = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int w = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += w;
        }
        if (lane == 31) sh.warp_count[warp] = inc;
        __syncthreads();
        int at = n + inc - c, total = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w < warp) at += sh.warp_count[w];
            total += sh.warp_count[w];
        }
        if (c) {
#pragma unroll
            for (int e = 0; e < Row<T>::E; ++e)
                if (x[e] == v) {
                    if (at < k) best[at] = order_key(v, row.first_id(vec) + e);
                    ++at;
                }
        }
        n += total;
        __syncthreads();
    }
    return min(n, k);
}

// Largest element below `below` (strictly) among the vectors [v0, v1); -inf if there is none.  Whole CTA.
template <typename T>
__device__ float largest_below(const Row<T>& row, int v0, int v1, float below, Shared& sh) {
    float m = -INFINITY;
    for (int vec = v0 + (int)threadIdx.x; vec < v1; vec += NT) {
        float x[Row<T>::E];
        row.load(vec, x);
#pragma unroll
        for (int e = 0; e < Row<T>::E; ++e)
            if (x[e] < below) m = fmaxf(m, x[e]);
    }
    m = warp_max(m);
    if ((threadIdx.x & 31) == 0) sh.bound[threadIdx.x >> 5] = m;
    __syncthreads();
    m = sh.bound[0];
    for (int w = 1; w < NW; ++w) m = fmaxf(m, sh.bound[w]);
    __syncthreads();
    return m;
}

// This CTA's best `k` elements, in order, to sh.best[0..k) (0 = none).  tile_max[tile][thread] holds the maxima, mine = the
// largest of this thread's.
template <typename T>
__device__ void best_of_segment(const Row<T>& row, int v0, int v1, int n_tiles, const float* tile_max, float mine, int k, Shared& sh) {
    constexpr int E = Row<T>::E, VPT = TILE / E;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long* best = sh.best;
    // Of the warps whose threads all have elements (in a short row not all eight), the ceil(k / warps)-th largest thread maximum
    const int active = min(NW, max(1, (v1 - v0) / 32));
    float rest = mine, bound = -INFINITY;
    for (int i = 0; i < (k + active - 1) / active; ++i) {
        bound = warp_max(rest);
        const unsigned who = __ballot_sync(0xffffffffu, rest == bound);
        if (lane == __ffs(who) - 1) rest = -INFINITY;
    }
    if (lane == 0) sh.bound[warp] = bound;
    if (threadIdx.x < 32) best[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.n_cand = sh.n_tile = 0;
    __syncthreads();
    float thr = sh.bound[0];
#pragma unroll
    for (int w = 1; w < NW; ++w)
        if (w < active) thr = fminf(thr, sh.bound[w]);
    // Candidates are the elements from `bar` on: equal ones too, unless there are many of them, or they are -inf (which are never
    // drawn).
    bool many_equal = __syncthreads_count(mine == thr) > MANY_EQUAL && thr > -INFINITY;
    const float bar = many_equal || thr == -INFINITY ? nextafterf(thr, INFINITY) : thr;
    // the tiles to read again: each thread marks its own (at most MAX_TILES), a warp takes places for all of its at once
    unsigned long long marks = 0;
    if (mine >= bar) {
#pragma unroll 4
        for (int i = 0; i < n_tiles; ++i) marks |= (unsigned long long)(tile_max[i * NT + threadIdx.x] >= bar) << i;
    }
    if (__any_sync(0xffffffffu, marks != 0)) {
        for (int at = warp_places(__popcll(marks), &sh.n_tile); marks; ++at, marks &= marks - 1)
            if (at < TILES) sh.tile[at] = (__ffsll(marks) - 1) * NT + (int)threadIdx.x;
    }
    __syncthreads();
    const int n_again = sh.n_tile;
    if (n_again <= TILES) {
        for (int i0 = 0; i0 < n_again * VPT; i0 += NT) {
            const int i = i0 + (int)threadIdx.x, which = i < n_again * VPT ? sh.tile[i / VPT] : 0;
            const int vec = v0 + (which / NT * VPT + i % VPT) * NT + which % NT;
            float x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = -INFINITY;
            if (i < n_again * VPT && vec < v1) row.load(vec, x);
            int count = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) count += x[e] >= bar;
            if (__any_sync(0xffffffffu, count > 0)) {
                int at = warp_places(count, &sh.n_cand);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (x[e] >= bar) {
                        if (at < CAP) sh.cand[at] = order_key(x[e], row.first_id(vec) + e);
                        ++at;
                    }
            }
        }
    }
    __syncthreads();
    int n = sh.n_cand;
    if (n_again > TILES || n > CAP) {
        // More candidates than are held here (a few threads own most of the large elements): value by value.
        int got = 0;
        float below = INFINITY;
        while (got < k) {
            const float top = largest_below(row, v0, v1, below, sh);
            if (top == -INFINITY) break;
            got = append_equal(row, v0, v1, top, best, got, k, sh);
            below = top;
        }
        __syncthreads();
        return;
    }
    if (n > NT) {
        // A weak bound (a mask that leaves some warps nothing): the same again on the values of the candidates.
        unsigned long long mine_too[CAP / NT];
        unsigned top = 0;
#pragma unroll
        for (int j = 0; j < CAP / NT; ++j) {
            const int i = (int)threadIdx.x + j * NT;
            mine_too[j] = i < n ? sh.cand[i] : 0;
            top = max(top, (unsigned)(mine_too[j] >> 32));
        }
        unsigned left = top, least = 0;
        for (int i = 0; i < (k + NW - 1) / NW; ++i) {
            least = __reduce_max_sync(0xffffffffu, left);
            if (lane == __ffs(__ballot_sync(0xffffffffu, left == least)) - 1) left = 0;
        }
        if (lane == 0) sh.warp_count[warp] = (int)least;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) least = min(least, (unsigned)sh.warp_count[w]);
        if (threadIdx.x == 0) sh.n_cand = 0;
        int reach = 0;
#pragma unroll
        for (int j = 0; j < CAP / NT; ++j) reach += __syncthreads_count(mine_too[j] != 0 && (unsigned)(mine_too[j] >> 32) >= least);
        if (reach > NT) {                        // mostly equal ones: they are taken in id order
            many_equal = true;
            thr = key_value((unsigned long long)least << 32);
        }
#pragma unroll
        for (int j = 0; j < CAP / NT; ++j) {
            const unsigned value = (unsigned)(mine_too[j] >> 32);
            const bool in = mine_too[j] != 0 && (reach > NT ? value > least : value >= least);
            const int at = warp_places(in, &sh.n_cand);
            if (in) sh.cand[at] = mine_too[j];
        }
        __syncthreads();
        n = sh.n_cand;
    }
    // position of each candidate = how many others come before it
    if (threadIdx.x < 8) sh.cand[n + threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) {
        const unsigned long long key = sh.cand[i];
        const int pos = count_above(sh.cand, n, key);
        if (pos < k) best[pos] = key;
    }
    if (many_equal && n < k) append_equal(row, v0, v1, thr, best, n, k, sh);
    __syncthreads();
}

// Adds (m, s, t) of one part to another: sums rescaled to the common maximum.  t is kept in units of log 2.
__device__ __forceinline__ void merge(float& m, float& s, float& t, float m2, float s2, float t2) {
    const float M = fmaxf(m, m2);
    const float d1 = fmaxf((m - M) * LOG2E, -300.f), d2 = fmaxf((m2 - M) * LOG2E, -300.f);      // 2^-300 is 0 in fp32
    const float f1 = exp2_fast(d1), f2 = exp2_fast(d2);
    t = f1 * (t + d1 * s) + f2 * (t2 + d2 * s2);
    s = f1 * s + f2 * s2;
    m = M;
}

template <typename T>
__global__ void __launch_bounds__(NT) score_kernel(const ScoreParams p) {
    constexpr int E = Row<T>::E, VPT = TILE / E;
    extern __shared__ float tile_max[];          // [n_tiles][NT], used when alternatives are asked for
    __shared__ Shared sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int C = p.cluster;
    const uint32_t rank = C > 1 ? cluster_rank() : 0u;
    const long long r = blockIdx.x / (unsigned)C;
    if (C > 1) cluster_arrive();                 // every CTA of the cluster has started: waited for before the remote stores
    pdl_wait();
    pdl_launch();

    const Row<T> row(reinterpret_cast<const T*>(p.x) + r * p.ld, p.V);
    const int n_vec = (row.lead + p.V + E - 1) / E;
    const int v0 = min(n_vec, (int)rank * p.seg_vec), v1 = min(n_vec, v0 + p.seg_vec);

    // Two tiles in flight per thread.  All vectors of a tile lie inside the row, except in the first (elements in front of
    // the row) and from last_full on.
    uint4 buf[2][VPT];
    const int first_full = row.lead ? 1 : 0, last_full = (min(v1 * E, row.lead + p.V) / E - v0) / (VPT * NT);
    auto fetch = [&](int i, uint4 (&to)[VPT]) {
        const int vt = v0 + i * VPT * NT + (int)threadIdx.x;
        if (i >= first_full && i < last_full) {
#pragma unroll
            for (int j = 0; j < VPT; ++j) to[j] = row.raw(vt + j * NT, true);
        } else {
            const uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
            for (int j = 0; j < VPT; ++j) to[j] = vt + j * NT < v1 ? row.raw(vt + j * NT, false) : make_uint4(none, none, none, none);
        }
    };
    if (p.n_tiles > 0) fetch(0, buf[0]);
    if (p.n_tiles > 1) fetch(1, buf[1]);

    const int token = p.tokens ? p.tokens[r] : -1;
    const bool has_token = token >= 0 && token < p.V;
    const float x_t = has_token ? to_f32(row.p[token]) : 0.f;
    const float x_next = nextafterf(x_t, INFINITY);      // x >= x_next is x > x_t

    float m = -FLT_MAX, mine = -INFINITY;
    Pair s2 = pair(0.f, 0.f), t2 = pair(0.f, 0.f);       // t2: sum of u 2^u, in units of log 2
    int before = 0;
    auto fold = [&](int i, const uint4 (&from)[VPT]) {
        float x[TILE];
#pragma unroll
        for (int j = 0; j < VPT; ++j) Row<T>::widen(from[j], x + j * E);
        float tm = x[0];
#pragma unroll
        for (int e = 1; e < TILE; ++e) tm = fmaxf(tm, x[e]);
        if (p.top) tile_max[i * NT + threadIdx.x] = tm;
        mine = fmaxf(mine, tm);
        if (tm > m) {
            const float d = fmaxf((m - tm) * LOG2E, -300.f), f = exp2_fast(d);
            const Pair ff = pair(f, f);
            t2 = ff * fma(pair(d, d), s2, t2);
            s2 = ff * s2;
            m = tm;
        }
        const Pair minus_m = pair(-m, -m), log2e = pair(LOG2E, LOG2E);
        Pair sa[2] = {s2, pair(0.f, 0.f)}, ta[2] = {t2, pair(0.f, 0.f)};
#pragma unroll
        for (int e = 0; e < TILE; e += 2) {
            const Pair u = (pair(x[e], x[e + 1]) + minus_m) * log2e;
            const float u0 = lo(u), u1 = hi(u);
            // NaN for a NaN, and for +inf (m is +inf then): such a row is reported as NaN
            const Pair ex = pair(exp2_fast(u0), exp2_fast(u1));
            sa[(e >> 1) & 1] = sa[(e >> 1) & 1] + ex;
            ta[(e >> 1) & 1] = fma(pair(fmaxf(u0, -300.f), fmaxf(u1, -300.f)), ex, ta[(e >> 1) & 1]);
        }
        s2 = sa[0] + sa[1];
        t2 = ta[0] + ta[1];
        // tokens that come before the given one: of most tiles not even the largest does
        if (has_token && tm >= x_t) {
            const int vt = v0 + i * VPT * NT + (int)threadIdx.x, i0 = row.first_id(vt), i1 = row.first_id(vt + (VPT - 1) * NT) + E;
            if (i0 >= 0 && (i1 <= token || (i0 > token && vt + (VPT - 1) * NT < v1))) {
                const float bar = i1 <= token ? x_t : x_next;      // (behind the row's end lie elements read as -inf: never >= x_next)
                int c[4] = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < TILE; ++e) c[e & 3] += x[e] >= bar;
                before += (c[0] + c[1]) + (c[2] + c[3]);
            } else {
#pragma unroll
                for (int j = 0; j < VPT; ++j) {
                    if (vt + j * NT >= v1) continue;
                    const int id = row.first_id(vt + j * NT);
#pragma unroll
                    for (int e = 0; e < E; ++e) before += id + e >= 0 && id + e < p.V && x[j * E + e] >= (id + e < token ? x_t : x_next);
                }
            }
        }
    };
    for (int i = 0; i < p.n_tiles; i += 2) {
        fold(i, buf[0]);
        if (i + 2 < p.n_tiles) fetch(i + 2, buf[0]);
        if (i + 1 < p.n_tiles) fold(i + 1, buf[1]);
        if (i + 3 < p.n_tiles) fetch(i + 3, buf[1]);
    }
    float s = lo(s2) + hi(s2), t = lo(t2) + hi(t2);
    // the warp's sums, brought to its maximum; they meet in the cluster's first CTA
    Partial part;
    part.m = warp_max(m);
    {
        const float d = fmaxf((m - part.m) * LOG2E, -300.f), f = exp2_fast(d);
        part.t = warp_sum(f * (t + d * s));
        part.s = warp_sum(f * s);
        part.before = __reduce_add_sync(0xffffffffu, before);
    }
    if (p.top) best_of_segment(row, v0, v1, p.n_tiles, tile_max, mine, p.top, sh);

    if (C > 1) {
        cluster_wait();
        const uint32_t top0 = cluster_map((uint32_t)__cvta_generic_to_shared(&sh.top[rank][0]), 0);
        const uint32_t part0 = cluster_map((uint32_t)__cvta_generic_to_shared(&sh.part[rank * NW + warp]), 0);
        if (p.top && threadIdx.x < 32)
            asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(top0 + 8 * threadIdx.x), "l"(sh.best[threadIdx.x]) : "memory");
        if (lane == 0)
            asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(part0), "r"(__float_as_uint(part.m)),
                         "r"(__float_as_uint(part.s)), "r"(__float_as_uint(part.t)), "r"(part.before)
                         : "memory");
        cluster_arrive();
        cluster_wait();
        if (rank != 0) return;
    } else {
        if (lane == 0) sh.part[warp] = part;
        __syncthreads();
    }
    if (warp == NW - 1) {                        // (the first C warps order the alternatives meanwhile)
        // C * 8 parts, two per lane at most
        float pm = -FLT_MAX, ps = 0.f, pt = 0.f;
        int pb = 0;
        for (int i = lane; i < C * NW; i += 32) {
            const Partial q = sh.part[i];
            merge(pm, ps, pt, q.m, q.s, q.t);
            pb += q.before;
        }
        const float M = warp_max(pm), d = fmaxf((pm - M) * LOG2E, -300.f), f = exp2_fast(d);
        const float S = warp_sum(f * ps), U = warp_sum(f * (pt + d * ps));
        pb = __reduce_add_sync(0xffffffffu, pb);
        if (lane == 0) {
            const float nan = __int_as_float(0x7fffffff), log_s = logf(S);
            const bool undefined = isnan(S), empty = S == 0.f;         // empty: every logit is -inf
            if (p.lse) p.lse[r] = undefined ? nan : empty ? -INFINITY : M + log_s;
            if (p.entropy) p.entropy[r] = undefined ? nan : empty ? 0.f : log_s - U * LN2 / S;
            if (p.logprob) p.logprob[r] = undefined || !has_token ? nan : empty ? -INFINITY : (x_t - M) - log_s;
            if (p.rank) p.rank[r] = undefined || !has_token ? -1 : pb;
            sh.m = M;
            sh.log_s = undefined ? nan : log_s;
        }
    }
    if (!p.top) return;
    unsigned long long key = 0;
    int pos = threadIdx.x;
    if (C > 1) {
        // C lists, each in order: a key's position is the number of keys before it in all lists (found by bisection)
        if ((int)threadIdx.x < C * 32) key = sh.top[warp][lane];
        if (key) {
            int at[MAX_CLUSTER];
#pragma unroll
            for (int c = 0; c < MAX_CLUSTER; ++c) at[c] = 0;
#pragma unroll 1
            for (int step = 16; step > 0; step >>= 1)
#pragma unroll
                for (int c = 0; c < MAX_CLUSTER; ++c)
                    if (c < C && sh.top[c][at[c] + step - 1] > key) at[c] += step;
            pos = 0;
#pragma unroll
            for (int c = 0; c < MAX_CLUSTER; ++c)
                if (c < C) pos += at[c] + (at[c] == 31 && sh.top[c][31] > key);
        }
    } else if ((int)threadIdx.x < p.top) {
        key = sh.best[threadIdx.x];
    }
    const int found = __syncthreads_count(key != 0);
    const float log_s = sh.log_s;                // NaN: undefined row
    const long long at = r * p.top;
    if (key && pos < p.top) {
        if (p.top_ids) p.top_ids[at + pos] = isnan(log_s) ? -1 : key_id(key);
        if (p.top_lp) p.top_lp[at + pos] = isnan(log_s) ? log_s : (key_value(key) - sh.m) - log_s;
    }
    pos = threadIdx.x;
    if (pos < p.top && pos >= found) {
        if (p.top_ids) p.top_ids[at + pos] = -1;
        if (p.top_lp) p.top_lp[at + pos] = isnan(log_s) ? log_s : -INFINITY;
    }
}

template <typename T>
int run(const ops::Device* dev, ScoreParams p, long long rows, cudaStream_t st) {
    constexpr int E = Row<T>::E, VPT = TILE / E;
    // vectors of a row, whatever its alignment
    const int n_vec = (p.V + E - 2) / E + 1;
    const int tiles = (n_vec + VPT * NT - 1) / (VPT * NT);
    // CTAs per row: rows are cut, while a CTA keeps a tile of its own, until the CTAs are three per SM (256 rows of 151936 bf16: 29 us with
    // two, 35 with four, 44 with eight; one row: 8.7 us with eight, 21 with one).  Long rows that would fill only a few rounds of
    // the four CTAs an SM holds are cut once all the same (1024 rows of 157184 fp32: 117 us, 134 uncut).
    int c = 1;
    while (c < MAX_CLUSTER && c < tiles && (rows * c < 3LL * dev->n_sms || (p.top && (tiles + c - 1) / c > MAX_TILES))) c *= 2;
    const long long slots = 4LL * dev->n_sms;
    if (c == 1 && tiles > 8 && rows < 8 * slots) c = 2;
    p.cluster = c;
    p.n_tiles = (tiles + c - 1) / c;
    p.seg_vec = p.n_tiles * VPT * NT;
    const size_t smem = p.top ? (size_t)p.n_tiles * NT * 4 : 0;
    if (rows * c > 0x7fffffffLL) return ops::fail(S2D2_ERR_UNSUPPORTED, "score_logits: too many rows");
    const cudaError_t e = ops::launch(score_kernel<T>, dim3((unsigned)(rows * c)), NT, smem, c, st, p);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return ops::fail(S2D2_ERR_CUDA, "score_logits: %s", cudaGetErrorString(e));
    }
    return S2D2_OK;
}

}  // namespace

cudaError_t ops::load_score_kernels() {
    cudaError_t e = load(score_kernel<float>, MAX_SMEM);
    return e != cudaSuccess ? e : load(score_kernel<bf16>, MAX_SMEM);
}
}  // namespace s2d2

using namespace s2d2;

extern "C" int s2d2_score_logits(const void* d_logits, int32_t dtype, int64_t n_rows, int32_t vocab, int64_t row_stride,
                                 const int32_t* d_tokens, int32_t top_k, float* d_logprob, int32_t* d_rank, float* d_lse,
                                 float* d_entropy, int32_t* d_top_ids, float* d_top_logprobs, void* cuda_stream) {
    ops::clear_error();
    if (dtype != S2D2_DTYPE_F32 && dtype != S2D2_DTYPE_BF16) return ops::fail(S2D2_ERR_INVALID, "score_logits: dtype");
    if (n_rows < 0) return ops::fail(S2D2_ERR_INVALID, "score_logits: n_rows is negative");
    if (vocab < 1 || vocab > S2D2_SCORE_MAX_VOCAB)
        return ops::fail(S2D2_ERR_INVALID, "score_logits: vocab must be in 1..%d", S2D2_SCORE_MAX_VOCAB);
    if (row_stride < vocab) return ops::fail(S2D2_ERR_INVALID, "score_logits: row_stride is smaller than vocab");
    if (n_rows > 0 && row_stride > (INT64_MAX >> 3) / n_rows) return ops::fail(S2D2_ERR_INVALID, "score_logits: row_stride is too large");
    if (top_k < 0 || top_k > S2D2_SCORE_MAX_TOP)
        return ops::fail(S2D2_ERR_INVALID, "score_logits: top_k must be in 0..%d", S2D2_SCORE_MAX_TOP);
    if ((d_logprob || d_rank) && !d_tokens) return ops::fail(S2D2_ERR_INVALID, "score_logits: log probability and rank need tokens");
    if (top_k > 0 && !d_top_ids && !d_top_logprobs) return ops::fail(S2D2_ERR_INVALID, "score_logits: top_k without an output for it");
    if (top_k == 0 && (d_top_ids || d_top_logprobs)) return ops::fail(S2D2_ERR_INVALID, "score_logits: outputs for alternatives, but top_k is 0");
    if (!d_logprob && !d_rank && !d_lse && !d_entropy && !top_k) return ops::fail(S2D2_ERR_INVALID, "score_logits: no output");
    const ops::Device* dev;
    if (int rc = ops::device(&dev)) return rc;
    if (n_rows == 0) return S2D2_OK;
    const struct {
        const void* p;
        size_t align;
        const char* name;
    } ptrs[] = {{d_logits, dtype == S2D2_DTYPE_F32 ? 4u : 2u, "logits"}, {d_tokens, 4, "tokens"}, {d_logprob, 4, "logprob"},
                {d_rank, 4, "rank"}, {d_lse, 4, "lse"}, {d_entropy, 4, "entropy"}, {d_top_ids, 4, "top_ids"},
                {d_top_logprobs, 4, "top_logprobs"}};
    for (int i = 0; i < 8; ++i)
        if (i == 0 || ptrs[i].p)
            if (int rc = ops::check_ptr(dev, ptrs[i].p, ptrs[i].align, ptrs[i].name)) return rc;
    ScoreParams p = {};
    p.x = d_logits;
    p.ld = row_stride;
    p.V = vocab;
    p.tokens = d_tokens;
    p.top = top_k;
    p.logprob = d_logprob;
    p.rank = d_rank;
    p.lse = d_lse;
    p.entropy = d_entropy;
    p.top_ids = d_top_ids;
    p.top_lp = d_top_logprobs;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    return dtype == S2D2_DTYPE_F32 ? run<float>(dev, p, n_rows, st) : run<bf16>(dev, p, n_rows, st);
}
