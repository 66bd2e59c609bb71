// Rotary positions, norms of queries and keys with the rotation, and the append to a paged cache: s2d2_rope_frequencies,
// s2d2_qk_rope, s2d2_kv_append, and the checks of the structs of the operators on a paged cache.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace s2d2 {
namespace {

constexpr int RT = 256;              // threads of a CTA
constexpr int MAX_ROWS = 20;         // rows of a CTA, at most

// One of the matrices of a call: [rows, heads, head_dim], rows `ld` elements apart.
struct Mat {
    const void* in;
    void* out;                       // (into the cache: null)
    const float* gain;
    long long in_ld, out_ld;
    int heads;
};
struct RopeParams {
    Mat q, k, v;                     // v: append only
    const int* pos;                  // null: the cache index
    const double* freqs;
    float scale, eps, inv_dim;       // inv_dim: 1 / head_dim
    int rot, interleaved, head_dim;
    long long n_rows;
    int rows_per_cta;
    int tph;                         // threads of a head (a power of two), with vectors
    paged::Batch b;                  // append only
    paged::Cache c;
};

// Where a row of the batch goes.  seq < 0: it belongs to no sequence; page < 0: it has no place in the cache.
struct Place {
    int seq, pos, page, token;
};

// Two operations in one instruction
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
// Eight elements as they stand in memory, and in fp32.
template <typename T>
struct Raw8 {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    }
    __device__ __forceinline__ void values(float2* v) const {
        if (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 a = w[i % (sizeof(T) / 2)];
                v[2 * i] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
                v[2 * i + 1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
            }
        } else {
            const uint32_t x[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = make_float2(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u));
        }
    }
};
// 1 / sqrt(x), the approximation improved by a step of Newton's method: within 2 units in the last place
__device__ __forceinline__ float inverse_root(float x) {
    const float y = rsqrtf(x);
    return x > 0.f && x < INFINITY ? y * fmaf(-0.5f * x * y, y, 1.5f) : y;
}
__device__ __forceinline__ void store8(float* p, const float2* v) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
    *(reinterpret_cast<float4*>(p) + 1) = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
}
__device__ __forceinline__ void store8(bf16* p, const float2* v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[i].x, v[i].y);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// The angle is reduced in turns in 64 bits (an error of 2^-53 of the position's turns), its cosine and sine are taken in fp32.
__device__ __forceinline__ float2 turn(int pos, double freq, float scale) {
    const double t = (double)pos * (freq * 0.15915494309189533577);      // 1 / (2 pi)
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    return make_float2(c * scale, s * scale);
}

template <bool APPEND>
__device__ __forceinline__ Place place_of(const RopeParams& p, long long row, int seq) {      // seq: append only
    Place w;
    if (!APPEND) {
        w.seq = 0;
        w.pos = p.pos && p.rot ? p.pos[row] : 0;
        w.page = w.token = 0;
        return w;
    }
    w.seq = seq;
    w.page = -1;
    w.pos = w.token = 0;
    if (w.seq < 0) return w;
    const paged::Seq s = paged::read_seq(p.b, w.seq);
    const int j = s.kv - s.n + ((int)row - s.row0);
    w.pos = p.pos ? p.pos[row] : j;
    if (s.ok && j >= 0) {
        w.page = paged::page_of(p.b, w.seq, j);
        w.token = j & p.c.page_mask;
    }
    return w;
}
// Rows of a CTA that the search in row0 gave to no sequence: they pad the batch, or row0 decreases and the search went the wrong way.  The CTA looks
// through all sequences; the first that has a row gets it.
__device__ __forceinline__ void find_by_scan(const RopeParams& p, long long row0, int rows, Place* places) {
    __shared__ int owner[MAX_ROWS];
    const bool lost = threadIdx.x < rows && places[threadIdx.x].seq < 0;
    if (threadIdx.x < rows) owner[threadIdx.x] = p.b.n_seqs;
    __syncthreads();
    for (int s = threadIdx.x; s < p.b.n_seqs; s += RT) {
        const paged::Seq q = paged::read_seq(p.b, s);
        if (!q.n) continue;
        const int first = q.row0 - (int)row0, end = min(rows, first + q.n);
        for (int r = max(0, first); r < end; ++r) atomicMin(&owner[r], s);
    }
    __syncthreads();
    if (lost && owner[threadIdx.x] < p.b.n_seqs) places[threadIdx.x] = place_of<true>(p, row0 + threadIdx.x, owner[threadIdx.x]);
    __syncthreads();
}
// First element of a head of the output, or null where there is none.
template <typename TO, bool APPEND>
__device__ __forceinline__ TO* target(const RopeParams& p, const Place& w, int kind, long long row, int head) {
    if (APPEND && kind) {
        if (w.page < 0) return nullptr;
        return (TO*)(kind == 1 ? p.c.k : p.c.v) + w.page * p.c.page_stride + head * p.c.head_stride + w.token * p.c.token_stride;
    }
    return (TO*)(kind ? p.k.out : p.q.out) + row * (kind ? p.k.out_ld : p.q.out_ld) + (long long)head * p.head_dim;
}
// Eight numbers from shared memory.
__device__ __forceinline__ void read8(const float* p, float2* v) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *(reinterpret_cast<const float4*>(p) + 1);
    v[0] = make_float2(a.x, a.y), v[1] = make_float2(a.z, a.w), v[2] = make_float2(b.x, b.y), v[3] = make_float2(b.z, b.w);
}
// (x, y) turned by the angle of cosine c and sine s
__device__ __forceinline__ void rotate(float& x, float& y, float c, float s) {
    const float t = x * c - y * s;
    y = y * c + x * s;
    x = t;
}

// One pass: a head is read once, its squares are summed by the threads that hold it, and it is rotated in registers.  Cosines and sines of
// a row are computed once per CTA, in shared memory, for all of its heads.  Should be bound by memory; what it has to watch is the start of
// a CTA (positions, angles, two barriers: with two rows a CTA 42 us for 8192 x 40 heads, with 14 33 us, 5.1 TB/s) and the number of
// instructions (packed arithmetic 46.7 -> 42 us, loads a round ahead 56 -> 47).
// VEC: a thread holds two groups of eight elements of a head: the two halves of eight pairs (half layout), or two neighbours'.
// Otherwise a warp takes a head, element pair by element pair, and reads it twice where there is a norm.
template <typename TI, typename TO, bool APPEND, bool VEC>
__global__ void __launch_bounds__(RT) rope_kernel(const RopeParams p) {
    extern __shared__ __align__(16) float table[];                   // [rows_per_cta][2][rot / 2]: cosines, sines; VEC: gains of q and k
    __shared__ Place places[MAX_ROWS];
    pdl_wait();
    pdl_launch();
    const long long row0 = (long long)blockIdx.x * p.rows_per_cta;
    const int rows = (int)min((long long)p.rows_per_cta, p.n_rows - row0), pairs = p.rot >> 1, hd = p.head_dim;
    float* gains = table + p.rows_per_cta * p.rot;
    const int heads = p.q.heads + p.k.heads + (APPEND ? p.v.heads : 0);
    const int lanes = VEC ? p.tph : 32, sub = threadIdx.x & (lanes - 1), step = RT / lanes;
    const int total = rows * heads;
    // VEC: groups of eight elements of this thread: the two halves of eight pairs (half layout) or any two; behind the rotated part neighbours
    const int n = hd >> 4, n_rot = p.rot >> 4;               // threads with elements, with pairs
    const int c0 = sub < n_rot ? sub : 2 * sub, c1 = sub < n_rot ? sub + n_rot : 2 * sub + 1;
    struct Task {
        int r, head, kind;                                   // row, head of q, k or v (r >= rows: none)
        const TI* in;
    };
    // the heads of all rows one after the other; this thread's tasks are `step` apart
    const int step_r = step / heads, step_h = step - step_r * heads;
    const long long q_ld = p.q.in_ld, k_ld = p.k.in_ld, v_ld = p.v.in_ld;
    const TI* q_in = (const TI*)p.q.in + row0 * q_ld;
    const TI* k_in = (const TI*)p.k.in + row0 * k_ld;
    const TI* v_in = APPEND ? (const TI*)p.v.in + row0 * v_ld : nullptr;
    int at_r = (int)(threadIdx.x / lanes) / heads, at_h = (int)(threadIdx.x / lanes) - at_r * heads;
    auto next_task = [&]() {
        Task t;
        t.r = at_r, t.head = at_h, t.kind = 0;
        t.in = q_in + at_r * q_ld;
        if (t.head >= p.q.heads) {
            t.head -= p.q.heads, t.kind = 1;
            t.in = k_in + at_r * k_ld;
            if (APPEND && t.head >= p.k.heads) t.head -= p.k.heads, t.kind = 2, t.in = v_in + at_r * v_ld;
        }
        t.in += t.head * hd;
        at_r += step_r, at_h += step_h;
        if (at_h >= heads) at_h -= heads, ++at_r;
        return t;
    };
    // a head's elements are asked for while the angles are computed, or the head before is
    Task t = next_task();
    Raw8<TI> ra, rb;
    if (VEC && t.r < rows && sub < n) ra.load(t.in + c0 * 8), rb.load(t.in + c1 * 8);
    if (VEC) {
        for (int i = threadIdx.x; i < hd; i += RT) {
            if (p.q.gain) gains[i] = p.q.gain[i];
            if (p.k.gain) gains[hd + i] = p.k.gain[i];
        }
    }
    bool lost = false;
    if (threadIdx.x < rows) {
        const int seq = APPEND ? paged::find_seq(p.b, (int)(row0 + threadIdx.x)) : 0;
        places[threadIdx.x] = place_of<APPEND>(p, row0 + threadIdx.x, seq);
        lost = seq < 0;
    }
    if (APPEND) {
        if (__syncthreads_or(lost)) find_by_scan(p, row0, rows, places);
    } else {
        __syncthreads();
    }
    for (int i = threadIdx.x; i < rows * pairs; i += RT) {
        const int r = i / pairs, f = i - r * pairs;
        const float2 cs = turn(places[r].pos, p.freqs[f], p.scale);
        table[r * p.rot + f] = cs.x;
        table[r * p.rot + pairs + f] = cs.y;
    }
    __syncthreads();
    // (whole warps stay together: the sums below are shuffles)
    for (int rounds = (total + step - 1) / step; rounds; --rounds) {
        const Task next = next_task();
        const int r = min(t.r, rows - 1), kind = t.kind;
        const Place w = places[r];
        TO* out = t.r < rows && w.seq >= 0 ? target<TO, APPEND>(p, w, kind, row0 + r, t.head) : nullptr;
        const TI* in = t.in;
        const float* gain = kind == 0 ? p.q.gain : kind == 1 ? p.k.gain : nullptr;
        const float* cosines = table + r * p.rot;
        const float* sines = cosines + pairs;
        const bool turned = !APPEND || kind < 2;
        if (VEC) {
            const bool mine = out && sub < n;
            float2 a[4], b[4], c[4], s[4];
            ra.values(a);
            rb.values(b);
            if (next.r < rows && sub < n) ra.load(next.in + c0 * 8), rb.load(next.in + c1 * 8);
            t = next;
            if (p.q.gain || p.k.gain) {                              // (the same for all threads)
                float2 ss = make_float2(0.f, 0.f);
                if (mine) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) ss = fma2(a[e], a[e], fma2(b[e], b[e], ss));
                }
                float square = ss.x + ss.y;
                for (int o = lanes >> 1; o; o >>= 1) square += __shfl_xor_sync(0xffffffffu, square, o);
                if (gain && mine) {
                    const float inv = inverse_root(fmaf(square, p.inv_dim, p.eps));
                    const float2 ii = make_float2(inv, inv);
                    read8(gains + (kind ? hd : 0) + c0 * 8, c);
                    read8(gains + (kind ? hd : 0) + c1 * 8, s);
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[e] = mul2(mul2(a[e], ii), c[e]), b[e] = mul2(mul2(b[e], ii), s[e]);
                }
            }
            if (!mine) continue;
            if (turned && sub < n_rot) {
                // half: pairs 8 sub .. 8 sub + 7 of a and b.  interleaved: four pairs of a from 4 c0 on, four of b from 4 c1 on
                if (!p.interleaved) {
                    read8(cosines + sub * 8, c);
                    read8(sines + sub * 8, s);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 x = a[e], y = b[e];
                        a[e] = fma2(make_float2(-y.x, -y.y), s[e], mul2(x, c[e]));
                        b[e] = fma2(x, s[e], mul2(y, c[e]));
                    }
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float4 cc = *reinterpret_cast<const float4*>(cosines + (h ? c1 : c0) * 4);
                        const float4 sn = *reinterpret_cast<const float4*>(sines + (h ? c1 : c0) * 4);
                        float2* v = h ? b : a;
                        rotate(v[0].x, v[0].y, cc.x, sn.x);
                        rotate(v[1].x, v[1].y, cc.y, sn.y);
                        rotate(v[2].x, v[2].y, cc.z, sn.z);
                        rotate(v[3].x, v[3].y, cc.w, sn.w);
                    }
                }
            }
            store8(out + c0 * 8, a);
            store8(out + c1 * 8, b);
        } else {
            t = next;
            if (!out) continue;                                      // the same for all lanes
            float inv = 1.f;
            if (gain) {
                float ss = 0.f;
                for (int e = sub; e < hd; e += 32) {
                    const float x = to_f32(in[e]);
                    ss = fmaf(x, x, ss);
                }
                inv = inverse_root(fmaf(warp_sum(ss), p.inv_dim, p.eps));
            }
            const int n_rot = turned ? pairs : 0;
            for (int i = sub; i < n_rot; i += 32) {
                const int e0 = p.interleaved ? 2 * i : i, e1 = p.interleaved ? 2 * i + 1 : i + pairs;
                float x = to_f32(in[e0]), y = to_f32(in[e1]);
                if (gain) x *= inv * gain[e0], y *= inv * gain[e1];
                rotate(x, y, cosines[i], sines[i]);
                out[e0] = from_f32<TO>(x);
                out[e1] = from_f32<TO>(y);
            }
            for (int e = 2 * n_rot + sub; e < hd; e += 32) {
                float x = to_f32(in[e]);
                if (gain) x *= inv * gain[e];
                out[e] = from_f32<TO>(x);
            }
        }
    }
}

template <typename TI, typename TO, bool APPEND>
cudaError_t load_kernels() {
    cudaError_t e = ops::load(rope_kernel<TI, TO, APPEND, true>);
    return e ? e : ops::load(rope_kernel<TI, TO, APPEND, false>);
}

bool aligned(const void* p, long long ld, size_t size) { return ((uintptr_t)p & 15) == 0 && (ld * (long long)size) % 16 == 0; }

int check_mat(const ops::Device* dev, const char* op, const char* name, const Mat& m, int head_dim, size_t in_size, size_t out_size) {
    if (m.in_ld < (long long)m.heads * head_dim || m.in_ld > (1LL << 40))
        return ops::fail(S2D2_ERR_INVALID, "%s: %s_stride must be in heads * head_dim..2^40", op, name);
    if (out_size && (m.out_ld < (long long)m.heads * head_dim || m.out_ld > (1LL << 40)))
        return ops::fail(S2D2_ERR_INVALID, "%s: %s_out_stride must be in heads * head_dim..2^40", op, name);
    if (!dev) return S2D2_OK;
    if (int rc = ops::check_ptr(dev, m.in, in_size, name)) return rc;
    if (out_size)
        if (int rc = ops::check_ptr(dev, m.out, out_size, name)) return rc;
    if (m.gain) return ops::check_ptr(dev, m.gain, 4, "gain");
    return S2D2_OK;
}

int check_rope(const char* op, const s2d2_rope* r, int head_dim) {
    if (r->rot_dim < 0 || r->rot_dim > head_dim || (r->rot_dim & 1)) return ops::fail(S2D2_ERR_INVALID, "%s: rot_dim must be even, 0..head_dim", op);
    if (r->layout != S2D2_ROPE_HALF && r->layout != S2D2_ROPE_INTERLEAVED) return ops::fail(S2D2_ERR_INVALID, "%s: layout", op);
    if (!isfinite(r->scale)) return ops::fail(S2D2_ERR_INVALID, "%s: scale must be finite", op);
    if (!(r->eps >= 0.f) || !isfinite(r->eps)) return ops::fail(S2D2_ERR_INVALID, "%s: eps must be at least 0", op);
    return S2D2_OK;
}

template <bool APPEND>
int launch_rope(const char* op, const ops::Device* dev, RopeParams& p, int dtype, cudaStream_t st) {
    const size_t size = dtype == S2D2_DTYPE_F32 ? 4 : 2;
    const int heads = p.q.heads + p.k.heads + (APPEND ? p.v.heads : 0);
    bool vec = p.head_dim % 16 == 0 && p.rot % 16 == 0;
    for (const Mat* m : {&p.q, &p.k, &p.v})
        if (m->heads) {
            vec = vec && aligned(m->in, m->in_ld, size);
            if (m->out) vec = vec && aligned(m->out, m->out_ld, APPEND ? 2 : size);
        }
    p.inv_dim = 1.f / (float)p.head_dim;
    p.tph = 1;
    while (p.tph * 16 < p.head_dim) p.tph *= 2;                      // at most 32 (head_dim 512)
    const int at_once = vec ? RT / p.tph : RT / 32;
    // Rows of a CTA: as few rounds over the heads as possible in all waves of CTAs (four on an SM), a wave's start counted as three rounds
    // (8192 rows of 40 heads of 128 with norm, bf16: 14 rows, one wave 33 us; 8 rows 34, 9 38, 2 42).
    p.rows_per_cta = 1;
    long long best = 1LL << 62;
    for (int rows = 1; rows <= MAX_ROWS; ++rows) {
        const long long blocks = (p.n_rows + rows - 1) / rows, waves = (blocks + dev->n_sms * 4 - 1) / (dev->n_sms * 4);
        const long long cost = waves * ((rows * heads + at_once - 1) / at_once + 3);
        if (cost < best) best = cost, p.rows_per_cta = rows;
    }
    const long long grid = (p.n_rows + p.rows_per_cta - 1) / p.rows_per_cta;
    if (grid > 0x7fffffffLL) return ops::fail(S2D2_ERR_INVALID, "%s: too many rows", op);
    const size_t smem = ((size_t)p.rows_per_cta * p.rot + (vec ? 2 * p.head_dim : 0)) * 4;       // at most 44 KB
    cudaError_t e;
    if (dtype == S2D2_DTYPE_F32) {
        typedef typename std::conditional<APPEND, bf16, float>::type TO;
        e = vec ? ops::launch(rope_kernel<float, TO, APPEND, true>, dim3((unsigned)grid), RT, smem, 1, st, p)
                : ops::launch(rope_kernel<float, TO, APPEND, false>, dim3((unsigned)grid), RT, smem, 1, st, p);
    } else {
        e = vec ? ops::launch(rope_kernel<bf16, bf16, APPEND, true>, dim3((unsigned)grid), RT, smem, 1, st, p)
                : ops::launch(rope_kernel<bf16, bf16, APPEND, false>, dim3((unsigned)grid), RT, smem, 1, st, p);
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        return ops::fail(S2D2_ERR_CUDA, "%s: %s", op, cudaGetErrorString(e));
    }
    return S2D2_OK;
}

}  // namespace

namespace ops {

cudaError_t load_rope_kernels() {
    cudaError_t e = load_kernels<float, float, false>();
    if (!e) e = load_kernels<bf16, bf16, false>();
    if (!e) e = load_kernels<float, bf16, true>();
    return e ? e : load_kernels<bf16, bf16, true>();
}

int check_rows(const char* op, const s2d2_rows* r) {
    if (!r) return fail(S2D2_ERR_INVALID, "%s: rows: null pointer", op);
    if (r->n_rows < 0) return fail(S2D2_ERR_INVALID, "%s: n_rows must not be negative", op);
    if (r->n_seqs < 0) return fail(S2D2_ERR_INVALID, "%s: n_seqs must not be negative", op);
    if (r->max_pages < 0) return fail(S2D2_ERR_INVALID, "%s: max_pages must not be negative", op);
    if (r->n_rows && (r->max_rows < 1 || r->max_rows > r->n_rows)) return fail(S2D2_ERR_INVALID, "%s: max_rows must be in 1..n_rows", op);
    return S2D2_OK;
}

int check_kv(const char* op, const s2d2_paged_kv* c) {
    if (!c) return fail(S2D2_ERR_INVALID, "%s: kv: null pointer", op);
    if (c->n_pages < 1) return fail(S2D2_ERR_INVALID, "%s: n_pages must be positive", op);
    if (c->page_tokens < 8 || c->page_tokens > S2D2_MAX_PAGE_TOKENS || (c->page_tokens & (c->page_tokens - 1)))
        return fail(S2D2_ERR_INVALID, "%s: page_tokens must be a power of two, 8..%d", op, S2D2_MAX_PAGE_TOKENS);
    if (c->n_kv_heads < 1 || c->n_kv_heads > S2D2_MAX_HEADS) return fail(S2D2_ERR_INVALID, "%s: n_kv_heads must be in 1..%d", op, S2D2_MAX_HEADS);
    if (c->head_dim < 8 || c->head_dim > S2D2_ROPE_MAX_DIM || c->head_dim % 8)
        return fail(S2D2_ERR_INVALID, "%s: head_dim must be a multiple of 8, 8..%d", op, S2D2_ROPE_MAX_DIM);
    const long long t = c->token_stride, h = c->head_stride, g = c->page_stride, top = 1LL << 38;
    if (t % 8 || h % 8 || g % 8 || t < 1 || h < 1 || g < 1 || t > top || h > top || g > top)
        return fail(S2D2_ERR_INVALID, "%s: cache strides must be positive multiples of 8, at most 2^38", op);
    // Nothing may lie on something else: from the smallest stride on, each must be at least what lies inside of it (spans in 128 bits: they are up to 2^69)
    struct Dim {
        long long stride, size;
    } dims[3] = {{t, c->page_tokens}, {h, c->n_kv_heads}, {g, c->n_pages}};
    std::sort(dims, dims + 3, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
    __int128 span = c->head_dim;
    for (const Dim& d : dims) {
        if (d.size == 1) continue;
        if (d.stride < span) return fail(S2D2_ERR_INVALID, "%s: cache strides: elements overlap, or the dimensions do not nest", op);
        span += (__int128)d.stride * (d.size - 1);
    }
    return S2D2_OK;
}

int device_rows(const Device* d, const s2d2_rows* r, const s2d2_paged_kv* c, paged::Batch* out) {
    if (int rc = check_ptr(d, r->d_row0, 4, "row0")) return rc;
    if (int rc = check_ptr(d, r->d_kv_len, 4, "kv_len")) return rc;
    if (r->max_pages)
        if (int rc = check_ptr(d, r->d_pages, 4, "pages")) return rc;
    out->row0 = r->d_row0;
    out->kv_len = r->d_kv_len;
    out->pages = r->d_pages;
    out->n_rows = r->n_rows;
    out->n_seqs = r->n_seqs;
    out->max_pages = r->max_pages;
    out->n_pages = c->n_pages;
    out->page_shift = 0;
    while ((1 << out->page_shift) < c->page_tokens) ++out->page_shift;
    out->max_kv = (long long)r->max_pages * c->page_tokens;
    return S2D2_OK;
}

int device_kv(const Device* d, const s2d2_paged_kv* c, paged::Cache* out) {
    if (int rc = check_ptr(d, c->d_k, 16, "cache keys")) return rc;
    if (int rc = check_ptr(d, c->d_v, 16, "cache values")) return rc;
    out->k = (bf16*)c->d_k;
    out->v = (bf16*)c->d_v;
    out->page_stride = c->page_stride;
    out->head_stride = c->head_stride;
    out->token_stride = c->token_stride;
    out->page_mask = c->page_tokens - 1;
    return S2D2_OK;
}

}  // namespace ops
}  // namespace s2d2

using namespace s2d2;

extern "C" int s2d2_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double original_len, double turns_fast,
                                     double turns_slow, double* freqs, float* scale) {
    ops::clear_error();
    const char* op = "rope_frequencies";
    if (!freqs || !scale) return ops::fail(S2D2_ERR_INVALID, "%s: null pointer", op);
    if (rot_dim < 2 || rot_dim > S2D2_ROPE_MAX_DIM || (rot_dim & 1)) return ops::fail(S2D2_ERR_INVALID, "%s: rot_dim must be even, 2..%d", op, S2D2_ROPE_MAX_DIM);
    if (!(base > 1.) || !isfinite(base)) return ops::fail(S2D2_ERR_INVALID, "%s: base must be above 1", op);
    if (scaling < S2D2_ROPE_SCALING_NONE || scaling > S2D2_ROPE_SCALING_BANDS) return ops::fail(S2D2_ERR_INVALID, "%s: scaling", op);
    if (scaling != S2D2_ROPE_SCALING_NONE && (!(factor >= 1.) || !isfinite(factor))) return ops::fail(S2D2_ERR_INVALID, "%s: factor must be at least 1", op);
    const double two_pi = 6.283185307179586477;
    const bool blend = scaling == S2D2_ROPE_SCALING_YARN || scaling == S2D2_ROPE_SCALING_BANDS;
    if (blend) {
        if (!(original_len > 0.) || !isfinite(original_len)) return ops::fail(S2D2_ERR_INVALID, "%s: original_len must be positive", op);
        if (!(turns_slow > 0.) || !(turns_fast > turns_slow) || !isfinite(turns_fast))
            return ops::fail(S2D2_ERR_INVALID, "%s: turns_fast must be above turns_slow, turns_slow above 0", op);
    }
    if (scaling == S2D2_ROPE_SCALING_NTK) {
        if (rot_dim == 2) return ops::fail(S2D2_ERR_INVALID, "%s: ntk needs rot_dim above 2", op);
        base *= pow(factor, rot_dim / (rot_dim - 2.));
    }
    double low = 0., high = 1.;
    if (scaling == S2D2_ROPE_SCALING_YARN) {
        low = floor(rot_dim * log(original_len / (turns_fast * two_pi)) / (2. * log(base)));
        high = ceil(rot_dim * log(original_len / (turns_slow * two_pi)) / (2. * log(base)));
        low = low < 0. ? 0. : low;
        high = high > rot_dim - 1. ? rot_dim - 1. : high;
        if (high <= low) high = low + 0.001;                         // a step
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = pow(base, -2. * i / rot_dim);
        double slow = scaling == S2D2_ROPE_SCALING_LINEAR ? 1. : 0.;
        if (scaling == S2D2_ROPE_SCALING_YARN) slow = (i - low) / (high - low);
        if (scaling == S2D2_ROPE_SCALING_BANDS) slow = 1. - (original_len * f / two_pi - turns_slow) / (turns_fast - turns_slow);
        slow = slow < 0. ? 0. : slow > 1. ? 1. : slow;
        freqs[i] = slow > 0. ? f / factor * slow + f * (1. - slow) : f;
    }
    *scale = scaling == S2D2_ROPE_SCALING_YARN ? (float)(0.1 * log(factor) + 1.) : 1.f;
    return S2D2_OK;
}

extern "C" int s2d2_qk_rope(const void* d_q, int64_t q_stride, void* d_q_out, int64_t q_out_stride, int32_t n_q_heads, const void* d_k,
                            int64_t k_stride, void* d_k_out, int64_t k_out_stride, int32_t n_k_heads, int32_t dtype, int64_t n_rows,
                            int32_t head_dim, const int32_t* d_pos, const s2d2_rope* rope, void* cuda_stream) {
    ops::clear_error();
    const char* op = "qk_rope";
    if (dtype != S2D2_DTYPE_F32 && dtype != S2D2_DTYPE_BF16) return ops::fail(S2D2_ERR_INVALID, "%s: dtype", op);
    if (n_rows < 0 || n_rows > (1LL << 31)) return ops::fail(S2D2_ERR_INVALID, "%s: n_rows must be in 0..2^31", op);
    if (n_q_heads < 0 || n_q_heads > S2D2_MAX_HEADS) return ops::fail(S2D2_ERR_INVALID, "%s: n_q_heads must be in 0..%d", op, S2D2_MAX_HEADS);
    if (n_k_heads < 0 || n_k_heads > S2D2_MAX_HEADS) return ops::fail(S2D2_ERR_INVALID, "%s: n_k_heads must be in 0..%d", op, S2D2_MAX_HEADS);
    if (head_dim < 1 || head_dim > S2D2_ROPE_MAX_DIM) return ops::fail(S2D2_ERR_INVALID, "%s: head_dim must be in 1..%d", op, S2D2_ROPE_MAX_DIM);
    if (!rope) return ops::fail(S2D2_ERR_INVALID, "%s: rope: null pointer", op);
    if (int rc = check_rope(op, rope, head_dim)) return rc;
    RopeParams p = {};
    p.q = Mat{d_q, d_q_out, rope->d_q_gain, q_stride, q_out_stride, n_q_heads};
    p.k = Mat{d_k, d_k_out, rope->d_k_gain, k_stride, k_out_stride, n_k_heads};
    const size_t size = dtype == S2D2_DTYPE_F32 ? 4 : 2;
    for (int pass = 0; pass < 2; ++pass) {                           // sizes first: refused without a device, too
        const ops::Device* dev = nullptr;
        if (pass) {
            if (int rc = ops::device(&dev)) return rc;
            if (n_rows == 0 || n_q_heads + n_k_heads == 0) return S2D2_OK;
        }
        if (n_q_heads)
            if (int rc = check_mat(dev, op, "q", p.q, head_dim, size, size)) return rc;
        if (n_k_heads)
            if (int rc = check_mat(dev, op, "k", p.k, head_dim, size, size)) return rc;
        if (!pass) continue;
        if (rope->rot_dim) {
            if (int rc = ops::check_ptr(dev, d_pos, 4, "pos")) return rc;
            if (int rc = ops::check_ptr(dev, rope->d_freqs, 8, "freqs")) return rc;
        }
        p.pos = d_pos;
        p.freqs = rope->d_freqs;
        p.scale = rope->scale;
        p.eps = rope->eps;
        p.rot = rope->rot_dim;
        p.interleaved = rope->layout == S2D2_ROPE_INTERLEAVED;
        p.head_dim = head_dim;
        p.n_rows = n_rows;
        return launch_rope<false>(op, dev, p, dtype, (cudaStream_t)cuda_stream);
    }
    return S2D2_OK;
}

extern "C" int s2d2_kv_append(const void* d_q, int64_t q_stride, void* d_q_out, int64_t q_out_stride, int32_t n_q_heads, const void* d_k,
                              int64_t k_stride, const void* d_v, int64_t v_stride, int32_t dtype, const int32_t* d_pos,
                              const s2d2_rope* rope, const s2d2_rows* rows, const s2d2_paged_kv* kv, void* cuda_stream) {
    ops::clear_error();
    const char* op = "kv_append";
    if (dtype != S2D2_DTYPE_F32 && dtype != S2D2_DTYPE_BF16) return ops::fail(S2D2_ERR_INVALID, "%s: dtype", op);
    if (n_q_heads < 0 || n_q_heads > S2D2_MAX_HEADS) return ops::fail(S2D2_ERR_INVALID, "%s: n_q_heads must be in 0..%d", op, S2D2_MAX_HEADS);
    if (int rc = ops::check_rows(op, rows)) return rc;
    if (int rc = ops::check_kv(op, kv)) return rc;
    if (rope)
        if (int rc = check_rope(op, rope, kv->head_dim)) return rc;
    RopeParams p = {};
    const int hd = kv->head_dim;
    if (d_q && n_q_heads) p.q = Mat{d_q, d_q_out, rope ? rope->d_q_gain : nullptr, q_stride, q_out_stride, n_q_heads};
    p.k = Mat{d_k, nullptr, rope ? rope->d_k_gain : nullptr, k_stride, 0, kv->n_kv_heads};
    p.v = Mat{d_v, nullptr, nullptr, v_stride, 0, kv->n_kv_heads};
    const size_t size = dtype == S2D2_DTYPE_F32 ? 4 : 2;
    for (int pass = 0; pass < 2; ++pass) {
        const ops::Device* dev = nullptr;
        if (pass) {
            if (int rc = ops::device(&dev)) return rc;
            if (rows->n_rows == 0 || rows->n_seqs == 0) return S2D2_OK;
        }
        if (p.q.heads)
            if (int rc = check_mat(dev, op, "q", p.q, hd, size, 2)) return rc;
        if (int rc = check_mat(dev, op, "k", p.k, hd, size, 0)) return rc;
        if (int rc = check_mat(dev, op, "v", p.v, hd, size, 0)) return rc;
        if (!pass) continue;
        if (int rc = ops::device_rows(dev, rows, kv, &p.b)) return rc;
        if (int rc = ops::device_kv(dev, kv, &p.c)) return rc;
        if (d_pos)
            if (int rc = ops::check_ptr(dev, d_pos, 4, "pos")) return rc;
        if (rope && rope->rot_dim)
            if (int rc = ops::check_ptr(dev, rope->d_freqs, 8, "freqs")) return rc;
        p.pos = d_pos;
        if (rope) {
            p.freqs = rope->d_freqs;
            p.scale = rope->scale;
            p.eps = rope->eps;
            p.rot = rope->rot_dim;
            p.interleaved = rope->layout == S2D2_ROPE_INTERLEAVED;
        }
        p.head_dim = hd;
        p.n_rows = rows->n_rows;
        return launch_rope<true>(op, dev, p, dtype, (cudaStream_t)cuda_stream);
    }
    return S2D2_OK;
}
