// Attention of new rows over a paged cache on the tensor cores (sm_100a, tcgen05), and the join of its parts.
//
//   O[row] = sum_j p_j V[j] / sum_j p_j,   p_j = 2^(s_j - m),   s = scale log2(e) Q K^T,   in one pass over the keys with a running m and sum
//
// The query vectors of a kv head are its sequence's rows times the group of heads that read it (row-major: vector = row * group + head
// of the group), so K and V are read once for a whole group.  An item is (sequence, kv head, 256 query vectors); its units are the
// tiles of 128 keys that any of its rows sees.  All units, in the order of the items, are cut into as many equal ranges as there
// are CTAs: a long cache is shared by many CTAs, many short sequences by few, a ragged batch evenly, and no CTA gets more than
// one unit above the average.  Items that a cut went through leave parts (maximum, sum, weighted values) in the workspace, which
// join_kernel adds up in the order of the keys: deterministic, no tickets.  Lengths are read on the device.
#pragma once
#include "paged_attention.cuh"
#include "tc_ptx.cuh"

namespace s2d2 {
namespace patt {

using namespace tc;

constexpr int KEYS = 128;            // keys of a tile
constexpr int QTILE = 128;           // query vectors of an MMA
constexpr int QROWS = 256;           // of an item
constexpr int MAX_CTAS = 148;
constexpr int THREADS = 384;         // warps 0-3 and 4-7: softmax of the two halves of an item; 8: MMA; 9: copies (10, 11: none)

// ---- instructions ----
__device__ __forceinline__ bool elect() {                      // one lane of a converged warp
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e != 0;
}
__device__ __forceinline__ bool poll(uint64_t* bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return done;
}
// Bounded wait for the phase with the given parity; false when it has run out or another role of the CTA has given up.
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, uint32_t limit, volatile int* abort_flag) {
    for (uint32_t it = 0; it < WAIT_LIMIT; ++it) {
        if ((it & 31u) == 31u && (it >= limit || *abort_flag)) return false;
        if (poll(bar, parity)) return true;
    }
    return false;
}
__device__ __forceinline__ void arrive(uint64_t* bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory"); }
__device__ __forceinline__ void settle() {                     // after a time-out: copies in flight land
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
}
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
        : "memory");
}
// 16 bytes to shared memory, or 16 zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool some) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(some ? 16 : 0) : "memory");
}
// Operand tiles are rows of 128 bytes with the 128-byte swizzle: K-major (Q, K), or MN-major where the rows are the k index (V)
__device__ __forceinline__ uint64_t desc_k(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFF) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr, uint32_t chunk_bytes) {      // the next 64 columns are chunk_bytes further
    return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)(chunk_bytes >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// D fp32, A and B bf16, A K-major, M = 128; B K-major or MN-major
__device__ __forceinline__ uint32_t idesc_bf16(int n, int b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
// D (+)= A B with A in tensor memory: lane = row, a 32-bit column two neighbouring k
__device__ __forceinline__ void umma_bf16_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_ld32_issue(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {      // two operations in one instruction
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
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
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// ---- work ----
struct TileParams {
    Params a;
    int ctas;                        // CTAs that share the units, at most
    int stages;
    int seq_lanes;                   // threads that count a sequence's units: 1, or 32 where sequences have many items
    int control_at;                  // byte offset of Control
    float* part_o;                   // [2 ctas][QROWS][HDP]
    float2* part_ml;                 // [2 ctas][QROWS]: reference, sum
    int4* split;                     // [ctas][2]: the item that CTA c begins and does not end: sequence, kv head, item, last CTA; row0, n, kv, ok (sequence -1: none)
    int* timeouts;
    uint32_t wait_limit;
    int withhold;                    // test tap: nothing is loaded, so that nothing ever completes a stage
};

__device__ __forceinline__ paged::Seq usable_seq(const Params& p, int s) {      // a length that is not followed reads as none
    paged::Seq q = paged::read_seq(p.b, s);
    if (!q.ok) q.kv = 0;
    return q;
}
__device__ __forceinline__ int items_of(const Params& p, int n) { return (n * p.group + QROWS - 1) / QROWS; }
// Units of item qt of a sequence: at least one, so that rows that see nothing are written.
__device__ __forceinline__ int units_of(const Params& p, const paged::Seq& s, int qt) {
    const int last = (min(s.n * p.group, (qt + 1) * QROWS) - 1) / p.group;
    const int end = paged::key_end(p.mask_block, p.row_mask != nullptr, s.n, s.kv, last);
    return max(1, (end + KEYS - 1) / KEYS);
}

// The items of a CTA's range, one after the other.
struct Items {
    int seq, kvh, qt, j;             // the next unit
    long long left;                  // units of the range that are left
    paged::Seq s;                    // of seq
};
struct Item {
    paged::Seq s;
    int seq, kvh, qt, j0, j1, units;
    __device__ __forceinline__ bool whole() const { return j0 == 0 && j1 == units; }
};
__device__ __forceinline__ bool next_item(const Params& p, Items& t, Item& w) {
    if (t.left <= 0) return false;
    while (t.qt >= items_of(p, t.s.n)) {       // behind the last item of a head
        t.qt = 0;
        if (t.s.n == 0 || ++t.kvh >= p.kv_heads) {
            t.kvh = 0;
            if (++t.seq >= p.b.n_seqs) {       // (cannot be: the range ends with the last unit)
                t.left = 0;
                return false;
            }
            t.s = usable_seq(p, t.seq);
        }
    }
    w.s = t.s;
    w.seq = t.seq;
    w.kvh = t.kvh;
    w.qt = t.qt;
    w.j0 = t.j;
    w.units = units_of(p, t.s, t.qt);
    w.j1 = (int)min((long long)w.units, t.j + t.left);
    t.left -= w.j1 - w.j0;
    if (w.j1 == w.units) ++t.qt, t.j = 0;
    else t.j = w.j1;
    return true;
}

struct Setup {
    long long warp_sum[THREADS / 32];
    long long at;                    // units in front of the sequence of the first unit
    long long total, ctas, u1;       // all units, the CTAs that share them, the end of this CTA's range
    Items first;
};

// All threads: the first unit of this CTA's range and its length, from the lengths on the device.  Sequences are counted THREADS / seq_lanes at a time.
__device__ __forceinline__ void plan(const TileParams& tp, Setup& sh, Items& out) {
    const Params& p = tp.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, per = THREADS / tp.seq_lanes;
    auto units = [&](int s) -> long long {      // of a sequence, by seq_lanes threads; the first of them has the sum
        long long n = 0;
        if (s < p.b.n_seqs) {
            const paged::Seq q = usable_seq(p, s);
            const int items = items_of(p, q.n);
            for (int t = tid & (tp.seq_lanes - 1); t < items; t += tp.seq_lanes) n += units_of(p, q, t);
        }
        for (int o = tp.seq_lanes >> 1; o; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
        return (tid & (tp.seq_lanes - 1)) ? 0 : n * p.kv_heads;
    };
    long long total = 0, mine = 0, before = 0;
    // inclusive sums over the CTA's threads; `before` excludes the thread's own
    auto scan = [&](long long v) -> long long {
        long long x = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        __syncthreads();
        if (lane == 31) sh.warp_sum[warp] = x;
        __syncthreads();
        long long all = 0, front = 0;
#pragma unroll
        for (int i = 0; i < THREADS / 32; ++i) {
            if (i == warp) front = all;
            all += sh.warp_sum[i];
        }
        before = front + x - v;
        return all;
    };
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += per) {
        mine = units(s0 + tid / tp.seq_lanes);
        total += scan(mine);
    }
    const long long ctas = min((long long)tp.ctas, total), c = blockIdx.x;
    out.left = 0;
    if (tid == 0) tp.split[2 * c] = make_int4(-1, 0, 0, 0);
    if (c >= ctas) return;
    const long long u0 = total * c / ctas, u1 = total * (c + 1) / ctas;
    long long base = 0;
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += per) {
        if (p.b.n_seqs > per) mine = units(s0 + tid / tp.seq_lanes);
        const long long all = p.b.n_seqs > per ? scan(mine) : total;
        if (mine > 0 && base + before <= u0 && u0 < base + before + mine) {
            sh.first.seq = s0 + tid / tp.seq_lanes;
            sh.at = base + before;
        }
        base += all;
        if (u0 < base) break;                  // (the same for all threads)
    }
    __syncthreads();
    if (warp == 0) {                           // the head and the item inside the sequence
        Items t;
        t.seq = sh.first.seq;
        t.s = usable_seq(p, t.seq);
        const int items = items_of(p, t.s.n);
        long long per_head = 0;
        for (int i = lane; i < items; i += 32) per_head += units_of(p, t.s, i);
#pragma unroll
        for (int o = 16; o; o >>= 1) per_head += __shfl_xor_sync(0xffffffffu, per_head, o);
        long long rest = u0 - sh.at;
        t.kvh = (int)(rest / per_head);
        rest -= t.kvh * per_head;
        for (t.qt = 0;; t.qt += 32) {          // 32 items at a time
            const int n = t.qt + lane < items ? units_of(p, t.s, t.qt + lane) : 0;
            int x = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            const unsigned in = __ballot_sync(0xffffffffu, rest < x);      // inclusive sums grow: the first lane above
            if (in) {
                const int at = __ffs(in) - 1;
                rest -= __shfl_sync(0xffffffffu, x - n, at);
                t.qt += at;
                break;
            }
            rest -= __shfl_sync(0xffffffffu, x, 31);
            if (t.qt + 32 >= items) {          // (cannot be)
                rest = 0;
                break;
            }
        }
        t.j = (int)rest;
        t.left = u1 - u0;
        if (lane == 0) sh.first = t, sh.total = total, sh.ctas = ctas, sh.u1 = u1;
    }
    __syncthreads();
    out = sh.first;
}
// Notes the item that this CTA's range begins and does not end for join_kernel (one thread).
__device__ __forceinline__ void note_split(const TileParams& tp, const Setup& sh, const Item& w) {
    if (w.j0 || w.j1 == w.units) return;
    const long long end = sh.u1 + (w.units - w.j1);          // behind its last unit
    tp.split[2 * blockIdx.x] = make_int4(w.seq, w.kvh, w.qt, (int)((end * sh.ctas + sh.total - 1) / sh.total - 1));
    tp.split[2 * blockIdx.x + 1] = make_int4(w.s.row0, w.s.n, w.s.kv, w.s.ok);
}

constexpr int MAX_STAGES = 12;
struct Control {
    uint64_t full[MAX_STAGES], empty[MAX_STAGES], q_full[2], s_full[2], p_full[2], o_full[2];
    int bad[16];                     // bad[i % 16] == i + 1: item i of this CTA has a page that is not one
    uint32_t tmem_slot;
    int abort_flag;
    Setup setup;
};
struct Ring {                        // position in the ring: stage, and the parity of its current use
    int s = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next(int stages) {
        if (++s == stages) s = 0, parity ^= 1;
    }
};

// Rows whose accumulators are not finite: a NaN or an infinity in a value that a row does not see has come in through a probability of zero (or the
// row sees it: then the result is the same).  The warp takes them again, one by one, without the keys that they do not see.
__device__ __noinline__ void repair_rows(const Params& p, const Item& w, int qv, bool bad, float* part_o, float2* part_ml, int hdp) {
    unsigned todo = __ballot_sync(0xffffffffu, bad);
    const int lane = threadIdx.x & 31;
    while (todo) {
        const int v = __shfl_sync(0xffffffffu, qv, __ffs(todo) - 1);
        todo &= todo - 1;
        const int i = v / p.group, h = w.kvh * p.group + (v - i * p.group);
        const long long row = w.s.row0 + i;
        const paged::View view = paged::row_view(p.mask_block, p.row_mask, w.s, i);
        const RowSum a = row_sum(p, w.seq, w.s.kv, w.kvh, p.q + row * p.q_ld + (long long)h * p.head_dim, view, w.j0 * KEYS, w.j1 * KEYS);
        const int r = v - w.qt * QROWS;
        const float inv = a.l == 0.f ? 0.f : 1.f / a.l;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int d = lane + 32 * e;
            if (w.whole()) {
                if (d < p.head_dim) p.out[row * p.out_ld + (long long)h * p.head_dim + d] = __float2bfloat16_rn(a.o[e] * inv);
            } else if (d < hdp) {
                part_o[r * hdp + d] = d < p.head_dim ? a.o[e] : 0.f;
            }
        }
        if (lane == 0) {
            if (!w.whole()) part_ml[r] = make_float2(a.m, a.l);
            else if (p.lse) p.lse[row * p.heads + h] = a.l == 0.f ? -INFINITY : (a.m + log2f(a.l)) * 0.6931471805599453f;
        }
    }
}

// After a time-out: NaN in all outputs of the CTA's range, those that were finished included.
__device__ __noinline__ void all_nan(const TileParams& tp, const Setup& sh, Items t, int hdp) {
    const Params& p = tp.a;
    const float nan = __int_as_float(0x7fffffff);
    Item w;
    while (next_item(p, t, w)) {
        if (threadIdx.x == 0) note_split(tp, sh, w);
        const int n = min(QROWS, w.s.n * p.group - w.qt * QROWS);
        for (int r = threadIdx.x; r < n; r += THREADS) {
            const int qv = w.qt * QROWS + r, i = qv / p.group, h = w.kvh * p.group + (qv - i * p.group);
            const long long row = w.s.row0 + i;
            if (w.whole()) {
                for (int d = 0; d < p.head_dim; ++d) p.out[row * p.out_ld + (long long)h * p.head_dim + d] = __float2bfloat16_rn(nan);
                if (p.lse) p.lse[row * p.heads + h] = nan;
            } else {
                const int slot = 2 * blockIdx.x + (w.j0 == 0);
                tp.part_ml[(size_t)slot * QROWS + r] = make_float2(0.f, nan);
                for (int d = 0; d < hdp; ++d) tp.part_o[((size_t)slot * QROWS + r) * hdp + d] = nan;
            }
        }
    }
}

// Softmax warps: a thread has a query vector's row of scores, S[128], in a lane of tensor memory.  Its probabilities take the place of the
// scores as bf16 pairs (the left operand of the second product, straight from tensor memory).  The reference m follows the running maximum
// lazily, when that has grown by more than 2^8: the probabilities stay below 256 (their bf16 rounding is relative) and
// the accumulator is rarely rescaled.  That is safe without a wait: scores of tile j are complete after the product with the values of tile j - 1,
// and the next one waits for these probabilities.
template <int HDP>
__device__ __forceinline__ bool softmax_role(const TileParams& tp, Control& ctl, uint8_t* q_tiles, Items t, int half) {
    const Params& p = tp.a;
    volatile int* abort_flag = &ctl.abort_flag;
    const int tid = threadIdx.x & 127, warp = tid >> 5;
    const uint32_t tmem = ctl.tmem_slot, lanes = (uint32_t)(warp * 32) << 16;
    const uint32_t ts = tmem + half * KEYS + lanes, to = tmem + 2 * KEYS + half * HDP + lanes;
    const uint32_t q_addr = smem_u32(q_tiles) + half * (QTILE * HDP * 2);
    const float inv_group = 1.f / (float)p.group;
    uint32_t s_parity = 0, o_parity = 0;

    // Q rows of an item's half: copies of 16 bytes into the swizzled tile; rows and elements that do not exist are zero.
    auto load_q = [&](const Item& w) {
        constexpr int CH = HDP / 8;
        const int q0 = w.qt * QROWS + half * QTILE, nq = w.s.n * p.group;
        const int i0 = q0 / p.group, g0 = q0 - i0 * p.group;
#pragma unroll 4
        for (int k = 0; k < QTILE * CH / 128; ++k) {
            const int idx = tid + k * 128, r = idx / CH, c = idx % CH;
            int i = (int)(((float)(g0 + r) + 0.5f) * inv_group);                  // (g0 + r) / group, of numbers below 2^13
            const int g = g0 + r - i * p.group;
            const bool some = q0 + r < nq && c * 8 < p.head_dim;
            const bf16* src = p.q + (long long)(w.s.row0 + i0 + i) * p.q_ld + (long long)(w.kvh * p.group + g) * p.head_dim + c * 8;
            copy16(q_addr + (c >> 3) * (QTILE * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4), some ? src : p.q, some);
        }
    };
    auto q_ready = [&]() {
        asm volatile("cp.async.wait_all;" ::: "memory");
        fence_async_shared();
        arrive(&ctl.q_full[half]);
    };
    auto active = [&](const Item& w) { return w.s.n * p.group > w.qt * QROWS + half * QTILE; };

    Item w, next;
    bool have = next_item(p, t, w);
    if (have && active(w)) {
        load_q(w);
        q_ready();
    }
    for (int index = 0; have; ++index) {
        const bool have_next = next_item(p, t, next);
        if (half == 0 && tid == 0) note_split(tp, ctl.setup, w);
        if (active(w)) {
            const int qv = w.qt * QROWS + half * QTILE + tid;
            const bool valid = qv < w.s.n * p.group;
            const int i = (valid ? qv : 0) / p.group;
            paged::View view;
            view.lim = 0x7fffffff;
            view.base = 0;
            view.bits = 0;
            if (valid) view = paged::row_view(p.mask_block, p.row_mask, w.s, i);
            float m = -INFINITY, l = 0.f;
            for (int j = w.j0; j < w.j1; ++j) {
                if (!__all_sync(0xffffffffu, wait(&ctl.s_full[half], s_parity, tp.wait_limit, abort_flag))) return false;
                s_parity ^= 1;
                tc_fence_after();
                const bool last = j + 1 == w.j1;
                if (last && have_next && active(next)) load_q(next);              // the scores of this item are complete: its Q tile is free
                uint32_t v[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32_issue(ts + c * 32, v[c]);
                tmem_ld_wait();
                const int key0 = j * KEYS;
                if (!__all_sync(0xffffffffu, key0 + KEYS <= view.lim)) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int n = view.lim - (key0 + 32 * c), d = key0 + 32 * c - view.base;
                        uint32_t seen = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1;
                        if (d >= 0 && d < 64) seen |= (uint32_t)(view.bits >> d);
                        else if (d < 0 && d > -32) seen |= (uint32_t)view.bits << -d;
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (!(seen >> e & 1)) v[c][e] = 0xff800000u;          // -inf
                    }
                }
                float mx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx[c] = __uint_as_float(v[c][0]);
#pragma unroll
                    for (int e = 1; e < 31; e += 2) mx[c] = max3(mx[c], __uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1]));
                    mx[c] = fmaxf(mx[c], __uint_as_float(v[c][31]));
                }
                const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]) * p.scale_log2;
                float alpha = 1.f;
                if (top > m + 8.f || (m == -INFINITY && top > m)) {
                    alpha = exp2_fast(m - top);
                    m = top;
                }
                if (__any_sync(0xffffffffu, alpha != 1.f)) {
                    l *= alpha;
                    if (j > w.j0) {
#pragma unroll
                        for (int c = 0; c < HDP; c += 16) {
                            float o[16];
                            tmem_ld16(to + c, o);
                            uint32_t u[16];
#pragma unroll
                            for (int e = 0; e < 16; ++e) u[e] = __float_as_uint(o[e] * alpha);
                            tmem_st16(to + c, u);
                        }
                    }
                }
                const float ref = m == -INFINITY ? 0.f : -m;
                float factor = p.scale_log2;
                if (__any_sync(0xffffffffu, fabsf(ref) > 1048576.f)) {
                    // s c - m in one operation: m is rounded, so the largest score's difference is off by up to 2^-24 m.  That only moves the
                    // reference, unless m is so large that it leaves the range of the exponentials: then scores are rounded like m first.
                    factor = 1.f;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[c][e] = __float_as_uint(__fmul_rn(__uint_as_float(v[c][e]), p.scale_log2));
                }
                const float2 cc = make_float2(factor, factor), rr = make_float2(ref, ref);
                float2 sum = make_float2(0.f, 0.f), sum1 = sum;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        const float2 x = fma2(make_float2(__uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1])), cc, rr);
                        const float2 y = make_float2(exp2_fast(x.x), exp2_fast(x.y));
                        if (e & 2) sum1 = add2(sum1, y);
                        else sum = add2(sum, y);
                        pk[e / 2] = pack2(y.x, y.y);
                    }
                    tmem_st16(ts + c * 16, pk);
                }
                sum = add2(sum, sum1);
                l += sum.x + sum.y;
                tmem_st_wait();
                tc_fence_before();
                arrive(&ctl.p_full[half]);
                if (last && have_next && active(next)) q_ready();
            }
            // ---- the item's end: divide, or leave a part ----
            if (!__all_sync(0xffffffffu, wait(&ctl.o_full[half], o_parity, tp.wait_limit, abort_flag))) return false;
            o_parity ^= 1;
            tc_fence_after();
            const long long row = w.s.row0 + i;
            const int h = w.kvh * p.group + (qv - i * p.group);
            const int slot = 2 * blockIdx.x + (w.j0 == 0), r = half * QTILE + tid;
            float* part_o = tp.part_o + (size_t)slot * QROWS * HDP;
            float2* part_ml = tp.part_ml + (size_t)slot * QROWS;
            const bool nan = !w.s.ok || *(volatile int*)&ctl.bad[index & 15] == index + 1;
            const float undefined = __int_as_float(0x7fffffff);
            if (nan) l = undefined;
            const float inv = w.whole() ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
            float check = l * 0.f;                                                 // NaN where something is not finite
#pragma unroll
            for (int c = 0; c < HDP; c += 32) {
                uint32_t o[32];
                tmem_ld32_issue(to + c, o);
                tmem_ld_wait();
                float f[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    f[e] = __uint_as_float(o[e]);
                    check = fmaf(f[e], 0.f, check);
                    f[e] = nan ? undefined : f[e] * inv;
                }
                if (!valid) {
                } else if (w.whole()) {
                    bf16* dst = p.out + row * p.out_ld + (long long)h * p.head_dim + c;
#pragma unroll
                    for (int e = 0; e < 32; e += 8)
                        if (c + e < p.head_dim)
                            *reinterpret_cast<uint4*>(dst + e) =
                                make_uint4(pack2(f[e], f[e + 1]), pack2(f[e + 2], f[e + 3]), pack2(f[e + 4], f[e + 5]), pack2(f[e + 6], f[e + 7]));
                } else {
                    float* dst = part_o + (size_t)r * HDP + c;
#pragma unroll
                    for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(dst + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
                }
                __syncwarp();
            }
            tc_fence_before();                                                     // (the next product's start waits for the next probabilities)
            if (valid) {
                if (!w.whole()) part_ml[r] = make_float2(m, l);
                else if (p.lse) p.lse[row * p.heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            }
            const bool bad = valid && !nan && check != check;
            if (__any_sync(0xffffffffu, bad)) {
                __syncwarp();
                repair_rows(p, w, qv, bad, part_o, part_ml, HDP);
            }
        } else if (have_next && active(next)) {
            load_q(next);                                                          // (the tile has been free since the item that it was last loaded for)
            q_ready();
        }
        w = next;
        have = have_next;
    }
    return true;
}

// MMA warp.  Per unit and half: O += P V, then the scores of the half's next unit, so that one half's softmax runs beside the other's MMAs.
template <int HDP>
__device__ __forceinline__ bool mma_role(const TileParams& tp, Control& ctl, uint8_t* q_tiles, uint8_t* ring, Items t) {
    const Params& p = tp.a;
    constexpr int SB = KEYS * HDP * 2;
    volatile int* abort_flag = &ctl.abort_flag;
    const int lane = threadIdx.x & 31;
    const uint32_t tmem = ctl.tmem_slot, idesc_s = idesc_bf16(KEYS, 0), idesc_o = idesc_bf16(HDP, 1);
    const uint32_t qa = smem_u32(q_tiles), ra = smem_u32(ring);
    Ring rk, rv;                                             // K of the next scores, V of the next product
    rv.next(tp.stages);
    uint32_t q_parity[2] = {0, 0}, p_parity[2] = {0, 0};
    auto all = [&](bool ok) { return __all_sync(0xffffffffu, ok); };
    auto scores = [&](int half, int stage) {
        tc_fence_after();
        if (elect()) {
#pragma unroll
            for (int k = 0; k < HDP / 16; ++k)
                umma_bf16(tmem + half * KEYS, desc_k(qa + half * (QTILE * HDP * 2) + (k >> 2) * (QTILE * 128)) + 2 * (k & 3),
                          desc_k(ra + stage * SB + (k >> 2) * (KEYS * 128)) + 2 * (k & 3), idesc_s, k ? 1u : 0u);
            umma_commit(&ctl.s_full[half]);
        }
        __syncwarp();
    };
    auto release = [&](Ring& r) {
        if (elect()) umma_commit(&ctl.empty[r.s]);
        __syncwarp();
        r.next(tp.stages);
        r.next(tp.stages);
    };
    auto active = [&](const Item& w, int half) { return w.s.n * p.group > w.qt * QROWS + half * QTILE; };

    Item w, next;
    bool have = next_item(p, t, w);
    int issued = 0;                                          // halves whose first scores of the item are on their way
    while (have) {
        const bool have_next = next_item(p, t, next);
        int issued_next = 0;
        if (!all(wait(&ctl.full[rk.s], rk.parity, tp.wait_limit, abort_flag))) return false;
#pragma unroll
        for (int half = 0; half < 2; ++half)
            if (active(w, half) && !(issued >> half & 1)) {
                if (!all(wait(&ctl.q_full[half], q_parity[half], tp.wait_limit, abort_flag))) return false;
                q_parity[half] ^= 1;
                scores(half, rk.s);
            }
        release(rk);
        for (int j = w.j0; j < w.j1; ++j) {
            const bool last = j + 1 == w.j1;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (!active(w, half)) continue;
                if (!all(wait(&ctl.p_full[half], p_parity[half], tp.wait_limit, abort_flag))) return false;
                p_parity[half] ^= 1;
                if (half == 0) {                             // (half 0 of an item is never empty)
                    if (!all(wait(&ctl.full[rv.s], rv.parity, tp.wait_limit, abort_flag))) return false;
                    const int n = w.s.kv - j * KEYS;         // tokens of the tile
                    if (n < KEYS) {
                        // values behind the last token are whatever stands in the page or in the ring: a NaN times a probability of zero is a NaN
                        for (int e = lane; e < (KEYS - max(n, 0)) * (HDP / 64) * 8; e += 32) {
                            const int r = max(n, 0) + (e >> 3) / (HDP / 64), c = e & 7, hh = (e >> 3) % (HDP / 64);
                            *reinterpret_cast<uint4*>(ring + rv.s * SB + hh * (KEYS * 128) + r * 128 + c * 16) = make_uint4(0, 0, 0, 0);
                        }
                        fence_async_shared();
                        __syncwarp();
                    }
                }
                tc_fence_after();
                if (elect()) {
#pragma unroll
                    for (int k = 0; k < KEYS / 16; ++k)
                        umma_bf16_ta(tmem + 2 * KEYS + half * HDP, tmem + half * KEYS + k * 8, desc_mn(ra + rv.s * SB + k * 2048, KEYS * 128), idesc_o,
                                     (j > w.j0 || k) ? 1u : 0u);
                    if (last) umma_commit(&ctl.o_full[half]);
                }
                __syncwarp();
                if (!last) {
                    if (half == 0 && !all(wait(&ctl.full[rk.s], rk.parity, tp.wait_limit, abort_flag))) return false;
                    scores(half, rk.s);
                } else if (have_next && active(next, half) && all(poll(&ctl.q_full[half], q_parity[half])) && all(poll(&ctl.full[rk.s], rk.parity))) {
                    q_parity[half] ^= 1;                     // the next item's first scores, if everything is there
                    scores(half, rk.s);
                    issued_next |= 1 << half;
                }
            }
            release(rv);
            if (!last) release(rk);
        }
        w = next;
        have = have_next;
        issued = issued_next;
    }
    return true;
}

// Copy warp: K and V tiles of 128 keys, page by page (a lane per page), in the order in which the MMA warp takes them.
template <int HDP>
__device__ __forceinline__ bool copy_role(const TileParams& tp, Control& ctl, uint8_t* ring, Items t, const CUtensorMap* map_k, const CUtensorMap* map_v) {
    const Params& p = tp.a;
    constexpr int SB = KEYS * HDP * 2;
    const int lane = threadIdx.x & 31, box = min(KEYS, p.c.page_mask + 1), pages = KEYS / box;
    const uint32_t ra = smem_u32(ring);
    Ring r;
    r.parity = 1;                                            // a fresh barrier passes a wait for the phase before its first
    Item w;
    for (int index = 0; next_item(p, t, w); ++index) {
        for (int j = w.j0; j < w.j1; ++j) {
            const int key = j * KEYS + lane * box;
            bool some = lane < pages && key < w.s.kv;
            const int page = some ? paged::page_of(p.b, w.seq, key) : -1;
            if (some && page < 0) {
                *(volatile int*)&ctl.bad[index & 15] = index + 1;
                some = false;
            }
            const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, some)) * box * HDP * 2;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                if (!__all_sync(0xffffffffu, wait(&ctl.empty[r.s], r.parity, tp.wait_limit, &ctl.abort_flag))) return false;
                __syncwarp();
                if (!tp.withhold) {
                    if (lane == 0) mbar_expect_tx(&ctl.full[r.s], bytes);
                    __syncwarp();
                    if (some) {
#pragma unroll
                        for (int h = 0; h < HDP / 64; ++h)
                            load_4d(ra + r.s * SB + h * (KEYS * 128) + lane * box * 128, kv ? map_v : map_k, h * 64, key & p.c.page_mask, w.kvh, page, &ctl.full[r.s]);
                    }
                }
                __syncwarp();
                r.next(tp.stages);
            }
        }
    }
    return true;
}

template <int HDP>
__global__ void __launch_bounds__(THREADS, 1) tile_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ TileParams tp) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* base = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* ring = base + 2 * QTILE * HDP * 2;
    Control& ctl = *(Control*)(base + tp.control_at);
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int s = 0; s < tp.stages; ++s) mbar_init(&ctl.full[s], 1), mbar_init(&ctl.empty[s], 1);
        for (int h = 0; h < 2; ++h) mbar_init(&ctl.q_full[h], 128), mbar_init(&ctl.s_full[h], 1), mbar_init(&ctl.p_full[h], 128), mbar_init(&ctl.o_full[h], 1);
        ctl.abort_flag = 0;
        for (int i = 0; i < 16; ++i) ctl.bad[i] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    }
    if (warp == 8) {
        tmem_alloc(&ctl.tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch();
    // all warps: nothing in front reads or writes what this kernel does, and the bounded waits begin behind it
    pdl_wait();
    Items items;
    plan(tp, ctl.setup, items);
    bool ok = true;
    // 168 registers per thread at launch: 2 x 216 + 72 = 3 x 168
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        ok = softmax_role<HDP>(tp, ctl, base, items, warp >> 2);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 8) ok = mma_role<HDP>(tp, ctl, base, ring, items);
        else if (warp == 9) ok = copy_role<HDP>(tp, ctl, ring, items, &map_k, &map_v);
    }
    if (!ok) *(volatile int*)&ctl.abort_flag = 1;
    __syncwarp();
    __syncthreads();
    const bool failed = *(volatile int*)&ctl.abort_flag;
    if (failed) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        settle();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) tmem_dealloc(ctl.tmem_slot, 512);
    if (failed) {
        if (threadIdx.x == 0) atomicAdd(tp.timeouts, 1);
        all_nan(tp, ctl.setup, items, HDP);
    }
}

// Sum of the parts of an item that the cuts went through, in the order of the keys: block (c, y) takes 32 vectors of the item that CTA c
// began, a warp a vector at a time, a lane four elements (HDP 64: two).
template <int HDP>
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ TileParams tp) {
    constexpr int E = HDP / 32;
    pdl_wait();
    pdl_launch();
    const Params& p = tp.a;
    const int c = blockIdx.x;
    const int4 d = tp.split[2 * c];
    if (d.x < 0) return;
    const int4 s = tp.split[2 * c + 1];
    const int q0 = d.z * QROWS, n = min(QROWS, s.y * p.group - q0), lane = threadIdx.x & 31;
    for (int r = blockIdx.y * 32 + (threadIdx.x >> 5); r < min(n, (int)blockIdx.y * 32 + 32); r += 8) {
        float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 4
        for (int part = c; part <= d.w; ++part) {
            const size_t slot = 2 * part + (part == c);
            const float2 ml = tp.part_ml[slot * QROWS + r];
            const float* src = tp.part_o + (slot * QROWS + r) * HDP + lane * E;
            float x[E];
            if constexpr (E == 4) {
                const float4 v = *reinterpret_cast<const float4*>(src);
                x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
            } else {
                const float2 v = *reinterpret_cast<const float2*>(src);
                x[0] = v.x, x[1] = v.y;
            }
            const float top = fmaxf(m, ml.x), ref = top == -INFINITY ? 0.f : top;
            const float f = exp2_fast(m - ref), g = exp2_fast(ml.x - ref);
            l = l * f + ml.y * g;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = o[e] * f + x[e] * g;
            m = top;
        }
        const int qv = q0 + r, i = qv / p.group, h = d.y * p.group + (qv - i * p.group);
        const long long row = s.x + i;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        bf16* out = p.out + row * p.out_ld + (long long)h * p.head_dim + lane * E;
        if (lane * E < p.head_dim) {
            if constexpr (E == 4) *reinterpret_cast<uint2*>(out) = make_uint2(pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv));
            else *reinterpret_cast<uint32_t*>(out) = pack2(o[0] * inv, o[1] * inv);
        }
        if (p.lse && lane == 0) p.lse[row * p.heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
    }
}

}  // namespace patt
}  // namespace s2d2
