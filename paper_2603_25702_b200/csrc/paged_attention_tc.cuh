// Attention of new rows over a paged cache on the tensor cores (sm_100a, tcgen05), and the join of its parts.
//
//   O[row] = sum_j p_j V[j] / sum_j p_j,   p_j = 2^(s_j - m),   s = scale log2(e) Q K^T,   in one pass over the keys with a running m and sum
//
// The query vectors of a kv head are its sequence's rows times the group of heads that read it, so K and V are read once for a whole group:
// a MMA tile of 128 takes as many whole rows as fit (128 / group; of a group above 128 the largest part of it that divides it).  An item is
// (sequence, heads, one or two tiles of query vectors, its halves); its units are the tiles of 128 keys that any of its rows sees.  All units, in the order of the items, are cut into as many equal ranges as there
// are CTAs (an item counts one unit more than it has: its start and its end cost about as much), so that a long cache is shared by many
// CTAs, many short sequences by few, and a ragged batch evenly.  Items that a cut went through leave parts (maximum, sum, weighted
// values) in the workspace, which join_kernel adds up in the order of the keys: deterministic, no tickets.  Lengths are read on
// the device.
#pragma once
#include "paged_attention.cuh"
#include "tc_ptx.cuh"

namespace s2d2 {
namespace patt {

using namespace tc;

constexpr int KEYS = 128;            // keys of a tile
constexpr int QTILE = 128;           // query vectors of an MMA
constexpr int MAX_CTAS = 148;
// NH: MMA tiles of query vectors in an item, its halves (2: many rows; 1: few).  Warps 0 .. 4 NH - 1: softmax; then items and copies, Q,
// and NH for the MMAs.
__host__ __device__ constexpr int threads(int nh) { return 128 * nh + 128; }

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
// Whether the phase is over, without waiting (poll() may wait for some microseconds).
__device__ __forceinline__ bool peek(uint64_t* bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return done;
}
// What ends or lengthens the waits of a CTA
struct Watch {
    int abort;                       // a role has given up
    int progress;                    // counts blocks of keys of rows that are taken again: what waits for them does not give up
};
// Bounded wait for the phase with the given parity; false when it has run out (`limit` polls without progress) or another role of the CTA has given
// up.  (Not unrolled: that was most of the kernel's code, 200 KB, which had to be fetched again and again; a wait that was over took 300 cycles instead
// of 75.)
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, uint32_t limit, const volatile Watch* watch) {
    int progress = 0;
#pragma unroll 1
    for (uint32_t it = 0;; ++it) {
        if (poll(bar, parity)) return true;
        if ((it & 31u) != 31u) continue;
        if (watch->abort) return false;
        if (it >= limit) {
            const int now = watch->progress;
            if (now == progress) return false;
            progress = now;
            it = 0;
        }
    }
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
// Operand tiles are rows of 128 bytes with the 128-byte swizzle: K-major (Q, K), or MN-major where the rows are the k index (V)
__device__ __forceinline__ uint64_t desc_k(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFF) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr, uint32_t chunk_bytes) {      // the next 64 columns are chunk_bytes further
    return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)(chunk_bytes >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
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
__device__ __forceinline__ float max3_nan(float a, float b, float c) {      // NaN if there is one
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
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
    int gs, vsub;                    // heads of a tile; tiles' heads in a group
    int rows_half;                   // rows of a tile: 128 / gs
    uint32_t items_magic;            // n / (rows of an item) = n * items_magic >> 32 for n below 2^23; 0: an item is a row
    int seq_lanes;                   // lanes that count a sequence's units: a power of two up to 32
    int control_at;                  // byte offset of Control
    float* part_o;                   // [2 ctas][128 NH][HDP]
    float2* part_ml;                 // [2 ctas][128 NH]: reference, sum
    int4* split;                     // [ctas][2]: the item that CTA c begins and does not end: first head (-1: none), item, last CTA, row0; n
    int* timeouts;
    uint32_t wait_limit;
    int out_32;                      // rows of heads of the output are multiples of 32 bytes and aligned to them
    int withhold;                    // test tap: nothing is loaded, so that nothing ever completes a stage
};

__device__ __forceinline__ paged::Seq usable_seq(const Params& p, int s) {      // a length that is not followed reads as none
    paged::Seq q = paged::read_seq(p.b, s);
    if (!q.ok) q.kv = 0;
    return q;
}
template <int NH>
__device__ __forceinline__ int items_of(const TileParams& tp, int n) {
    return tp.items_magic ? (int)__umulhi((uint32_t)(n + NH * tp.rows_half - 1), tp.items_magic) : n;
}
// Units of item qt of a sequence: at least one, so that rows that see nothing are written.
template <int NH>
__device__ __forceinline__ int units_of(const TileParams& tp, const paged::Seq& s, int qt) {
    const int end = paged::key_end(tp.a.mask_block, tp.a.row_mask != nullptr, s.n, s.kv, min(s.n, (qt + 1) * NH * tp.rows_half) - 1);
    return max(1, (end + KEYS - 1) / KEYS);
}

// The items of a CTA's range, one after the other.  Ranges are in costs: an item has `extra` in front of its units.
struct Items {
    int seq, vh, qt, extra;
    int at, left;                    // costs of item qt in front of the range, costs of the range that are left
    paged::Seq s;                    // of seq
};
struct Item {
    paged::Seq s;
    int seq, kvh, head0, qt, j0, j1, units;     // head0: first query head; j1 = 0: there are no more
    __device__ __forceinline__ bool whole() const { return j0 == 0 && j1 == units; }
};
template <int NH>
__device__ __forceinline__ bool next_item(const TileParams& tp, Items& t, Item& w) {
    const Params& p = tp.a;
    while (t.left > 0) {
        while (t.qt >= items_of<NH>(tp, t.s.n)) {      // behind the last item of these heads
            t.qt = 0;
            if (t.s.n == 0 || ++t.vh >= p.kv_heads * tp.vsub) {
                t.vh = 0;
                if (++t.seq >= p.b.n_seqs) {           // (cannot be: the range ends with the last unit)
                    t.left = 0;
                    return false;
                }
                t.s = usable_seq(p, t.seq);
            }
        }
        w.s = t.s;
        w.seq = t.seq;
        w.kvh = tp.vsub == 1 ? t.vh : t.vh / tp.vsub;
        w.head0 = t.vh * tp.gs;
        w.qt = t.qt;
        w.units = units_of<NH>(tp, t.s, t.qt);
        const int end = min(t.at + t.left, w.units + t.extra);
        w.j0 = max(0, t.at - t.extra);
        w.j1 = max(0, end - t.extra);
        t.left -= end - t.at;
        t.at = 0;
        ++t.qt;
        if (w.j1 > w.j0) return true;                  // else the cut went through the extra
    }
    return false;
}

struct Setup {
    uint32_t u1, base, more;         // end of this CTA's range; costs of a CTA, CTAs that have one more
    Items first;
};

// One warp: whether a sequence with rows begins in front of the end of an earlier one that has some.
__device__ __noinline__ bool out_of_order(const Params& p) {
    const int lane = threadIdx.x & 31;
    int front = 0;                             // end of the rows so far
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += 32) {
        int first = 0, end = 0;
        if (s0 + lane < p.b.n_seqs) {
            const paged::Seq q = paged::read_seq(p.b, s0 + lane);
            if (q.n) first = q.row0, end = q.row0 + q.n;
        }
        int most = end;                        // inclusive maxima
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, most, o);
            if (lane >= o) most = max(most, y);
        }
        const int before = __shfl_up_sync(0xffffffffu, most, 1);
        if (__any_sync(0xffffffffu, end && first < max(front, lane ? before : 0))) return true;
        front = max(front, __shfl_sync(0xffffffffu, most, 31));
    }
    return false;
}

// One warp: the begin of this CTA's range and its length, from the lengths on the device.  Sequences are counted 32 / seq_lanes at a time.
template <int NH>
__device__ __forceinline__ void plan(const TileParams& tp, Setup& sh, Items& out) {
    const Params& p = tp.a;
    const int lane = threadIdx.x & 31, per = 32 / tp.seq_lanes, heads = p.kv_heads * tp.vsub;
    bool falls = false;                        // row0 decreases somewhere
    // items (x) and units (y) of a sequence, by seq_lanes lanes; the first of them has the sums
    auto count = [&](int s) {
        uint2 n = make_uint2(0, 0);
        if (s < p.b.n_seqs) {
            const paged::Seq q = usable_seq(p, s);
            falls |= p.b.row0[s + 1] < q.row0;
            const int items = items_of<NH>(tp, q.n);
            for (int t = lane & (tp.seq_lanes - 1); t < items; t += tp.seq_lanes) n.y += units_of<NH>(tp, q, t), ++n.x;
        }
        for (int o = tp.seq_lanes >> 1; o; o >>= 1) n.x += __shfl_xor_sync(0xffffffffu, n.x, o), n.y += __shfl_xor_sync(0xffffffffu, n.y, o);
        return (lane & (tp.seq_lanes - 1)) ? make_uint2(0, 0) : n;
    };
    uint2 mine = make_uint2(0, 0);
    uint32_t items = 0, units = 0;
#pragma unroll 2
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += per) {
        mine = count(s0 + lane / tp.seq_lanes);
        items += mine.x, units += mine.y;
    }
    items = __reduce_add_sync(0xffffffffu, items);
    units = __reduce_add_sync(0xffffffffu, units);
    out.left = 0;
    if (lane == 0) tp.split[2 * blockIdx.x] = make_int4(-1, 0, 0, 0), sh.first.left = 0;
    // With less than a unit per CTA every one of them counts more than an even spread of starts and ends (tokens over 1222: 80 units 12.2 us without
    // the extra, 12.4 with it; 160 units 13.4, 13.2; 320 16.5, 15.4; 800 21.3, 20.1; a ragged batch of 776 units 41.5, 31.0)
    const uint32_t extra = (unsigned long long)units * heads > tp.ctas ? 1 : 0;
    const uint32_t total = (units + extra * items) * heads, ctas = min((uint32_t)tp.ctas, total), c = blockIdx.x;
    if (c >= ctas) return;
    // Rows of several sequences would be written by several CTAs, and the host's bound on the costs would not hold: such a list is not followed at all.
    // (One that never decreases has none.)
    if (__any_sync(0xffffffffu, falls) && out_of_order(p)) return;
    const uint32_t base = total / ctas, more = total - base * ctas;
    const uint32_t u0 = c * base + min(c, more), u1 = u0 + base + (c < more);
    uint32_t front = 0, at = 0;
    int seq = 0;
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += per) {
        if (p.b.n_seqs > per) mine = count(s0 + lane / tp.seq_lanes);
        const uint32_t cost = (mine.y + extra * mine.x) * heads;
        uint32_t x = cost;                     // inclusive sums
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        const unsigned in = __ballot_sync(0xffffffffu, u0 < front + x);
        if (in) {                              // the first lane whose sum is above
            const int i = __ffs(in) - 1;
            seq = s0 + i / tp.seq_lanes;
            at = u0 - (front + __shfl_sync(0xffffffffu, x - cost, i));
            break;
        }
        front += __shfl_sync(0xffffffffu, x, 31);
    }
    // the heads and the item inside the sequence
    Items t;
    t.seq = seq;
    t.s = usable_seq(p, seq);
    t.extra = (int)extra;
    const int n_items = items_of<NH>(tp, t.s.n);
    uint32_t per_head = 0;
    for (int i = lane; i < n_items; i += 32) per_head += units_of<NH>(tp, t.s, i) + extra;
    per_head = __reduce_add_sync(0xffffffffu, per_head);
    t.vh = at / per_head;
    at -= t.vh * per_head;
    for (t.qt = 0; t.qt + 1 < n_items; t.qt += 32) {          // 32 items at a time
        const uint32_t n = t.qt + lane < n_items ? units_of<NH>(tp, t.s, t.qt + lane) + extra : 0;
        uint32_t x = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        const unsigned in = __ballot_sync(0xffffffffu, at < x);
        if (in) {
            const int i = __ffs(in) - 1;
            at -= __shfl_sync(0xffffffffu, x - n, i);
            t.qt += i;
            break;
        }
        at -= __shfl_sync(0xffffffffu, x, 31);
    }
    t.at = (int)at;
    t.left = (int)(u1 - u0);
    if (lane == 0) sh.first = t, sh.u1 = u1, sh.base = base, sh.more = more;
    __syncwarp();
    out = t;
}
// Notes the item that this CTA's range begins and does not end for join_kernel (one thread).
__device__ __forceinline__ void note_split(const TileParams& tp, const Setup& sh, const Item& w) {
    if (w.j0 || w.j1 == w.units) return;
    const uint32_t last = sh.u1 + (w.units - w.j1) - 1, longer = sh.more * (sh.base + 1);      // its last unit; costs of the CTAs with one more
    const uint32_t cta = last < longer ? last / (sh.base + 1) : sh.more + (last - longer) / sh.base;
    tp.split[2 * blockIdx.x] = make_int4(w.head0, w.qt, (int)cta, w.s.row0);
    tp.split[2 * blockIdx.x + 1] = make_int4(w.s.n, 0, 0, 0);
}

constexpr int MAX_STAGES = 12;
constexpr int ITEMS = 8;             // that the copy warp may be ahead of the others
struct Control {
    uint64_t full[MAX_STAGES], empty[MAX_STAGES], item_full[ITEMS], item_empty[ITEMS];
    // Per half and buffer (a unit's first and second 64 keys).  A barrier of a buffer cannot be two phases ahead of who waits for it.
    uint64_t s_full[2][2], o_full[2][2], p_full[2][2];
    uint64_t q_full[2], q_empty[2];                                          // per half
    Item items[ITEMS];
    int bad[2 * ITEMS];                    // bad[i % 16] == i + 1: item i of this CTA has a page that is not one
    uint32_t tmem_slot;
    Watch watch;
    Setup setup;
};
constexpr int BARRIERS = 2 * MAX_STAGES + 2 * ITEMS + 16;
struct Ring {                        // position in the ring: stage, and the parity of its current use
    int s = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next(int stages) {
        if (++s == stages) s = 0, parity ^= 1;
    }
};

// Rows whose accumulators are not finite: a NaN or an infinity in a value that a row does not see has come in through a probability of zero (or the
// row sees it: then the result is the same).  The warp takes them again, one by one, without the keys that they do not see.  `i`, `h`: this
// lane's row of the sequence and head; `slot`: its place in the parts; `progress` counts for the roles that wait.
__device__ __noinline__ void repair_rows(const TileParams& tp, const Item& w, int i, int h, bool bad, unsigned long long slot, int hdp, int* progress) {
    const Params& p = tp.a;
    unsigned todo = __ballot_sync(0xffffffffu, bad);
    const int lane = threadIdx.x & 31;
    while (todo) {
        const int from = __ffs(todo) - 1;
        todo &= todo - 1;
        const int ri = __shfl_sync(0xffffffffu, i, from), rh = __shfl_sync(0xffffffffu, h, from);
        const unsigned long long rs = __shfl_sync(0xffffffffu, slot, from);
        const long long row = w.s.row0 + ri;
        const paged::View view = paged::row_view(p.mask_block, p.row_mask, w.s, ri);
        const RowSum a = row_sum(p, w.seq, w.s.kv, w.kvh, p.q + row * p.q_ld + (long long)rh * p.head_dim, view, w.j0 * KEYS, w.j1 * KEYS, progress);
        const float inv = a.l == 0.f ? 0.f : 1.f / a.l;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int d = lane + 32 * e;
            if (w.whole()) {
                if (d < p.head_dim) p.out[row * p.out_ld + (long long)rh * p.head_dim + d] = __float2bfloat16_rn(a.o[e] * inv);
            } else if (d < hdp) {
                tp.part_o[rs * hdp + d] = d < p.head_dim ? a.o[e] : 0.f;
            }
        }
        if (lane == 0) {
            if (!w.whole()) tp.part_ml[rs] = make_float2(a.m, a.l);
            else if (p.lse) p.lse[row * p.heads + rh] = a.l == 0.f ? -INFINITY : (a.m + log2f(a.l)) * 0.6931471805599453f;
        }
    }
}

// After a time-out: NaN in all outputs of the CTA's range, those that were finished included.
template <int NH>
__device__ __noinline__ void all_nan(const TileParams& tp, const Setup& sh, int hdp) {
    const Params& p = tp.a;
    const float nan = __int_as_float(0x7fffffff);
    Items t = sh.first;
    Item w;
    while (next_item<NH>(tp, t, w)) {
        if (threadIdx.x == 0) note_split(tp, sh, w);
        for (int r = threadIdx.x; r < 128 * NH; r += threads(NH)) {
            const int ti = (r & 127) / tp.gs, i = (w.qt * NH + (r >> 7)) * tp.rows_half + ti, h = w.head0 + (r & 127) - ti * tp.gs;
            if (ti >= tp.rows_half || i >= w.s.n) continue;
            const long long row = w.s.row0 + i;
            if (w.whole()) {
                for (int d = 0; d < p.head_dim; ++d) p.out[row * p.out_ld + (long long)h * p.head_dim + d] = __float2bfloat16_rn(nan);
                if (p.lse) p.lse[row * p.heads + h] = nan;
            } else {
                const size_t at = (size_t)(2 * blockIdx.x + (w.j0 == 0)) * (128 * NH) + r;
                tp.part_ml[at] = make_float2(0.f, nan);
                for (int d = 0; d < hdp; ++d) tp.part_o[at * hdp + d] = nan;
            }
        }
    }
}

// Tensor memory: columns 0-255 scores, two buffers of 64 keys for each half; probabilities (bf16 pairs, 32 columns) stand over the scores that
// they come from; accumulators of the halves from column 256 on.
constexpr int STEP = 64;

// The items of this CTA as its copy warp lists them, in order; every warp gives them back.
struct Listed {
    int index = 0;
    __device__ __forceinline__ bool get(Control& ctl, const TileParams& tp, Item& w) const {
        if (!__all_sync(0xffffffffu, wait(&ctl.item_full[index % ITEMS], index / ITEMS & 1, tp.wait_limit, &ctl.watch))) return false;
        w = ctl.items[index % ITEMS];
        return true;
    }
    __device__ __forceinline__ void done(Control& ctl) {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) arrive(&ctl.item_empty[index % ITEMS]);
        ++index;
    }
};
template <int NH>
__device__ __forceinline__ bool active(const TileParams& tp, const Item& w, int half) { return half == 0 || w.s.n > (w.qt * NH + half) * tp.rows_half; }

// 32 bytes of a lane's own row: with one store, a whole sector, where rows are aligned to that.
__device__ __forceinline__ void store32(void* dst, const uint32_t* v, bool aligned, bool second) {
    if (aligned) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]),
                     "r"(v[6]), "r"(v[7])
                     : "memory");
    } else {
        *reinterpret_cast<uint4*>(dst) = make_uint4(v[0], v[1], v[2], v[3]);
        if (second) *(reinterpret_cast<uint4*>(dst) + 1) = make_uint4(v[4], v[5], v[6], v[7]);
    }
}

// 32 probabilities 2^(s factor - m) of scores s as bf16 pairs, and what that rounding left, rounded like them (REST); adds them to `sum`, four chains.
template <bool REST>
__device__ __forceinline__ void probabilities(const uint32_t (&v)[32], float factor, float minus_m, uint32_t (&pk)[16], uint32_t (&rest)[16], float2 (&sum)[2]) {
    const float2 cc = make_float2(factor, factor), rr = make_float2(minus_m, minus_m);
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
        const float2 x = fma2(make_float2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), cc, rr), y = make_float2(exp2_fast(x.x), exp2_fast(x.y));
        sum[e >> 1 & 1] = add2(sum[e >> 1 & 1], y);
        pk[e / 2] = pack2(y.x, y.y);
        if (REST) {
            const float2 d = add2(y, make_float2(-__uint_as_float(pk[e / 2] << 16), -__uint_as_float(pk[e / 2] & 0xffff0000u)));
            rest[e / 2] = pack2(d.x, d.y);
        }
    }
}
__device__ __forceinline__ float first_reference(const uint32_t (&v)[32]) {
    float m = fmaxf(__uint_as_float(v[0]), __uint_as_float(v[31]));
#pragma unroll
    for (int e = 1; e < 31; e += 2) asm("max.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(__uint_as_float(v[e])), "f"(__uint_as_float(v[e + 1])));
    return m;
}
// -inf for the keys from `key` on that are not seen
__device__ __forceinline__ void mask32(uint32_t (&v)[32], const paged::View& view, int key) {
    const int n = view.lim - key, d = key - view.base;
    uint32_t seen = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1;
    if (d >= 0 && d < 64) seen |= (uint32_t)(view.bits >> d);
    else if (d < 0 && d > -32) seen |= (uint32_t)view.bits << -d;
#pragma unroll
    for (int e = 0; e < 32; ++e)
        if (!(seen >> e & 1)) v[e] = 0xff800000u;
}

// The reference goes up by a whole number, so far that `total` is below 1 against it; gives the factor of what was added up against the old one.
__device__ __forceinline__ float raise_reference(float& m, float& l, float total) {
    const float before = m;
    m += (float)((int)(__float_as_uint(total) >> 23) - 126);
    const float alpha = exp2_fast(before - m);
    l *= alpha;
    return alpha;
}

// Softmax warps: a thread has a query vector's row of scores, a lane of tensor memory, and takes it in steps of 64 keys.  It leaves the probabilities
// over the scores as bf16 pairs, the left operand of the second product.  The scores of the next step are computed meanwhile (two buffers
// of 64 columns; with one of 128, the most that fits beside the accumulators, every unit waited 1500 cycles for its scores).  The
// reference m is not the maximum: it is the maximum of the first 32 scores with one that the row sees, and goes up by a whole number when a step's
// probabilities add up to more than 512, from the next step on.  So no maximum is taken, the accumulator is rarely rescaled, and nothing
// has to wait for a sum; probabilities above 1 lose nothing, their rounding to bf16 is relative.  A row whose probabilities add up to more
// than 2^100 in a step, the last of an item or part included, or whose reference is above 2^20, where s c - m is too coarse, is taken again at the end
// (repair_rows), like one with a NaN.
// Rounding: with probabilities in bf16 the output is off by 1.4 times the rounding of the output itself (0.0023 of it, root mean square; 0.0016).  Items of
// one tile, bound by memory, also take what the rounding left of the first 32 of a step's 64 probabilities: 1.2 times, for 3 % of
// the time (131072 tokens 94.5 -> 97.7 us); of all 64 it would be 11 % (105), and items of two tiles are bound by this warp.
// What bounds it: of a step's 2000 cycles with two halves 1180 are exponentials (16 a cycle: 1024), 830 waits, loads and stores of
// both halves at the same time.  With the maximum first a prompt of 4096 took 164 us instead of 155, with a check of each step's sum before its
// probabilities are given away 157, with a quarter of the exponentials as polynomials on the other units 165.
template <int HDP, int NH>
__device__ __forceinline__ bool softmax_role(const TileParams& tp, Control& ctl) {
    constexpr float FAR = 1048576.f, MOST = 1.2676506e30f;     // 2^20, 2^100
    const Params& p = tp.a;
    const volatile Watch* watch = &ctl.watch;
    const int half = threadIdx.x >> 7, r = threadIdx.x & 127;
    const uint32_t tmem = ctl.tmem_slot + ((uint32_t)(r & 96) << 16), to = tmem + 256 + half * HDP;
    const int ti = r / tp.gs, hi = r - ti * tp.gs;           // row of the half, head of the tile
    uint32_t steps = 0;                                      // of this half so far
    Listed list;
    Item w;
    for (;; list.done(ctl)) {
        if (!list.get(ctl, tp, w)) return false;
        if (w.j1 == 0) return true;
        if (!active<NH>(tp, w, half)) continue;
        const int i = (w.qt * NH + half) * tp.rows_half + ti;
        const bool valid = ti < tp.rows_half && i < w.s.n, any = __any_sync(0xffffffffu, valid);
        paged::View view;
        view.lim = 0x7fffffff;
        view.base = 0;
        view.bits = 0;
        if (valid) view = paged::row_view(p.mask_block, p.row_mask, w.s, i);
        float m = valid ? -INFINITY : 0.f, l = 0.f, total = 0.f;          // total: of the step in front
        bool live = valid, fresh = true;                         // fresh: a row of the warp has no reference yet
        const int end = w.j1 * KEYS, all_see = __reduce_min_sync(0xffffffffu, view.lim);
        for (int key = w.j0 * KEYS; key < end; key += STEP, ++steps) {
            const uint32_t buf = steps & 1;
            if (!__all_sync(0xffffffffu, wait(&ctl.s_full[half][buf], steps >> 1 & 1, tp.wait_limit, watch))) return false;
            if (any) {
                tc_fence_after();
                const uint32_t ts = tmem + half * 2 * STEP + buf * STEP;
                if (!__all_sync(0xffffffffu, !live || total <= 512.f)) {
                    float alpha = 1.f;
                    if (!(total <= MOST)) {
                        l = __int_as_float(0x7fffffff);
                        live = false;
                    } else if (total > 512.f) {
                        alpha = raise_reference(m, l, total);
                    }
                    if (!__all_sync(0xffffffffu, wait(&ctl.o_full[half][buf ^ 1], (steps - 1) >> 1 & 1, tp.wait_limit, watch))) return false;      // the product before this one's
                    tc_fence_after();
#pragma unroll 1
                    for (int d = 0; d < HDP; d += 16) {
                        float o[16];
                        tmem_ld16(to + d, o);
                        uint32_t u[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) u[e] = __float_as_uint(o[e] * alpha);
                        tmem_st16(to + d, u);
                    }
                }
                uint32_t v[2][32], pk[16], rest[16];
                tmem_ld32_issue(ts, v[0]);
                tmem_ld32_issue(ts + 32, v[1]);
                tmem_ld_wait();
                if (key + STEP > all_see) {
                    mask32(v[0], view, key);
                    mask32(v[1], view, key + 32);
                }
                if (fresh) {
                    if (m == -INFINITY) m = fmaxf(first_reference(v[0]) * p.scale_log2, m);
                    if (m == -INFINITY) m = fmaxf(first_reference(v[1]) * p.scale_log2, m);
                    fresh = __any_sync(0xffffffffu, m == -INFINITY);
                }
                const float minus_m = m == -INFINITY ? 0.f : -m;
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                probabilities<NH == 1>(v[0], p.scale_log2, minus_m, pk, rest, sum);
                tmem_st16(ts, pk);
                if (NH == 1) tmem_st16(ts + 32, rest);
                probabilities<false>(v[1], p.scale_log2, minus_m, pk, rest, sum);
                tmem_st16(ts + 16, pk);
                sum[0] = add2(sum[0], sum[1]);
                total = sum[0].x + sum[0].y;
                l += total;
                tmem_st_wait();
                tc_fence_before();
            }
            arrive(&ctl.p_full[half][buf]);
        }
        // ---- the item's end: divide, or leave a part ----
        if (!__all_sync(0xffffffffu, wait(&ctl.o_full[half][1], (steps - 1) >> 1 & 1, tp.wait_limit, watch))) return false;
        if (any) {
            tc_fence_after();
            const long long row = w.s.row0 + i;
            const int h = w.head0 + hi;
            const bool nan = !w.s.ok || *(volatile int*)&ctl.bad[list.index % (2 * ITEMS)] == list.index + 1, whole = w.whole();
            const float undefined = __int_as_float(0x7fffffff);
            // what the step in front of a next one would do with the last one's sum; a part's reference goes up, too, so that join_kernel weighs parts
            // by references that are not far below what they hold
            float raised = 1.f;
            if (nan || !(total <= MOST) || (fabsf(m) > FAR && m != -INFINITY)) {
                l = undefined;
            } else if (!whole && total > 512.f) {
                raised = raise_reference(m, l, total);
            }
            const float factor = nan ? undefined : whole ? (l == 0.f ? 0.f : 1.f / l) : raised;
            const size_t slot = ((size_t)(2 * blockIdx.x + (w.j0 == 0)) * NH + half) * QTILE + r;
            char* dst = whole ? (char*)(p.out + row * p.out_ld + (long long)h * p.head_dim) : (char*)(tp.part_o + slot * HDP);
            float check = fabsf(l), check1 = 0.f;                                  // infinite or NaN where something is
#pragma unroll 1
            for (int c = 0; c < HDP; c += 32) {
                uint32_t u[32];
                __syncwarp();
                tmem_ld32_issue(to + c, u);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    check = max3_nan(check, fabsf(__uint_as_float(u[e])), fabsf(__uint_as_float(u[e + 1])));
                    check1 = max3_nan(check1, fabsf(__uint_as_float(u[e + 2])), fabsf(__uint_as_float(u[e + 3])));
                }
                if (whole) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) u[e] = pack2(__uint_as_float(u[2 * e]) * factor, __uint_as_float(u[2 * e + 1]) * factor);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) u[e] = __float_as_uint(__uint_as_float(u[e]) * factor);
                }
                if (valid) {
                    if (whole) {
                        if (c < p.head_dim) store32(dst, u, tp.out_32, c + 8 < p.head_dim);
                        if (c + 16 < p.head_dim) store32(dst + 32, u + 8, tp.out_32, c + 24 < p.head_dim);
                        dst += 64;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) store32(dst + 32 * e, u + 8 * e, true, true);
                        dst += 128;
                    }
                }
            }
            __syncwarp();
            tc_fence_before();                                                     // (the next product waits for the next probabilities)
            if (valid) {
                if (!whole) tp.part_ml[slot] = make_float2(m, l);
                else if (p.lse) p.lse[row * p.heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            }
            const bool bad = valid && !nan && !(max3_nan(check, check1, check1) < INFINITY);
            if (__any_sync(0xffffffffu, bad)) {
                __syncwarp();
                repair_rows(tp, w, i, h, bad, slot, HDP, &ctl.watch.progress);
            }
        }
    }
}

// Q warp: the query vectors of each item's halves, a box of rows x heads x 64 elements at a time.  Rows behind the sequence's are some other
// rows or zeros, and the tile's last vectors (128 is no multiple of the group) whatever was there: nobody looks at their results.
template <int HDP, int NH>
__device__ __forceinline__ bool query_role(const TileParams& tp, Control& ctl, uint8_t* q_tiles, const CUtensorMap* map_q) {
    uint32_t items[2] = {0, 0};                              // of a half so far
    Listed list;
    Item w;
    for (;; list.done(ctl)) {
        if (!list.get(ctl, tp, w)) return false;
        if (w.j1 == 0) return true;
#pragma unroll
        for (int half = 0; half < NH; ++half) {
            if (!active<NH>(tp, w, half)) continue;
            if (!__all_sync(0xffffffffu, wait(&ctl.q_empty[half], (items[half] & 1) ^ 1, tp.wait_limit, &ctl.watch))) return false;
            ++items[half];
            if (elect()) {
                mbar_expect_tx(&ctl.q_full[half], (uint32_t)(tp.gs * tp.rows_half) * HDP * 2);
#pragma unroll
                for (int c = 0; c < HDP / 64; ++c)
                    tma_load_3d(q_tiles + (half * (HDP / 64) + c) * (QTILE * 128), map_q, c * 64, w.head0, w.s.row0 + (w.qt * NH + half) * tp.rows_half, &ctl.q_full[half]);
            }
            __syncwarp();
        }
    }
}

// MMA warps, one per half: a warp that has to look after both needs more time for its instructions and waits (2300 cycles per half and unit)
// than the tensor core for the MMAs.  The scores of the next step go in front of O += P V.  The tensor core takes MMAs of a thread in the
// order of their issue: the scores of step u + 1 come behind the product of step u - 1, whose probabilities they overwrite.
template <int HDP, int NH>
__device__ __forceinline__ bool mma_role(const TileParams& tp, Control& ctl, uint8_t* q_tiles, uint8_t* ring, int half) {
    const Params& p = tp.a;
    constexpr int SB = KEYS * HDP * 2;
    const volatile Watch* watch = &ctl.watch;
    const int lane = threadIdx.x & 31;
    const uint32_t t_s = ctl.tmem_slot + half * 2 * STEP, t_o = ctl.tmem_slot + 256 + half * HDP;
    // D fp32, A and B bf16, M = 128; A K-major, B K-major (keys) or MN-major (values)
    constexpr uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(STEP >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    constexpr uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(HDP >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
    const uint64_t q_desc = desc_k(smem_u32(q_tiles) + half * (QTILE * HDP * 2)), k_desc = desc_k(smem_u32(ring)), v_desc = desc_mn(smem_u32(ring), KEYS * 128);
    Ring rk, rv;                                             // K of the next scores, V of the next product
    rv.next(tp.stages);
    uint32_t steps = 0, items = 0;                           // products, and items whose scores have begun, of this half
    auto all = [&](bool ok) { return __all_sync(0xffffffffu, ok); };
    auto given = [&](uint64_t* bar, uint32_t parity) { return all(wait(bar, parity, tp.wait_limit, watch)); };
    auto step = [&](Ring& r) {
        r.next(tp.stages);
        r.next(tp.stages);
    };
    // S = Q K^T for the first or second 64 keys of the K tile; behind the second the tile is free, and Q if the item has no more
    auto scores = [&](int part, bool last) {
        tc_fence_after();
        if (elect()) {
#pragma unroll
            for (int k = 0; k < HDP / 16; ++k) {
                const int at = (k >> 2) * (QTILE * 128 >> 4) + 2 * (k & 3);
                umma_bf16(t_s + part * STEP, q_desc + at, k_desc + (rk.s * (SB >> 4) + part * (STEP * 128 >> 4) + at), idesc_s, k ? 1u : 0u);
            }
            umma_commit(&ctl.s_full[half][part]);
            if (part) umma_commit(&ctl.empty[rk.s]);
            if (last) umma_commit(&ctl.q_empty[half]);
        }
        __syncwarp();
        if (part) step(rk);
    };
    auto is_active = [&](const Item& x) { return active<NH>(tp, x, half); };

    Listed list;
    Item w, next;
    if (!list.get(ctl, tp, w)) return false;
    bool issued = false;                                     // the first scores of the item are on their way
    while (w.j1) {
        list.done(ctl);
        if (!list.get(ctl, tp, next)) return false;
        if (!is_active(w)) {                                 // gives the stages back
            for (int j = w.j0; j < w.j1; ++j) {
                for (Ring* r : {&rk, &rv}) {
                    if (!given(&ctl.full[r->s], r->parity)) return false;
                    if (lane == 0) arrive(&ctl.empty[r->s]);
                    step(*r);
                }
            }
            w = next;
            continue;
        }
        if (!issued) {
            if (!given(&ctl.q_full[half], items & 1) || !given(&ctl.full[rk.s], rk.parity)) return false;
            scores(0, false);
            ++items;
        }
        issued = false;
        const int n_steps = 2 * (w.j1 - w.j0);
#pragma unroll 1
        for (int u = 0; u < n_steps; ++u, ++steps) {
            const int part = u & 1;
            // the scores of the next step: of this item, or of the next one if all that they need is there
            if (u + 1 < n_steps) {
                if (part && !given(&ctl.full[rk.s], rk.parity)) return false;
                scores(part ^ 1, u + 2 == n_steps);
            } else if (next.j1 && is_active(next) && all(peek(&ctl.q_full[half], items & 1) && peek(&ctl.full[rk.s], rk.parity))) {
                scores(0, false);
                issued = true;
                ++items;
            }
            if (!part) {
                if (!given(&ctl.full[rv.s], rv.parity)) return false;
                const int n = max(w.s.kv - (w.j0 + (u >> 1)) * KEYS, 0);          // tokens of the tile
                if (n < KEYS) {
                    // values behind the last token are whatever stands in the page or in the ring: a NaN times a probability of zero is a
                    // NaN (both MMA warps write the same zeros)
                    for (int e = lane; e < (KEYS - n) * (HDP / 64) * 8; e += 32) {
                        const int r = n + (e >> 3) / (HDP / 64), c = e & 7, hh = (e >> 3) % (HDP / 64);
                        *reinterpret_cast<uint4*>(ring + rv.s * SB + hh * (KEYS * 128) + r * 128 + c * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_async_shared();
                    __syncwarp();
                }
            }
            if (!given(&ctl.p_full[half][part], steps >> 1 & 1)) return false;
            tc_fence_after();
            if (elect()) {                                   // 64 keys of O += P V
#pragma unroll
                for (int k = 0; k < STEP / 16; ++k) {
                    const uint64_t d = v_desc + (rv.s * (SB >> 4) + part * (STEP * 128 >> 4) + k * 128);
                    umma_bf16_ta(t_o, t_s + part * STEP + k * 8, d, idesc_o, u || k ? 1u : 0u);
                    if (NH == 1 && k < 2) umma_bf16_ta(t_o, t_s + part * STEP + 32 + k * 8, d, idesc_o, 1u);
                }
                umma_commit(&ctl.o_full[half][part]);
                if (part) umma_commit(&ctl.empty[rv.s]);
            }
            __syncwarp();
            if (part) step(rv);
        }
        w = next;
    }
    return true;
}

// Copy warp: lists the items for the others, and loads their K and V tiles of 128 keys, page by page (a lane per page), in the order in which the
// MMA warp takes them.
template <int HDP, int NH>
__device__ __forceinline__ bool copy_role(const TileParams& tp, Control& ctl, uint8_t* ring, const CUtensorMap* map_k, const CUtensorMap* map_v) {
    const Params& p = tp.a;
    constexpr int SB = KEYS * HDP * 2;
    const int lane = threadIdx.x & 31, box = min(KEYS, p.c.page_mask + 1), pages = KEYS / box;
    const uint32_t ra = smem_u32(ring);
    Ring r;
    r.parity = 1;                                            // a fresh barrier passes a wait for the phase before its first
    Items t;
    plan<NH>(tp, ctl.setup, t);
    // The next item, or the end, is listed before this one's last tiles are loaded: the MMA warps want to know what comes behind an item that
    // they give room for.
    Item w, next;
    auto publish = [&](int index, Item& x) {
        if (!next_item<NH>(tp, t, x)) x.j1 = 0;
        if (!__all_sync(0xffffffffu, wait(&ctl.item_empty[index % ITEMS], (index / ITEMS & 1) ^ 1, tp.wait_limit, &ctl.watch))) return false;
        if (lane == 0) {
            ctl.items[index % ITEMS] = x;
            arrive(&ctl.item_full[index % ITEMS]);
            if (x.j1) note_split(tp, ctl.setup, x);
        }
        __syncwarp();
        return true;
    };
    if (!publish(0, w)) return false;
    for (int index = 0; w.j1; ++index, w = next) {
        for (int j = w.j0; j < w.j1; ++j) {
            if (j == w.j0 + 1 && !publish(index + 1, next)) return false;          // (the first tile is on its way)
            const int key = j * KEYS + lane * box;
            bool some = lane < pages && key < w.s.kv;
            const int page = some ? paged::page_of(p.b, w.seq, key) : -1;
            if (some && page < 0) {
                *(volatile int*)&ctl.bad[index % (2 * ITEMS)] = index + 1;
                some = false;
            }
            const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, some)) * box * HDP * 2;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                if (!__all_sync(0xffffffffu, wait(&ctl.empty[r.s], r.parity, tp.wait_limit, &ctl.watch))) return false;
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
        if (w.j1 - w.j0 == 1 && !publish(index + 1, next)) return false;
    }
    return true;
}

template <int HDP, int NH>
__global__ void __launch_bounds__(threads(NH), 1)
tile_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
            const __grid_constant__ TileParams tp) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* base = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* ring = base + NH * QTILE * HDP * 2;
    Control& ctl = *(Control*)(base + tp.control_at);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp == 0) {
        for (int i = lane; i < BARRIERS; i += 32) {
            const int k = i - 2 * MAX_STAGES;                // behind full (1) and empty (MMA warps); then the members of Control in their order
            const int count = k < 0 ? (i < MAX_STAGES ? 1 : NH) : k < ITEMS ? 1 : k < 2 * ITEMS ? 5 * NH + 1 : k < 2 * ITEMS + 8 ? 1 : k < 2 * ITEMS + 12 ? 128 : 1;
            mbar_init(&ctl.full[0] + i, count);
        }
        if (lane < 2 * ITEMS) ctl.bad[lane] = 0;
        if (lane == 0) ctl.watch = Watch{0, 0};
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (warp == 4 * NH + 2) {
        tmem_alloc(&ctl.tmem_slot, 512);
        tmem_relinquish();
    } else if (warp == 4 * NH && lane < 3) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &map_q : lane == 1 ? &map_k : &map_v) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch();
    // all warps: nothing in front reads or writes what this kernel does, and the bounded waits begin behind it
    pdl_wait();
    bool ok = true;
    if (warp < 4 * NH) ok = softmax_role<HDP, NH>(tp, ctl);
    else if (warp == 4 * NH) ok = copy_role<HDP, NH>(tp, ctl, ring, &map_k, &map_v);
    else if (warp == 4 * NH + 1) ok = query_role<HDP, NH>(tp, ctl, base, &map_q);
    else if (warp - 4 * NH - 2 < NH) ok = mma_role<HDP, NH>(tp, ctl, base, ring, warp - 4 * NH - 2);
    if (!ok) *(volatile int*)&ctl.watch.abort = 1;
    __syncwarp();
    __syncthreads();
    const bool failed = *(volatile int*)&ctl.watch.abort;
    if (failed) settle();
    tc_fence_before();
    __syncthreads();
    if (warp == 4 * NH + 2) tmem_dealloc(ctl.tmem_slot, 512);
    if (failed) {
        if (threadIdx.x == 0) atomicAdd(tp.timeouts, 1);
        all_nan<NH>(tp, ctl.setup, HDP);
    }
}

// Sum of the parts of an item that the cuts went through, in the order of the keys: a block takes JOIN_WARPS * join_vectors vectors of the item that
// CTA blockIdx.x began, a warp join_vectors at a time.  The lanes take the parts' references and sums, 32 at a time, then four elements each
// (HDP 64: two) of all parts.  Blocks of 8 warps find room on a SM beside the tiles' CTA, where they wait for its end (131072 tokens 3.9 us
// less than with blocks of 32, one token 1.3 less).  Items of two halves have parts of 256 vectors, of which a warp has two in flight together (ragged
// chunks 64 us, one by one 67); with one half that costs more than it gives (131072 tokens 3.4 us more).
constexpr int JOIN_WARPS = 8;
__host__ __device__ constexpr int join_vectors(int nh) { return nh; }
template <int HDP, int NH>
__global__ void __launch_bounds__(32 * JOIN_WARPS) join_kernel(const __grid_constant__ TileParams tp) {
    constexpr int E = HDP / 32, V = join_vectors(NH);
    pdl_wait();
    pdl_launch();
    const Params& p = tp.a;
    const int c = blockIdx.x;
    const int4 d = tp.split[2 * c];
    if (d.x < 0) return;
    const int rows = tp.split[2 * c + 1].x, r0 = (blockIdx.y * JOIN_WARPS + (threadIdx.x >> 5)) * V, lane = threadIdx.x & 31;
    int i[V], h[V];
    bool some[V], any = false;
    float m[V], l[V], o[V][E];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int r = r0 + v, ti = (r & 127) / tp.gs;
        i[v] = (d.y * NH + (r >> 7)) * tp.rows_half + ti;
        h[v] = d.x + (r & 127) - ti * tp.gs;
        some[v] = ti < tp.rows_half && i[v] < rows;
        any |= some[v];
        m[v] = -INFINITY;
        l[v] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[v][e] = 0.f;
    }
    if (!any) return;
    for (int first = c; first <= d.z; first += 32) {
        const int part = first + lane, n = min(32, d.z + 1 - first);
        float g[V];
        float2 ml[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            ml[v] = make_float2(-INFINITY, 0.f);
            if (some[v] && lane < n) ml[v] = tp.part_ml[(size_t)(2 * part + (part == c)) * (128 * NH) + r0 + v];
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float top = fmaxf(m[v], warp_max(ml[v].x)), ref = top == -INFINITY ? 0.f : top, f = exp2_fast(m[v] - ref);
            g[v] = exp2_fast(ml[v].x - ref);
            l[v] = l[v] * f + warp_sum(ml[v].y * g[v]);
            m[v] = top;
#pragma unroll
            for (int e = 0; e < E; ++e) o[v][e] *= f;
        }
#pragma unroll 8 / V
        for (int k = 0; k < n; ++k) {
            const float* src = tp.part_o + ((size_t)(2 * (first + k) + (first + k == c)) * (128 * NH) + r0) * HDP + lane * E;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float weight = __shfl_sync(0xffffffffu, g[v], k);
                float x[E];
                if constexpr (E == 4) {
                    const float4 u = some[v] ? *reinterpret_cast<const float4*>(src + v * HDP) : make_float4(0.f, 0.f, 0.f, 0.f);
                    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w;
                } else {
                    const float2 u = some[v] ? *reinterpret_cast<const float2*>(src + v * HDP) : make_float2(0.f, 0.f);
                    x[0] = u.x, x[1] = u.y;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) o[v][e] = fmaf(x[e], weight, o[v][e]);
            }
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (!some[v]) continue;
        const long long row = d.w + i[v];
        const float inv = l[v] == 0.f ? 0.f : 1.f / l[v];
        bf16* out = p.out + row * p.out_ld + (long long)h[v] * p.head_dim + lane * E;
        if (lane * E < p.head_dim) {
            if constexpr (E == 4) *reinterpret_cast<uint2*>(out) = make_uint2(pack2(o[v][0] * inv, o[v][1] * inv), pack2(o[v][2] * inv, o[v][3] * inv));
            else *reinterpret_cast<uint32_t*>(out) = pack2(o[v][0] * inv, o[v][1] * inv);
        }
        if (p.lse && lane == 0) p.lse[row * p.heads + h[v]] = l[v] == 0.f ? -INFINITY : (m[v] + log2f(l[v])) * 0.6931471805599453f;
    }
}

}  // namespace patt
}  // namespace s2d2
