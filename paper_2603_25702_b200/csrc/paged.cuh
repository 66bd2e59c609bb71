// What the operators on a paged cache share: the batch's rows, the cache, and which keys a row sees.
#pragma once
#include "common.cuh"
#include "ops_host.h"

namespace s2d2 {
namespace paged {

struct Batch {
    const int* row0;
    const int* kv_len;
    const int* pages;
    int n_rows, n_seqs, max_pages, page_shift, n_pages;
    long long max_kv;                // max_pages * page_tokens
};
struct Cache {
    bf16* k;
    bf16* v;
    long long page_stride, head_stride, token_stride;
    int page_mask;                   // page_tokens - 1
};
// A sequence as the device finds it: n = 0 where row0 is not usable; ok = false where the length is not.
struct Seq {
    int row0, n, kv;
    bool ok;
};
__device__ __forceinline__ Seq read_seq(const Batch& b, int s) {
    Seq q;
    const int first = b.row0[s], next = b.row0[s + 1];
    q.kv = b.kv_len[s];
    q.row0 = first;
    q.n = first >= 0 && next >= first && next <= b.n_rows ? next - first : 0;
    q.ok = q.kv >= 0 && q.kv <= b.max_kv;
    return q;
}
// The sequence of a row, or -1 (row0 is searched as if it did not decrease; what is found is checked).
__device__ __forceinline__ int find_seq(const Batch& b, int row) {
    int lo = 0, hi = b.n_seqs;       // first s with row0[s + 1] > row
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (b.row0[mid + 1] > row) hi = mid;
        else lo = mid + 1;
    }
    if (lo >= b.n_seqs) return -1;
    return b.row0[lo] >= 0 && b.row0[lo] <= row && b.row0[lo + 1] <= b.n_rows ? lo : -1;
}
// Page of cache index j (0 <= j < max_kv), or -1.
__device__ __forceinline__ int page_of(const Batch& b, int s, int j) {
    const int page = b.pages[(long long)s * b.max_pages + (j >> b.page_shift)];
    return page >= 0 && page < b.n_pages ? page : -1;
}

// Keys that a row sees: j < lim, and base + b for the bits b that are set.
struct View {
    int lim, base;
    unsigned long long bits;
    __device__ __forceinline__ bool sees(int j) const {
        const unsigned d = (unsigned)(j - base);
        return j < lim || (d < 64 && (bits >> d & 1));
    }
};
// End of the keys that row i (or a row in front of it) may see.
__device__ __forceinline__ int key_end(int mask_block, bool masked, int n, int kv, int i) {
    if (masked || mask_block == 0) return kv;
    const int p = kv - n + i;
    if (p < 0) return 0;
    if (mask_block == 1) return p + 1;
    const long long end = ((long long)(p / mask_block) + 1) * mask_block;
    return end < kv ? (int)end : kv;
}
__device__ __forceinline__ View row_view(int mask_block, const unsigned long long* row_mask, const Seq& s, int i) {
    View v;
    v.base = s.kv - s.n;
    if (row_mask) {
        v.lim = max(0, v.base);
        v.bits = row_mask[s.row0 + i];
        if (s.n < 64) v.bits &= (1ull << s.n) - 1;
    } else {
        v.lim = key_end(mask_block, false, s.n, s.kv, i);
        v.bits = 0;
    }
    return v;
}

}  // namespace paged

namespace ops {
// Checks of the structs and their device forms (rope.cu); `op` names the call.
int check_rows(const char* op, const s2d2_rows* r);                              // fields only
int check_kv(const char* op, const s2d2_paged_kv* c);
int device_rows(const Device* d, const s2d2_rows* r, const s2d2_paged_kv* c, paged::Batch* out);     // and pointers
int device_kv(const Device* d, const s2d2_paged_kv* c, paged::Cache* out);
}  // namespace ops
}  // namespace s2d2
