// Paged cache of head states: the index arithmetic that the kernels, the host checks and the tests share (host and device).
//
// A cache is two pools (keys, values) of pages of `page` slots (a power of two).  Row (page p, head h, slot i) of either pool is row
// p * page_rows + h * page + i of d values: bf16, or the codes of kv_quant.hip with one fp32 scale a row.  Sequence s of a batch owns
// tokens [q_starts[s], q_starts[s+1]) of the call, the last of its kv_lens[s] keys; key j of it lies in slot j mod page of page
// block_table[s][j / page].  Nothing that these arrays hold is trusted with an address: see span_of() and key_row().
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hbl {

struct PagedCache {
    uint8_t* k;
    uint8_t* v;
    float* k_scales;      // nullptr for bf16
    float* v_scales;
    int64_t page_rows;    // rows between two pages
    int n_pages, heads, page_shift;
};
struct PagedBatch {
    const int32_t* q_starts;      // [n_seqs + 1]
    const int32_t* kv_lens;       // [n_seqs]
    const int32_t* block_table;   // [n_seqs][table_stride]
    int64_t table_stride;
    int n_seqs;
    int capacity;                 // keys that a row of the table has pages for (at most 2^31 - 4096)
};

// Sequence s as the kernels take it: tokens [first, first + n) inside the call's T, `keys` inside its row of the table.  `total` is
// kv_lens[s] itself: token first + i has position total - n + i (negative: it has no place, nor does it see anything).
struct SeqSpan {
    int first, n, keys, total;
};
__host__ __device__ inline SeqSpan make_span(int start, int end, int total, int T, int capacity) {
    SeqSpan r;
    r.first = start < 0 ? 0 : (start < T ? start : T);
    const int last = end < r.first ? r.first : (end < T ? end : T);
    r.n = last - r.first;
    r.total = total < 0 ? 0 : total;
    r.keys = r.total < capacity ? r.total : capacity;
    return r;
}
__host__ __device__ inline SeqSpan span_of(const PagedBatch& b, int T, int s) {
    return make_span(b.q_starts[s], b.q_starts[s + 1], b.kv_lens[s], T, b.capacity);
}
// First row of a page for one head, or -1 if the table's entry names no page.
__host__ __device__ inline int64_t page_row(const PagedCache& c, int page, int head) {
    if ((uint32_t)page >= (uint32_t)c.n_pages) return -1;
    return (int64_t)page * c.page_rows + ((int64_t)head << c.page_shift);
}
// Row of key j (0 <= j < keys of the span) of sequence s, or -1.
__host__ __device__ inline int64_t key_row(const PagedCache& c, const PagedBatch& b, int s, int j, int head) {
    const int64_t row = page_row(c, b.block_table[s * b.table_stride + (j >> c.page_shift)], head);
    return row < 0 ? -1 : row + (j & ((1 << c.page_shift) - 1));
}

// Keys [lo, hi) that the token at position p sees: those not after it, or before the prefix's end, and less than `window` before it
// (0: however far).
struct KeyRange {
    int lo, hi;
};
__host__ __device__ inline KeyRange visible_keys(int p, int keys, int window, int prefix) {
    KeyRange r{0, 0};
    if (p < 0) return r;
    const int end = p + 1 > prefix ? p + 1 : prefix;
    r.hi = end < keys ? end : keys;
    r.lo = window > 0 && p - window + 1 > 0 ? p - window + 1 : 0;
    if (r.lo > r.hi) r.lo = r.hi;
    return r;
}

}  // namespace hbl
