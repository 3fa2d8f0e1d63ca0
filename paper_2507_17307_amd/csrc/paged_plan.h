// Arithmetic of the calls on caches in pages: which spans are in range, and which positions a block of an attention call reads.
// Plain C++ without HIP types, so that it can also be compiled and checked on a CPU.
#pragma once

#include "attn_plan.h"

namespace rs {

constexpr int PAGED_MAX_SEQS = 1024;

struct PagedSpans {
    const int *slot, *off, *pos0, *table;      // off null: one row a sequence
    int n_seqs, n_rows, n_slots, n_pages, max_pages, page_shift, n_kv;
    unsigned int *flags;                       // may be null
};

// Rows first .. first + m - 1 at positions p0, p0 + 1, ... of a slot.
struct Span { int first, m, slot, p0; };

// Sequence b of the call; false: something of it is out of range (its rows are skipped).
RS_HD bool paged_span(const PagedSpans &a, int b, Span &s) {
    s.first = a.off ? a.off[b] : b;
    const int end = a.off ? a.off[b + 1] : b + 1;
    s.slot = a.slot[b]; s.p0 = a.pos0[b]; s.m = 0;
    if (s.first < 0 || end < s.first || end > a.n_rows) return false;
    s.m = end - s.first;
    if (s.slot < 0 || s.slot >= a.n_slots || s.p0 < 0) return false;
    return (long long)s.p0 + s.m <= (long long)a.max_pages << a.page_shift;
}

// Positions of an append workgroup: an aligned block of one sequence, so that a channel of V is written in whole pieces of a page's row.
constexpr int APPEND_BLOCK = 64;
RS_HD int append_blocks_of(const Span &s) { return s.m > 0 ? (s.p0 % APPEND_BLOCK + s.m + APPEND_BLOCK - 1) / APPEND_BLOCK : 0; }
// ... of a call, at most: a span of m rows touches at most m blocks, and at most m / APPEND_BLOCK + 2
RS_HD int append_blocks_most(int n_seqs, int n_rows) {
    const int few = n_rows / APPEND_BLOCK + 2 * n_seqs;
    return few < n_rows ? few : n_rows;
}

}  // namespace rs
