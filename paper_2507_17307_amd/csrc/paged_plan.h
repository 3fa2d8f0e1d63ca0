// Arithmetic of the calls on caches in pages: which spans are in range, and which positions a block of an attention call reads.
// Plain C++ without HIP types, so that it can also be compiled and checked on a CPU.
#pragma once

#include "attn_plan.h"

namespace rs {

constexpr int PAGED_MAX_SEQS = 1024;

struct PagedSpans {
    const int *slot, *off, *pos0, *table;      // off null: one row a sequence
    const int *info;                           // not null: in the place of those three, per sequence {first row, end row, slot, first row's position}, first row < 0: invalid
    int n_seqs, n_rows, n_slots, n_pages, max_pages, page_shift, n_kv;
    unsigned int *flags;                       // may be null
};

// Rows first .. first + m - 1 at positions p0, p0 + 1, ... of a slot.
struct Span { int first, m, slot, p0; };

// Sequence b of the call; false: something of it is out of range (its rows are skipped).
RS_HD bool paged_span(const PagedSpans &a, int b, Span &s) {
    int end;
    s.m = 0;
    if (a.info) { s.first = a.info[4 * b]; end = a.info[4 * b + 1]; s.slot = a.info[4 * b + 2]; s.p0 = a.info[4 * b + 3]; }
    else {
        s.first = a.off ? a.off[b] : b;
        end = a.off ? a.off[b + 1] : b + 1;
        s.slot = a.slot[b]; s.p0 = a.pos0[b];
    }
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

// ------------------------------------------------------------------------------------------------
// Split of an attention call.  An item is a block of `rows` rows of one span (what the columns of a workgroup's tiles hold, times the query
// heads of a KV head) and one KV head; its work are the tiles of positions that some row of the block sees.  Items are counted
// sequence by sequence, KV head by KV head, block by block; the tiles of all items in that order are dealt to the workgroups in equal
// runs, whatever the spans and contexts are.  A run may start and end inside an item: what is cut is joined by a second kernel.
// ------------------------------------------------------------------------------------------------
RS_HD int paged_blocks(const Span &s, int rows) { return (s.m + rows - 1) / rows; }

// Positions lo .. hi - 1 that rows r0 .. r1 - 1 of the span see between them.
RS_HD void paged_seen(const Span &s, int r0, int r1, int window, int &lo, int &hi) {
    const int first = s.p0 + r0;
    lo = window > 0 && first >= window ? first - window + 1 : 0;
    hi = s.p0 + r1;
}

// Tiles t0 .. t1 - 1 of block j.
RS_HD void paged_tiles(const Span &s, int rows, int window, int tile_shift, int j, int &t0, int &t1) {
    int lo, hi;
    const int r0 = j * rows, r1 = r0 + rows < s.m ? r0 + rows : s.m;
    paged_seen(s, r0, r1, window, lo, hi);
    t0 = lo >> tile_shift; t1 = ((hi - 1) >> tile_shift) + 1;
}

// First tile of run w of W over T tiles: T w / W, rounded down (no product beyond T).
RS_HD long long paged_run(long long T, int W, int w) {
    if (T == W) return w;
    if (T >> 31 == 0) { const unsigned t = (unsigned)T, n = (unsigned)W, k = (unsigned)w, q = t / n; return q * k + (t - q * n) * k / n; }      // (W is at most 2^11)
    return T / W * w + T % W * w / W;
}

// The run that tile t < T is in: the largest w with T w / W < t + 1.
RS_HD int paged_run_of(long long T, int W, long long t) {
    if (T < 1 << 20) return (int)((((unsigned)t + 1) * (unsigned)W - 1) / (unsigned)T);             // (below 2^31)
    if (T >> 50 == 0) return (int)(((t + 1) * W - 1) / T);
    int lo = 0, hi = W - 1;
    while (lo < hi) { const int mid = (lo + hi) / 2; if (paged_run(T, W, mid + 1) > t) hi = mid; else lo = mid + 1; }
    return lo;
}

}  // namespace rs
