// Argument checks and launches of the calls on caches in pages, for paged_api.h and for the models whose cache is in pages.  Included by rstitch.hip.
#pragma once

#include "paged_attention.h"
#include "paged_rope.h"

namespace {

const char *check_paged(const rs_paged_kv *c) {
    if (!c) return "null cache";
    if (!c->k || !c->v || !c->page_table) return "null cache pointer";
    if (((uintptr_t)c->k | (uintptr_t)c->v) % 16) return "K and V pages must be 16-byte aligned";
    if ((uintptr_t)c->page_table % 4) return "page_table must be 4-byte aligned";
    if (c->n_pages < 1 || c->n_slots < 1 || c->max_pages < 1 || c->n_kv_heads < 1) return "cache with a count below 1";
    if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return "page_size must be a power of two in 16..1024";
    if ((long long)c->page_size * c->max_pages > (1LL << 30)) return "page_size * max_pages must not exceed 2^30";
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 32, 64 or 128";
    if (c->n_kv_heads > 1024) return "more than 1024 KV heads";
    return nullptr;
}

const char *check_rope(const rs_rope *r, int head_dim) {
    if (r->rot_dim < 8 || r->rot_dim % 8 || r->rot_dim > head_dim) return "rot_dim must be a multiple of 8 in 8..head_dim";
    if (r->interleaved != 0 && r->interleaved != 1) return "interleaved must be 0 or 1";
    if (!r->d_inv_freq || (uintptr_t)r->d_inv_freq % 8) return "null or misaligned d_inv_freq";
    if (!std::isfinite(r->amplitude)) return "amplitude must be finite";
    return nullptr;
}

// Rows of `heads` heads, `stride` elements apart.
const char *check_rows(const void *p, int64_t stride, int dtype, long long heads, int head_dim) {
    const int size = dtype == RS_BF16 ? 2 : 4;
    if (!p) return "null row pointer";
    if ((uintptr_t)p % 16 || stride % (16 / size)) return "rows must be 16-byte aligned";
    if (stride < heads * head_dim) return "a row stride is smaller than a row";
    if (stride > ((int64_t)1 << 40)) return "a row stride is too large";
    return nullptr;
}

rs_status check_spans(int32_t n_seqs, int32_t n_rows, const int32_t *slot, const int32_t *off, const int32_t *pos0, const uint32_t *flags, int dtype) {
    if (n_seqs < 1 || n_rows < 1) return fail(RS_EINVAL, "n_seqs and n_rows must be at least 1");
    if (n_seqs > PAGED_MAX_SEQS) return fail(RS_ECAPACITY, "n_seqs %d exceeds %d", n_seqs, PAGED_MAX_SEQS);
    if (n_rows > (1 << 22)) return fail(RS_ECAPACITY, "n_rows %d exceeds 2^22", n_rows);
    if (!slot || !pos0) return fail(RS_EINVAL, "null argument");
    if (((uintptr_t)slot | (uintptr_t)off | (uintptr_t)pos0 | (uintptr_t)flags) % 4) return fail(RS_EINVAL, "slots, offsets, positions and flags must be 4-byte aligned");
    if (!off && n_rows < n_seqs) return fail(RS_EINVAL, "%d sequences of one row do not fit %d rows", n_seqs, n_rows);
    if (dtype != RS_F32 && dtype != RS_BF16) return fail(RS_EINVAL, "dtype must be RS_F32 or RS_BF16");
    return RS_OK;
}

PagedSpans paged_spans(const rs_paged_kv *c, int32_t n_seqs, int32_t n_rows, const int32_t *slot, const int32_t *off, const int32_t *pos0, uint32_t *flags) {
    PagedSpans s{};
    s.slot = slot; s.off = off; s.pos0 = pos0; s.table = c->page_table;
    s.n_seqs = n_seqs; s.n_rows = n_rows; s.n_slots = c->n_slots; s.n_pages = c->n_pages; s.max_pages = c->max_pages; s.n_kv = c->n_kv_heads;
    s.page_shift = __builtin_ctz((unsigned)c->page_size);
    s.flags = flags;
    return s;
}

// Which kernel takes a call, by the columns that a span brings on average (rows times query heads of a KV head) and by how many pairs of a sequence and a
// KV head there are to share the CUs.  us a call in a graph, 28 query heads on 4, contexts of 4000 positions, blocks of 16 / 32 / 128 columns, rows of each
// sequence 1, 3, 6, 8, 12 (7 to 84 columns):
//   fp32   1 sequence     15  18  24  26  30 /  18  23  28  31  38 /  20  21  23  24  27
//         16 sequences    41  52  80 100 140 /  47  54  68  82 103 /  55  57  58  60  69
//         64 sequences   113 156 299 348 490 / 118 135 199 263 360 / 179 181 182 183 193
//   bf16   1 sequence     14  17  22  25  30 /  15  20  25  28  35 /  19  19  20  21  24
//          8 sequences    32  37  50  57  80 /  34  40  45  50  59 /  25  27  29  29  35
//         64 sequences   112 158 295 355 501 / 113 124 177 252 328 / 103 111 116 118 131
// From 32 pairs on the rule takes the least of a line's three or is within 4 % of it: blocks grow with the columns, and with one plane of q the wide kernel, in which
// four waves fetch, is the fastest for single rows too.  Below, 16 columns are right for single rows and 128 for more than 64 columns, but between them the rule is too
// slow by up to 35 %: it takes 32 columns for 17 to 64, where 16 (up to 21 here) or 128 (from 42 on) are the least.
int paged_cols(int n_seqs, int n_rows, int group, int n_kv, int dtype) {
    const long long cols = ((long long)n_rows * group + n_seqs - 1) / n_seqs;
    const bool few = (long long)n_seqs * n_kv < 32;
    if (dtype == RS_BF16 && !few) return PAGED_COLS;
    return cols <= 16 ? 16 : cols <= (few ? 64 : 32) ? 32 : PAGED_COLS;
}

struct PagedShape { int cols, rows, runs; long long items; size_t of, odd, entries, ml, o, total; };
PagedShape paged_shape(const rs_paged_kv *cache, int n_seqs, int n_rows, int n_q_heads, int dtype) {
    const int n_kv = cache->n_kv_heads, head_dim = cache->head_dim, group = n_q_heads / n_kv;
    PagedShape p{};
    p.cols = paged_cols(n_seqs, n_rows, group, n_kv, dtype);
    p.rows = p.cols / group;
    p.runs = p.cols != PAGED_COLS ? PAGED_NARROW_RUNS : dtype == RS_F32 ? PAGED_WIDE_RUNS3 : PAGED_WIDE_RUNS;
    // at most so many items, and so many tiles in all: short page tables need fewer workgroups
    p.items = ((long long)n_rows / p.rows + n_seqs) * n_kv;
    const double tiles = (double)p.items * (((long long)cache->page_size * cache->max_pages >> PAGED_TILE) + 1);
    if (tiles < p.runs) p.runs = ((int)tiles + 7) / 8 * 8;                     // (whole rounds of the XCDs)
    p.of = align_up((size_t)p.runs * sizeof(int4));
    p.odd = p.of + align_up((size_t)p.runs * sizeof(int2));
    p.entries = p.odd + align_up((size_t)p.runs * 4);
    p.ml = p.entries + align_up(4);
    p.o = p.ml + align_up((size_t)2 * p.runs * 2 * p.cols * 4);
    p.total = p.o + align_up((size_t)2 * p.runs * p.cols * head_dim * 4);
    return p;
}

template <int HD, int PL, int COLS>
rs_status launch_paged(const PagedAttnArgs &a, const PagedShape &p, hipStream_t st) {
    if constexpr (COLS == PAGED_COLS) hipLaunchKernelGGL((k_paged_wide<HD, PL>), dim3(a.runs), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_paged_narrow<HD, PL, COLS / 16>), dim3(a.runs), dim3(64), 0, st, a);
    RS_LAUNCHED("paged_attention");
    // about 2048 workgroups, as far as a block has columns for them; by item at least one a run too, should it come to that
    constexpr int per = join_cols<HD, COLS>();
    const int entries = a.max_items > 0 ? a.max_items : a.runs, most = (a.rows * a.group + per - 1) / per, want = (2048 + entries - 1) / entries, shares = want < most ? want : most;
    const dim3 grid = a.max_items > 0 ? dim3(entries * shares > a.runs ? entries * shares : a.runs) : dim3(entries, shares);
    hipLaunchKernelGGL((k_paged_join<HD, PL, COLS>), grid, dim3(256), 0, st, a);
    RS_LAUNCHED("paged_join");
    return RS_OK;
}
template <int HD, int PL>
rs_status launch_paged_cols(const PagedAttnArgs &a, const PagedShape &p, hipStream_t st) {
    switch (p.cols) {
        case 16: return launch_paged<HD, PL, 16>(a, p, st);
        case 32: return launch_paged<HD, PL, 32>(a, p, st);
        default: return launch_paged<HD, PL, PAGED_COLS>(a, p, st);
    }
}
template <int PL>
rs_status launch_paged_hd(int head_dim, const PagedAttnArgs &a, const PagedShape &p, hipStream_t st) {
    switch (head_dim) {
        case 32: return launch_paged_cols<32, PL>(a, p, st);
        case 64: return launch_paged_cols<64, PL>(a, p, st);
        default: return launch_paged_cols<128, PL>(a, p, st);
    }
}

const char *check_paged_attention(const rs_paged_kv *c, int32_t n_q_heads) {
    if (const char *why = check_paged(c)) return why;
    if (n_q_heads < 1 || n_q_heads % c->n_kv_heads) return "n_kv_heads must divide n_q_heads";
    if (n_q_heads / c->n_kv_heads > 16) return "more than 16 query heads per KV head";
    return nullptr;
}

// Room behind a model's workspace: the places of the rows of a call, and the scratch of its attention, whatever the call's counts.
size_t paged_model_bytes(const rs_config &c, const rs_paged_kv &cache) {
    const int group = c.n_q_heads / c.n_kv_heads;
    size_t most = 0;
    for (int slots : {16, 32, PAGED_COLS}) {                     // a row of each kernel's calls; every one of its runs
        rs_paged_kv kv = cache;
        kv.max_pages = (1 << 30) / kv.page_size;
        const size_t n = paged_shape(&kv, 1, slots / group, c.n_q_heads, RS_F32).total;
        if (n > most) most = n;
    }
    return align_up((size_t)c.max_rows * 4) + most;
}

// The call itself: kernels on the spans of `spans`.  out_rsh < 0: rows, out_stride elements apart; else fp32 in operand order (PagedAttnArgs::rsh).
rs_status run_paged_attention(const rs_paged_kv *cache, const PagedSpans &spans, int dtype, int n_q_heads, const void *q, size_t q_stride, float scale, int window, void *out,
                              size_t out_stride, int out_rsh, float *lse, unsigned char *scratch, hipStream_t st) {
    PagedAttnArgs a{};
    const PagedShape p = paged_shape(cache, spans.n_seqs, spans.n_rows, n_q_heads, dtype);
    a.s = spans;
    a.kc = (const uint16_t *)cache->k; a.vc = (const uint16_t *)cache->v;
    a.q = q; a.out = out; a.lse = lse; a.q_stride = q_stride; a.out_stride = out_stride; a.rsh = out_rsh;
    a.n_q = n_q_heads; a.group = n_q_heads / cache->n_kv_heads; a.window = window; a.rows = p.rows;
    a.runs = p.runs; a.max_items = p.cols == PAGED_COLS && p.items <= p.runs ? (int)p.items : 0;
    a.c = scale * 1.44269504088896341f;
    a.cuts = (int4 *)scratch; a.cut_of = (int2 *)(scratch + p.of); a.odd = (unsigned int *)(scratch + p.odd); a.entries = (int *)(scratch + p.entries);
    a.part_ml = (float *)(scratch + p.ml); a.part_o = (float *)(scratch + p.o);
    return dtype == RS_F32 ? launch_paged_hd<3>(cache->head_dim, a, p, st) : launch_paged_hd<1>(cache->head_dim, a, p, st);
}

}  // namespace
