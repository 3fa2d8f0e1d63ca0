// C entry points of beam search: the selection over beams and vocabulary, and the pool of pages that its sequences share (see include/rstitch.h).
// Included by rstitch.hip.
#pragma once

#include "beam_select.h"
#include "page_pool.h"

namespace {

const char *check_pool(const rs_page_pool *c) {
    if (!c) return "null pool";
    if (!c->page_table || !c->page_ref) return "null page_table or page_ref";
    if (((uintptr_t)c->page_table | (uintptr_t)c->page_ref) % 4) return "page_table and page_ref must be 4-byte aligned";
    if (c->n_pages < 1 || c->n_slots < 1 || c->max_pages < 1) return "pool with a count below 1";
    if (c->n_pages > (1 << 30)) return "more than 2^30 pages";
    if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return "page_size must be a power of two in 16..1024";
    if ((long long)c->page_size * c->max_pages > (1LL << 30)) return "page_size * max_pages must not exceed 2^30";
    if ((long long)c->n_slots * c->max_pages > 0x7fffffffLL) return "n_slots * max_pages must be below 2^31";
    return nullptr;
}

// Workgroups for a page's K or V of one layer in k_pool_copy.
long long page_pieces(const rs_page_pool *c) {
    const long long units = (long long)c->n_kv_heads * c->head_dim * c->page_size / 8;
    return (units + 256 * COPY_UNITS - 1) / (256 * COPY_UNITS);
}

// ... of a call that moves what is in the pages
const char *check_contents(const rs_page_pool *c) {
    if (const char *why = check_pool(c)) return why;
    if (!c->k || !c->v) return "a pool without pages";
    if (((uintptr_t)c->k | (uintptr_t)c->v) % 16) return "K and V pages must be 16-byte aligned";
    if (c->n_layers < 1 || c->n_layers > 65536 || c->n_kv_heads < 1 || c->n_kv_heads > 1024) return "n_layers must be in 1..65536, n_kv_heads in 1..1024";
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 32, 64 or 128";
    if (page_pieces(c) * 2 * c->n_layers > 0xffffff) return "a page of all layers is too large";      // (what a grid takes)
    return nullptr;
}

Pool make_pool(const rs_page_pool *c, uint32_t *flags) {
    Pool p{};
    p.k = (uint16_t *)c->k; p.v = (uint16_t *)c->v; p.table = c->page_table; p.ref = c->page_ref;
    p.n_layers = c->n_layers; p.n_pages = c->n_pages; p.page_shift = __builtin_ctz((unsigned)c->page_size);
    p.n_slots = c->n_slots; p.max_pages = c->max_pages; p.n_kv = c->n_kv_heads; p.head_dim = c->head_dim; p.flags = flags;
    return p;
}

struct PoolScratch { size_t moves, ints, total; };                 // the count is the first word
PoolScratch pool_scratch(const rs_page_pool *c, int n) {
    PoolScratch s{};
    s.moves = ALIGN;
    const size_t most = (size_t)(n > c->n_pages / 2 ? n : c->n_pages / 2);      // a fork's or a compaction's
    s.ints = s.moves + align_up(most * sizeof(PageMove));
    s.total = s.ints + align_up((size_t)c->n_pages * 8);
    return s;
}

rs_status check_pool_scratch(const rs_page_pool *c, int n, void *scratch, size_t bytes) {
    if (!scratch || (uintptr_t)scratch % ALIGN) return fail(RS_EINVAL, "scratch must be 256-byte aligned");
    const size_t need = pool_scratch(c, n).total;
    if (bytes < need) return fail(RS_EINVAL, "scratch of %zu bytes is smaller than the %zu needed", bytes, need);
    return RS_OK;
}

rs_status check_pool_rows(int32_t n, const void *a, const void *b, const void *c, const uint32_t *flags) {
    if (n < 1) return fail(RS_EINVAL, "a call needs at least one row");
    if (n > POOL_ROWS) return fail(RS_ECAPACITY, "%d rows exceed %d", n, POOL_ROWS);
    if (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c | (uintptr_t)flags) % 4) return fail(RS_EINVAL, "row arguments and flags must be 4-byte aligned");
    return RS_OK;
}

// Workgroups of k_pool_copy, about: those without a move of their own cost their start (4096 / 16384, us of a call: 300 of the smallest pages, compacted, 18 / 23; 24
// pages of the 14B shape 126 / 121; 91 of the 7B shape, compacted, 149 / 145).
constexpr int COPY_WGS = 4096;
rs_status launch_copy(const rs_page_pool *to, CopyArgs a, int moves_most, hipStream_t st) {
    a.pieces = (int)page_pieces(to);
    const long long x = a.pieces * 2LL * to->n_layers, y = (COPY_WGS + x - 1) / x;
    hipLaunchKernelGGL(k_pool_copy, dim3((unsigned)x, (unsigned)(y < moves_most ? y : moves_most < 1 ? 1 : moves_most)), dim3(256), 0, st, a);
    RS_LAUNCHED("pool_copy");
    return RS_OK;
}

constexpr int BEAM_SLOTS = 1024;                                   // workgroups of k_beam_scan that run at once: four a CU, by its registers
struct BeamScratch { BeamPlan plan; size_t sums, scores, total; };
BeamScratch beam_scratch(int n_groups, int n_beams, int vocab, int n_out) {
    BeamScratch s{};
    s.plan = beam_plan(n_groups * n_beams, n_beams, vocab, n_out, BEAM_SLOTS);
    const size_t parts = (size_t)n_groups * n_beams * s.plan.parts;
    s.sums = align_up(parts * n_out * 8);
    s.scores = s.sums + align_up(parts * sizeof(BeamSum));
    s.total = s.scores + align_up((size_t)n_groups * n_beams * 8);
    return s;
}

}  // namespace

extern "C" {

size_t rs_beam_select_scratch_bytes(int32_t n_groups, int32_t n_beams, int32_t vocab, int32_t n_out) {
    if (n_groups < 1 || n_beams < 1 || n_beams > 64 || n_out < 1 || n_out > 64 || vocab < 1) { fail(RS_EINVAL, "need n_groups >= 1, n_beams and n_out in 1..64, vocab >= 1"); return 0; }
    if ((long long)n_groups * n_beams > 65535) { fail(RS_ECAPACITY, "more than 65535 rows"); return 0; }
    return beam_scratch(n_groups, n_beams, vocab, n_out).total;
}

rs_status rs_beam_select(const void *d_logits, int64_t row_stride, int32_t dtype, int32_t n_groups, int32_t n_beams, int32_t vocab,
                         const float *d_logit_scale, const void *d_score, const int32_t *d_last, int32_t eos, double length_penalty,
                         const int32_t *d_len, int32_t n_out, int32_t *d_parent, int32_t *d_token, void *d_score_out, int32_t *d_len_out,
                         uint32_t *d_flags, void *d_scratch, size_t scratch_bytes, void *stream) {
    if (!d_logits || !d_score || !d_parent || !d_token || !d_score_out || !d_scratch) return fail(RS_EINVAL, "null argument");
    const bool wide = dtype >= 0 && (dtype & RS_SCORES_F64);
    if (wide) dtype -= RS_SCORES_F64;
    if (dtype != RS_F32 && dtype != RS_BF16) return fail(RS_EINVAL, "dtype must be RS_F32 or RS_BF16, with or without RS_SCORES_F64");
    if (n_groups >= 1 && n_beams >= 1 && (long long)n_groups * n_beams > 65535) return fail(RS_ECAPACITY, "%lld rows exceed 65535", (long long)n_groups * n_beams);
    const size_t need = rs_beam_select_scratch_bytes(n_groups, n_beams, vocab, n_out);
    if (!need) return RS_EINVAL;
    if (row_stride < vocab || row_stride > ((int64_t)1 << 40)) return fail(RS_EINVAL, "row_stride must be at least vocab and at most 2^40");
    if (eos < -1 || eos >= vocab) return fail(RS_EINVAL, "eos must be -1 or a token");
    if (!(length_penalty >= 0.0 && length_penalty <= 30.0)) return fail(RS_EINVAL, "length_penalty must be in 0..30");      // ((2^31)^30 is a double)
    if (!d_len && (length_penalty > 0.0 || d_len_out)) return fail(RS_EINVAL, "lengths are needed for length_penalty and d_len_out");
    if ((uintptr_t)d_logits % (dtype == RS_F32 ? 4 : 2)) return fail(RS_EINVAL, "logits are not aligned to their type");
    if (((uintptr_t)d_logit_scale | (uintptr_t)d_score | (uintptr_t)d_last | (uintptr_t)d_len | (uintptr_t)d_parent | (uintptr_t)d_token | (uintptr_t)d_score_out |
         (uintptr_t)d_len_out | (uintptr_t)d_flags) % 4) return fail(RS_EINVAL, "row arguments and outputs must be 4-byte aligned");
    if (wide && ((uintptr_t)d_score | (uintptr_t)d_score_out) % 8) return fail(RS_EINVAL, "double scores must be 8-byte aligned");
    if ((uintptr_t)d_scratch % ALIGN) return fail(RS_EINVAL, "scratch must be 256-byte aligned");
    if (scratch_bytes < need) return fail(RS_EINVAL, "scratch of %zu bytes is smaller than the %zu needed", scratch_bytes, need);
    const int rows = n_groups * n_beams;
    const BeamScratch p = beam_scratch(n_groups, n_beams, vocab, n_out);
    unsigned char *scratch = (unsigned char *)d_scratch;
    BeamArgs a{};
    a.logits = d_logits; a.stride = (size_t)row_stride; a.scale = d_logit_scale; a.score = d_score; a.last = d_last; a.len = d_len;
    a.eos = eos; a.n_beams = n_beams; a.vocab = vocab; a.n_out = n_out; a.alpha = length_penalty; a.parts = p.plan.parts;
    a.parent = d_parent; a.token = d_token; a.len_out = d_len_out; a.score_out = d_score_out; a.wide = wide; a.flags = d_flags;
    a.keys = (unsigned long long *)scratch; a.sums = (BeamSum *)(scratch + p.sums); a.scores = (double *)(scratch + p.scores);
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid(a.parts, rows);
    if (dtype == RS_F32) hipLaunchKernelGGL((k_beam_scan<float>), grid, dim3(BEAM_THREADS), 0, st, a);
    else hipLaunchKernelGGL((k_beam_scan<uint16_t>), grid, dim3(BEAM_THREADS), 0, st, a);
    RS_LAUNCHED("beam_scan");
    const int keys = n_beams * a.parts * n_out;                    // (the smallest block that holds them: 608 keys, a call 12.6 us with 256 threads, 12.7 with 512, 13.6 with 1024)
    hipLaunchKernelGGL(k_beam_join, dim3(n_groups), dim3(keys <= 256 * JOIN_EACH ? 256 : keys <= 512 * JOIN_EACH ? 512 : 1024), 0, st, a);
    RS_LAUNCHED("beam_join");
    return RS_OK;
}

size_t rs_pages_scratch_bytes(const rs_page_pool *pool, int32_t n) {
    if (const char *why = check_pool(pool)) { fail(RS_EINVAL, "%s", why); return 0; }
    if (n < 1 || n > POOL_ROWS) { fail(RS_EINVAL, "n must be in 1..%d", POOL_ROWS); return 0; }
    return pool_scratch(pool, n).total;
}

rs_status rs_pages_release(const rs_page_pool *pool, int32_t n, const int32_t *d_slot, const int32_t *d_from, const int32_t *d_to, uint32_t *d_flags, void *stream) {
    if (const char *why = check_pool(pool)) return fail(RS_EINVAL, "%s", why);
    if (!d_slot || !d_to) return fail(RS_EINVAL, "null argument");
    if (rs_status rc = check_pool_rows(n, d_slot, d_from, d_to, d_flags)) return rc;
    RangeArgs a{};
    a.p = make_pool(pool, d_flags); a.slot = d_slot; a.from = d_from; a.to = d_to; a.n = n;
    hipLaunchKernelGGL(k_pool_release, dim3(n), dim3(256), 0, (hipStream_t)stream, a);
    RS_LAUNCHED("pool_release");
    return RS_OK;
}

rs_status rs_pages_reserve(const rs_page_pool *pool, int32_t n, const int32_t *d_slot, const int32_t *d_from, const int32_t *d_to, uint32_t *d_flags, void *d_scratch,
                           size_t scratch_bytes, void *stream) {
    if (const char *why = check_pool(pool)) return fail(RS_EINVAL, "%s", why);
    if (!d_slot || !d_to) return fail(RS_EINVAL, "null argument");
    if (rs_status rc = check_pool_rows(n, d_slot, d_from, d_to, d_flags)) return rc;
    if (rs_status rc = check_pool_scratch(pool, n, d_scratch, scratch_bytes)) return rc;
    RangeArgs a{};
    a.p = make_pool(pool, d_flags); a.slot = d_slot; a.from = d_from; a.to = d_to; a.n = n;
    a.list = (int *)((unsigned char *)d_scratch + pool_scratch(pool, n).ints);
    hipLaunchKernelGGL(k_pool_reserve, dim3(1), dim3(POOL_THREADS), 0, (hipStream_t)stream, a);
    RS_LAUNCHED("pool_reserve");
    return RS_OK;
}

rs_status rs_pages_fork(const rs_page_pool *pool, int32_t n_groups, int32_t n_beams, const int32_t *d_slot, const int32_t *d_parent, const int32_t *d_pos,
                        int32_t *d_pos_out, uint32_t *d_flags, void *d_scratch, size_t scratch_bytes, void *stream) {
    if (const char *why = check_contents(pool)) return fail(RS_EINVAL, "%s", why);
    if (!d_slot || !d_parent || !d_pos) return fail(RS_EINVAL, "null argument");
    if (n_groups < 1 || n_beams < 1) return fail(RS_EINVAL, "n_groups and n_beams must be at least 1");
    if ((long long)n_groups * n_beams > POOL_ROWS) return fail(RS_ECAPACITY, "%lld rows exceed %d", (long long)n_groups * n_beams, POOL_ROWS);
    const int n = n_groups * n_beams;
    if (rs_status rc = check_pool_rows(n, d_slot, d_parent, d_pos, d_flags)) return rc;
    if ((uintptr_t)d_pos_out % 4) return fail(RS_EINVAL, "positions must be 4-byte aligned");
    if (rs_status rc = check_pool_scratch(pool, n, d_scratch, scratch_bytes)) return rc;
    ForkArgs a{};
    a.p = make_pool(pool, d_flags); a.slot = d_slot; a.parent = d_parent; a.pos = d_pos; a.pos_out = d_pos_out; a.n_groups = n_groups; a.n_beams = n_beams;
    a.n_moves = (int *)d_scratch; a.moves = (PageMove *)((unsigned char *)d_scratch + pool_scratch(pool, n).moves);
    hipStream_t st = (hipStream_t)stream;
    if ((long long)n * pool->max_pages <= FORK_FEW_ENTRIES) hipLaunchKernelGGL((k_pool_fork<FORK_FEW>), dim3(1), dim3(POOL_THREADS), 0, st, a);
    else hipLaunchKernelGGL((k_pool_fork<8>), dim3(1), dim3(POOL_THREADS), 0, st, a);
    RS_LAUNCHED("pool_fork");
    CopyArgs c{};
    c.to = a.p; c.k = a.p.k; c.v = a.p.v; c.from_pages = a.p.n_pages; c.moves = a.moves; c.n_moves = a.n_moves;
    return launch_copy(pool, c, n, st);
}

rs_status rs_pages_copy(const rs_page_pool *to, const rs_page_pool *from, int32_t n, const int32_t *d_src, const int32_t *d_dst, uint32_t *d_flags, void *stream) {
    if (const char *why = check_contents(to)) return fail(RS_EINVAL, "to: %s", why);
    if (const char *why = check_contents(from)) return fail(RS_EINVAL, "from: %s", why);
    if (to->n_layers != from->n_layers || to->page_size != from->page_size || to->n_kv_heads != from->n_kv_heads || to->head_dim != from->head_dim)
        return fail(RS_EINVAL, "the pools differ in layers, page_size, heads or head_dim");
    if (!d_src || !d_dst) return fail(RS_EINVAL, "null argument");
    if (n < 1) return fail(RS_EINVAL, "a call needs at least one pair");
    if (n > (1 << 22)) return fail(RS_ECAPACITY, "%d pairs exceed 2^22", n);
    if (((uintptr_t)d_src | (uintptr_t)d_dst | (uintptr_t)d_flags) % 4) return fail(RS_EINVAL, "pages and flags must be 4-byte aligned");
    CopyArgs c{};
    c.to = make_pool(to, d_flags); c.k = (const uint16_t *)from->k; c.v = (const uint16_t *)from->v; c.from_pages = from->n_pages; c.src = d_src; c.dst = d_dst; c.n = n;
    return launch_copy(to, c, n, (hipStream_t)stream);
}

rs_status rs_pages_compact(const rs_page_pool *pool, int32_t *d_used, void *d_scratch, size_t scratch_bytes, void *stream) {
    if (const char *why = check_contents(pool)) return fail(RS_EINVAL, "%s", why);
    if (!d_used || (uintptr_t)d_used % 4) return fail(RS_EINVAL, "null or misaligned d_used");
    if (rs_status rc = check_pool_scratch(pool, 1, d_scratch, scratch_bytes)) return rc;
    const PoolScratch s = pool_scratch(pool, 1);
    CompactArgs a{};
    a.p = make_pool(pool, nullptr); a.used = d_used;
    a.n_moves = (int *)d_scratch; a.moves = (PageMove *)((unsigned char *)d_scratch + s.moves);
    a.map = (int *)((unsigned char *)d_scratch + s.ints); a.gaps = a.map + pool->n_pages;
    hipStream_t st = (hipStream_t)stream;
    hipLaunchKernelGGL(k_pool_compact, dim3(1), dim3(POOL_THREADS), 0, st, a);
    RS_LAUNCHED("pool_compact");
    CopyArgs c{};
    c.to = a.p; c.k = a.p.k; c.v = a.p.v; c.from_pages = a.p.n_pages; c.moves = a.moves; c.n_moves = a.n_moves; c.map = a.map;
    return launch_copy(pool, c, pool->n_pages / 2, st);
}

}  // extern "C"
