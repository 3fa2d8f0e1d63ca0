// C entry points of the caches in pages (see include/rstitch.h): argument checks and launches.  Included by rstitch.hip.
#pragma once

#include "paged_attention.h"
#include "paged_rope.h"

namespace {

const char *check_paged(const rs_paged_kv *c) {
    if (!c) return "null cache";
    if (!c->k || !c->v || !c->page_table) return "null cache pointer";
    if (((uintptr_t)c->k | (uintptr_t)c->v) % 16) return "K and V pages must be 16-byte aligned";
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

rs_status check_spans(int32_t n_seqs, int32_t n_rows, const int32_t *slot, const int32_t *off, const int32_t *pos0, int dtype) {
    if (n_seqs < 1 || n_rows < 1) return fail(RS_EINVAL, "n_seqs and n_rows must be at least 1");
    if (n_seqs > PAGED_MAX_SEQS) return fail(RS_ECAPACITY, "n_seqs %d exceeds %d", n_seqs, PAGED_MAX_SEQS);
    if (n_rows > (1 << 22)) return fail(RS_ECAPACITY, "n_rows %d exceeds 2^22", n_rows);
    if (!slot || !pos0) return fail(RS_EINVAL, "null argument");
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

// Which kernel takes a call: blocks of 16 or 32 columns where the spans have no more than that on average, else of 128.
struct PagedShape { int cols, rows, runs; long long items; size_t of, odd, ml, o, total; };
PagedShape paged_shape(int head_dim, int n_seqs, int n_rows, int group, int n_kv) {
    PagedShape p{};
    const long long slots = ((long long)n_rows * group + n_seqs - 1) / n_seqs;
    p.cols = slots <= 16 ? 16 : slots <= 32 ? 32 : PAGED_COLS;
    p.rows = p.cols / group;
    p.runs = p.cols == PAGED_COLS ? PAGED_WIDE_RUNS : PAGED_NARROW_RUNS;
    p.items = ((long long)n_rows / p.rows + n_seqs) * n_kv;                     // at most
    p.of = align_up((size_t)p.runs * sizeof(int4));
    p.odd = p.of + align_up((size_t)p.runs * sizeof(int2));
    p.ml = p.odd + align_up((size_t)p.runs * 4);
    p.o = p.ml + align_up((size_t)2 * p.runs * 2 * p.cols * 4);
    p.total = p.o + align_up((size_t)2 * p.runs * p.cols * head_dim * 4);
    return p;
}

template <int HD, int PL, int COLS>
rs_status launch_paged(const PagedAttnArgs &a, const PagedShape &p, hipStream_t st) {
    if constexpr (COLS == PAGED_COLS) hipLaunchKernelGGL((k_paged_wide<HD, PL>), dim3(a.runs), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_paged_narrow<HD, PL, COLS / 16>), dim3(a.runs), dim3(64), 0, st, a);
    RS_LAUNCHED("paged_attention");
    // about 2048 workgroups for the items that can be cut (one a run at most); the others end at once
    constexpr int per = join_cols<HD, COLS>();
    const int cut = p.items < a.runs ? (int)p.items : a.runs, most = (a.rows * a.group + per - 1) / per, want = (2048 + cut - 1) / cut;
    hipLaunchKernelGGL((k_paged_join<HD, PL, COLS>), dim3(a.runs, want < most ? want : most), dim3(256), 0, st, a);
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

}  // namespace

extern "C" {

rs_status rs_rope_frequencies(int32_t rot_dim, double theta, int32_t kind, double factor, double original_ctx, double beta_fast, double beta_slow,
                              double *h_inv_freq, float *h_amplitude) {
    if (!h_inv_freq) return fail(RS_EINVAL, "null argument");
    if (rot_dim < 2 || rot_dim % 2 || !(theta > 1.0) || !std::isfinite(theta)) return fail(RS_EINVAL, "need an even rot_dim >= 2 and a finite theta > 1");
    if (kind != RS_ROPE_PLAIN && kind != RS_ROPE_LINEAR && kind != RS_ROPE_BY_PARTS) return fail(RS_EINVAL, "unknown kind %d", kind);
    if (kind != RS_ROPE_PLAIN && !(factor >= 1.0 && std::isfinite(factor))) return fail(RS_EINVAL, "factor must be at least 1");
    if (kind == RS_ROPE_BY_PARTS && !(original_ctx >= 1.0 && std::isfinite(original_ctx) && beta_fast > beta_slow && beta_slow > 0.0 && std::isfinite(beta_fast)))
        return fail(RS_EINVAL, "need original_ctx >= 1 and beta_fast > beta_slow > 0");
    const double two_pi = 6.28318530717958647693;
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = std::pow(theta, -2.0 * i / rot_dim);
        if (kind == RS_ROPE_LINEAR) f /= factor;
        else if (kind == RS_ROPE_BY_PARTS) {
            double keep = (original_ctx * f / two_pi - beta_slow) / (beta_fast - beta_slow);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f *= keep + (1.0 - keep) / factor;
        }
        h_inv_freq[i] = f;
    }
    if (h_amplitude) *h_amplitude = kind == RS_ROPE_BY_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
    return RS_OK;
}

rs_status rs_rope_rows(const rs_rope *rope, int32_t n_rows, const int32_t *d_pos, int32_t dtype, int32_t n_heads, int32_t head_dim, const void *d_x,
                       int64_t x_stride, int32_t inverse, void *d_out, int64_t out_stride, void *stream) {
    if (!rope || !d_pos) return fail(RS_EINVAL, "null argument");
    if (n_rows < 1 || n_heads < 1) return fail(RS_EINVAL, "n_rows and n_heads must be at least 1");
    if (n_rows > (1 << 22) || n_heads > 65536) return fail(RS_ECAPACITY, "more than 2^22 rows or 65536 heads");
    if (head_dim < 8 || head_dim % 8 || head_dim > 1024) return fail(RS_EINVAL, "head_dim must be a multiple of 8 in 8..1024");
    if (dtype != RS_F32 && dtype != RS_BF16) return fail(RS_EINVAL, "dtype must be RS_F32 or RS_BF16");
    if (inverse != 0 && inverse != 1) return fail(RS_EINVAL, "inverse must be 0 or 1");
    if (const char *why = check_rope(rope, head_dim)) return fail(RS_EINVAL, "%s", why);
    if (const char *why = check_rows(d_x, x_stride, dtype, n_heads, head_dim)) return fail(RS_EINVAL, "%s", why);
    if (const char *why = check_rows(d_out, out_stride, dtype, n_heads, head_dim)) return fail(RS_EINVAL, "%s", why);
    if (d_x == d_out && x_stride != out_stride) return fail(RS_EINVAL, "in place needs equal strides");
    RopeRowsArgs a{};
    a.x = d_x; a.out = d_out; a.x_stride = x_stride; a.out_stride = out_stride; a.pos = d_pos; a.inv_freq = rope->d_inv_freq; a.amplitude = rope->amplitude;
    a.n_rows = n_rows; a.n_heads = n_heads; a.head_dim = head_dim; a.half = rope->rot_dim / 2; a.interleaved = rope->interleaved; a.inverse = inverse;
    a.rows_wg = n_rows >= 2048 ? 4 : 1; a.heads_wg = n_heads;
    const dim3 grid((n_rows + a.rows_wg - 1) / a.rows_wg, (n_heads + a.heads_wg - 1) / a.heads_wg);
    const size_t lds = (size_t)a.rows_wg * a.half * 8;
    hipStream_t st = (hipStream_t)stream;
    if (dtype == RS_F32) hipLaunchKernelGGL((k_rope_rows<float, 4>), grid, dim3(256), lds, st, a);
    else if (a.half % 8 == 0) hipLaunchKernelGGL((k_rope_rows<uint16_t, 8>), grid, dim3(256), lds, st, a);
    else hipLaunchKernelGGL((k_rope_rows<uint16_t, 4>), grid, dim3(256), lds, st, a);
    RS_LAUNCHED("rope_rows");
    return RS_OK;
}

rs_status rs_paged_append(const rs_paged_kv *cache, int32_t n_seqs, int32_t n_rows, const int32_t *d_seq_slot, const int32_t *d_span_offset,
                          const int32_t *d_pos0, const rs_rope *rope, int32_t dtype, int32_t n_q_heads, const void *d_q, int64_t q_stride,
                          const void *d_k, int64_t k_stride, const void *d_v, int64_t v_stride, void *d_q_out, int64_t q_out_stride, uint32_t *d_flags,
                          void *stream) {
    if (const char *why = check_paged(cache)) return fail(RS_EINVAL, "%s", why);
    if (rs_status rc = check_spans(n_seqs, n_rows, d_seq_slot, d_span_offset, d_pos0, dtype)) return rc;
    if (n_q_heads < 1 || n_q_heads > 16384) return fail(RS_EINVAL, "n_q_heads must be in 1..16384");
    const int hd = cache->head_dim;
    if (rope) if (const char *why = check_rope(rope, hd)) return fail(RS_EINVAL, "%s", why);
    if (const char *why = check_rows(d_q, q_stride, dtype, n_q_heads, hd)) return fail(RS_EINVAL, "q: %s", why);
    if (const char *why = check_rows(d_k, k_stride, dtype, cache->n_kv_heads, hd)) return fail(RS_EINVAL, "k: %s", why);
    if (const char *why = check_rows(d_v, v_stride, dtype, cache->n_kv_heads, hd)) return fail(RS_EINVAL, "v: %s", why);
    if (const char *why = check_rows(d_q_out, q_out_stride, dtype, n_q_heads, hd)) return fail(RS_EINVAL, "q_out: %s", why);
    if (d_q == d_q_out && q_stride != q_out_stride) return fail(RS_EINVAL, "q in place needs equal strides");
    AppendArgs a{};
    a.s = paged_spans(cache, n_seqs, n_rows, d_seq_slot, d_span_offset, d_pos0, d_flags);
    a.kc = (uint16_t *)cache->k; a.vc = (uint16_t *)cache->v;
    a.q = d_q; a.k = d_k; a.v = d_v; a.q_out = d_q_out;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride;
    if (rope) { a.inv_freq = rope->d_inv_freq; a.amplitude = rope->amplitude; a.half = rope->rot_dim / 2; a.interleaved = rope->interleaved; }
    a.n_q = n_q_heads; a.head_dim = hd;
    a.heads_wg = 8; a.v_heads_wg = 1;
    a.rope_wgs = (n_q_heads + cache->n_kv_heads + a.heads_wg - 1) / a.heads_wg;
    const dim3 grid(append_blocks_most(n_seqs, n_rows), a.rope_wgs + (cache->n_kv_heads + a.v_heads_wg - 1) / a.v_heads_wg);
    const size_t lds = append_lds_bytes(a.half, hd);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == RS_F32) hipLaunchKernelGGL((k_paged_append<float, 4>), grid, dim3(256), lds, st, a);
    else if (a.half % 8 == 0) hipLaunchKernelGGL((k_paged_append<uint16_t, 8>), grid, dim3(256), lds, st, a);
    else hipLaunchKernelGGL((k_paged_append<uint16_t, 4>), grid, dim3(256), lds, st, a);
    RS_LAUNCHED("paged_append");
    return RS_OK;
}

size_t rs_paged_attention_scratch_bytes(const rs_paged_kv *cache, int32_t n_seqs, int32_t n_rows, int32_t n_q_heads) {
    if (const char *why = check_paged_attention(cache, n_q_heads)) { fail(RS_EINVAL, "%s", why); return 0; }
    if (n_seqs < 1 || n_rows < 1 || n_seqs > PAGED_MAX_SEQS || n_rows > (1 << 22)) { fail(RS_EINVAL, "n_seqs must be in 1..%d and n_rows in 1..2^22", PAGED_MAX_SEQS); return 0; }
    return paged_shape(cache->head_dim, n_seqs, n_rows, n_q_heads / cache->n_kv_heads, cache->n_kv_heads).total;
}

rs_status rs_paged_attention(const rs_paged_kv *cache, int32_t n_seqs, int32_t n_rows, const int32_t *d_seq_slot, const int32_t *d_span_offset,
                             const int32_t *d_pos0, int32_t dtype, int32_t n_q_heads, const void *d_q, int64_t q_stride, float scale, int32_t window,
                             void *d_out, int64_t out_stride, float *d_lse, uint32_t *d_flags, void *d_scratch, size_t scratch_bytes, void *stream) {
    if (const char *why = check_paged_attention(cache, n_q_heads)) return fail(RS_EINVAL, "%s", why);
    if (rs_status rc = check_spans(n_seqs, n_rows, d_seq_slot, d_span_offset, d_pos0, dtype)) return rc;
    const int hd = cache->head_dim;
    if (const char *why = check_rows(d_q, q_stride, dtype, n_q_heads, hd)) return fail(RS_EINVAL, "q: %s", why);
    if (const char *why = check_rows(d_out, out_stride, dtype, n_q_heads, hd)) return fail(RS_EINVAL, "out: %s", why);
    if (d_q == d_out) return fail(RS_EINVAL, "out must not be q");
    if (!(scale > 0.f) || !std::isfinite(scale)) return fail(RS_EINVAL, "scale must be positive and finite");
    if (window < 0) return fail(RS_EINVAL, "window must be at least 0");
    if (!d_scratch || (uintptr_t)d_scratch % ALIGN) return fail(RS_EINVAL, "scratch must be 256-byte aligned");
    const size_t need = rs_paged_attention_scratch_bytes(cache, n_seqs, n_rows, n_q_heads);
    if (scratch_bytes < need) return fail(RS_EINVAL, "scratch of %zu bytes is smaller than the %zu needed", scratch_bytes, need);
    PagedAttnArgs a{};
    const PagedShape p = paged_shape(hd, n_seqs, n_rows, n_q_heads / cache->n_kv_heads, cache->n_kv_heads);
    a.s = paged_spans(cache, n_seqs, n_rows, d_seq_slot, d_span_offset, d_pos0, d_flags);
    a.kc = (const uint16_t *)cache->k; a.vc = (const uint16_t *)cache->v;
    a.q = d_q; a.out = d_out; a.lse = d_lse; a.q_stride = q_stride; a.out_stride = out_stride;
    a.n_q = n_q_heads; a.group = n_q_heads / cache->n_kv_heads; a.window = window; a.rows = p.rows;
    a.runs = p.cols == PAGED_COLS && dtype == RS_F32 ? PAGED_WIDE_RUNS3 : p.runs;
    a.c = scale * 1.44269504088896341f;
    a.cuts = (int4 *)d_scratch; a.cut_of = (int2 *)((unsigned char *)d_scratch + p.of); a.odd = (unsigned int *)((unsigned char *)d_scratch + p.odd); a.part_ml = (float *)((unsigned char *)d_scratch + p.ml); a.part_o = (float *)((unsigned char *)d_scratch + p.o);
    return dtype == RS_F32 ? launch_paged_hd<3>(hd, a, p, (hipStream_t)stream) : launch_paged_hd<1>(hd, a, p, (hipStream_t)stream);
}

}  // extern "C"
