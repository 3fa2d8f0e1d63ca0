// C entry points of the operators on caches in pages (see include/rstitch.h).  Included by rstitch.hip.
#pragma once

#include "paged_launch.h"

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
    if ((uintptr_t)d_pos % 4) return fail(RS_EINVAL, "positions must be 4-byte aligned");
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
    a.rows_wg = n_rows >= 2048 ? 4 : 1;
    const dim3 grid((n_rows + a.rows_wg - 1) / a.rows_wg);
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
    if (rs_status rc = check_spans(n_seqs, n_rows, d_seq_slot, d_span_offset, d_pos0, d_flags, dtype)) return rc;
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
    const int blocks = append_blocks_most(n_seqs, n_rows);
    // eight q and k heads a workgroup, which share the sines and cosines of its rows, or fewer where that leaves under 512 workgroups (us, 128 rows of one
    // position 6.2 with eight heads each, 9.0 with four; chunks of 8192 rows 47 with eight, 50 with six; 517 rows in 26 blocks 24 with eight, 12 with two)
    const int heads = n_q_heads + cache->n_kv_heads, split = (512 + blocks - 1) / blocks, each = (heads + split - 1) / split;
    a.heads_wg = each < 8 ? each : 8;
    a.rope_wgs = (heads + a.heads_wg - 1) / a.heads_wg;
    const dim3 grid(blocks, a.rope_wgs + cache->n_kv_heads);
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
    const size_t f = paged_shape(cache, n_seqs, n_rows, n_q_heads, RS_F32).total, b = paged_shape(cache, n_seqs, n_rows, n_q_heads, RS_BF16).total;
    return f > b ? f : b;
}

rs_status rs_paged_attention(const rs_paged_kv *cache, int32_t n_seqs, int32_t n_rows, const int32_t *d_seq_slot, const int32_t *d_span_offset,
                             const int32_t *d_pos0, int32_t dtype, int32_t n_q_heads, const void *d_q, int64_t q_stride, float scale, int32_t window,
                             void *d_out, int64_t out_stride, float *d_lse, uint32_t *d_flags, void *d_scratch, size_t scratch_bytes, void *stream) {
    if (const char *why = check_paged_attention(cache, n_q_heads)) return fail(RS_EINVAL, "%s", why);
    if (rs_status rc = check_spans(n_seqs, n_rows, d_seq_slot, d_span_offset, d_pos0, d_flags, dtype)) return rc;
    const int hd = cache->head_dim;
    if (const char *why = check_rows(d_q, q_stride, dtype, n_q_heads, hd)) return fail(RS_EINVAL, "q: %s", why);
    if (const char *why = check_rows(d_out, out_stride, dtype, n_q_heads, hd)) return fail(RS_EINVAL, "out: %s", why);
    if (d_q == d_out) return fail(RS_EINVAL, "out must not be q");
    if (!(scale > 0.f) || !std::isfinite(scale * 1.44269504088896341f)) return fail(RS_EINVAL, "scale must be positive and below 2^127");
    if ((uintptr_t)d_lse % 4) return fail(RS_EINVAL, "lse must be 4-byte aligned");
    if (window < 0) return fail(RS_EINVAL, "window must be at least 0");
    if (!d_scratch || (uintptr_t)d_scratch % ALIGN) return fail(RS_EINVAL, "scratch must be 256-byte aligned");
    const size_t need = rs_paged_attention_scratch_bytes(cache, n_seqs, n_rows, n_q_heads);
    if (scratch_bytes < need) return fail(RS_EINVAL, "scratch of %zu bytes is smaller than the %zu needed", scratch_bytes, need);
    return run_paged_attention(cache, paged_spans(cache, n_seqs, n_rows, d_seq_slot, d_span_offset, d_pos0, d_flags), dtype, n_q_heads, d_q, (size_t)q_stride, scale, window,
                               d_out, (size_t)out_stride, -1, d_lse, (unsigned char *)d_scratch, (hipStream_t)stream);
}

}  // extern "C"
