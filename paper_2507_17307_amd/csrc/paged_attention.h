// Attention of new tokens over a cache in pages (rs_paged_attention).
//
// out = sum_j p_j v_j / sum_j p_j with p_j = 2^(c (q.k_j - m)), c = scale log2 e, over the positions that the row sees, in one
// pass with a running maximum m.
#pragma once

#include "device_utils.h"
#include "paged_rope.h"

namespace rs {

struct PagedAttnArgs {
    PagedSpans s;
    const uint16_t *kc, *vc;
    const void *q; void *out; float *lse;
    size_t q_stride, out_stride;
    int n_q, group, window;
    float c;                                   // scale log2 e
};

// grid (n_rows, ceil(n_q / 4)): a wave per row and query head
template <typename T, int HD>
__global__ void __launch_bounds__(256) k_paged_attention(PagedAttnArgs a) {
    __shared__ float q_sh[4][HD];
    __shared__ int found;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.x, h = blockIdx.y * 4 + wave;
    if (tid == 0) found = -1;
    __syncthreads();
    for (int b = tid; b < a.s.n_seqs; b += 256) {
        Span s;
        if (!paged_span(a.s, b, s)) { if (row == 0 && blockIdx.y == 0) paged_flag(a.s, b); }
        else if (row >= s.first && row < s.first + s.m) found = b;
    }
    if (h < a.n_q)
        for (int c = lane; c < HD; c += 64) {
            const T x = ((const T *)a.q)[(size_t)row * a.q_stride + (size_t)h * HD + c];
            if constexpr (sizeof(T) == 2) q_sh[wave][c] = bf16_to_f32(x); else q_sh[wave][c] = x;
        }
    __syncthreads();
    if (found < 0 || h >= a.n_q) return;
    Span s;
    (void)paged_span(a.s, found, s);
    const int p = s.p0 + row - s.first, lo = a.window ? max(0, p - a.window + 1) : 0, kvh = h / a.group, ps = 1 << a.s.page_shift;
    float m = -INFINITY, l = 0.f, o[HD / 32] = {};
    for (int j0 = lo; j0 <= p; j0 += 64) {
        const int j = j0 + lane;
        float x = -INFINITY;
        const uint16_t *v = a.vc;
        if (j <= p) {
            int page = a.s.table[(size_t)s.slot * a.s.max_pages + (j >> a.s.page_shift)];
            if (page < 0 || page >= a.s.n_pages) { paged_flag(a.s, found); page = 0; }
            const size_t base = (((size_t)page * a.s.n_kv + kvh) << a.s.page_shift) * HD;
            const uint16_t *k = a.kc + base + (size_t)(j & (ps - 1)) * HD;
            v = a.vc + base + (j & (ps - 1));
            float dot = 0.f;
            for (int c = 0; c < HD; c += 8) {
                float y[8];
                RowVec<uint16_t, 8>::load(k + c, y);
#pragma unroll
                for (int i = 0; i < 8; ++i) dot = fmaf(q_sh[wave][c + i], y[i], dot);
            }
            x = dot * a.c;
        }
        const float m_new = fmaxf(m, wave_max(x)), m_use = m_new == -INFINITY ? 0.f : m_new, alpha = exp2f(m - m_use);
        const float w = j <= p ? exp2f(x - m_use) : 0.f;
        l = l * alpha + wave_sum(w);
        m = m_new;
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) o[i] *= alpha;
        for (int c = 0; c < HD; ++c) {
            const float t = wave_sum(j <= p ? w * bf16_to_f32(v[(size_t)c << a.s.page_shift]) : 0.f);
#pragma unroll
            for (int i = 0; i < HD / 32; ++i) if (c == i * 32 + (lane & 31)) o[i] += t;
        }
    }
    if (lane < 32) {
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) {
            const float y = o[i] / l;
            const size_t at = (size_t)row * a.out_stride + (size_t)h * HD + i * 32 + lane;
            if constexpr (sizeof(T) == 2) ((uint16_t *)a.out)[at] = f32_to_bf16(y); else ((float *)a.out)[at] = y;
        }
    }
    if (lane == 0 && a.lse) a.lse[(size_t)row * a.n_q + h] = m * 0.69314718055994531f + logf(l);
}

}  // namespace rs
