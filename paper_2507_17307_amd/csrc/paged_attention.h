// Attention of new tokens over a cache in pages (rs_paged_attention).
//
// out = sum_j p_j v_j / sum_j p_j with p_j = 2^(c (q.k_j - m)), c = scale log2 e, over the positions that the row sees, in one
// pass with a running maximum m.  Both products run on the matrix cores, transposed, so that a lane follows one (row, query head):
//   scores[position, column] = sum_d K[position, d] q[column, d]       A = K, B = q
//   out[d, column]           = sum_j V[j, d] p[column, j]              A = V, which the pages hold by channel, B = p
// The accumulators of the first product are the B operand of the second as they lie: which position a row of A stands for is free, and
// is chosen so that the lane that needs k slots 8 h .. 8 h + 7 holds the scores of eight consecutive positions.  With fp32 q both q
// and p are three bf16 planes (exact: 3 x 8 significant bits), with bf16 q they are one: p is rounded to bf16, an error of 2^-9 of each term at
// most that is smaller in the sum, as the output's own rounding is 2^-9.
//
// Positions that a row does not see have p = 0, whatever the page holds there.  0 does not take an infinity or a NaN away (and a low plane of p
// may be negative, which turns a seen infinity into a NaN), but every such product is a NaN in the sum: an item whose sums hold one
// is computed once more (by the kernel that joins cut items), with those values left out of the product and counted by the rows that do see them.  What lies behind a sequence's
// last position, where a page that has not been written yet is most likely to hold such values, is cleared instead.
#pragma once

#include "device_utils.h"
#include "model_kernels.h"
#include "paged_rope.h"

namespace rs {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int PAGED_COLS = 128;                // columns of a workgroup of k_paged_wide
constexpr int PAGED_WIDE_TILE = 6, PAGED_NARROW_TILE = 5;      // log2 positions of a tile
constexpr int PAGED_WIDE_RUNS = 512, PAGED_NARROW_RUNS = 1024, PAGED_NARROW_LEAST = 4;

struct PagedAttnArgs {
    PagedSpans s;
    const uint16_t *kc, *vc;
    const void *q; void *out; float *lse;
    size_t q_stride, out_stride;
    int n_q, group, window, rows;              // rows: of a block of columns
    float c;                                   // scale log2 e
    int4 *cuts;                                // per run: the cut item that ends in it {sequence, KV head, block, first run}, sequence < 0: none
    unsigned int *odd;                         // per run: bit k % 32: its item k is whole and its sums hold a NaN
    float *part_ml, *part_o;                   // [2 runs][2][columns], [2 runs][columns][head_dim]
};

struct PagedItem { int b, kvh, blk, n_blk; Span s; };
struct PagedRun { PagedItem at; int ta; long long left, T; int W; };       // first item, first tile of it, tiles of the run

constexpr int PAGED_RUN_LDS = 8;               // long long

// What run w has to do; false: nothing.  All threads of the workgroup (256) get the same.  sh: PAGED_RUN_LDS long long.
__device__ __forceinline__ bool paged_find_run(const PagedAttnArgs &a, int tile_shift, int most, int least, int w, long long *sh, PagedRun &run) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.s.n_seqs;
    // tiles per KV head of a few sequences a thread, or of one sequence by several threads
    int share = 1;
    while (share < 64 && 2 * share * n <= 256) share *= 2;
    const int per = (n * share + 255) / 256, b0 = min(tid / share * per, n), b1 = min(b0 + per, n), sub = tid % share;
    long long mine = 0, one = 0;                             // of all the thread's sequences; of the last one
    for (int b = b0; b < b1; ++b) {
        Span s;
        one = 0;
        if (!paged_span(a.s, b, s)) { if (blockIdx.x == 0 && sub == 0) paged_flag(a.s, b); }
        else {
            const int nb = paged_blocks(s, a.rows);
            for (int j = sub; j < nb; j += share) { int t0, t1; paged_tiles(s, a.rows, a.window, tile_shift, j, t0, t1); one += t1 - t0; }
        }
        mine += one;
    }
    for (int o = 1; o < share; o <<= 1) { one += __shfl_xor(one, o, RS_WAVE); }
    if (share > 1) mine = one;
    const long long own = sub == 0 ? mine * a.s.n_kv : 0;
    long long end = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const long long u = __shfl_up(end, o, RS_WAVE); if (lane >= o) end += u; }
    if (lane == 63) sh[wave] = end;
    __syncthreads();
    for (int i = 0; i < wave; ++i) end += sh[i];
    const long long T = sh[0] + sh[1] + sh[2] + sh[3];
    const int W = paged_runs(T, most, least);
    if (w >= W || T == 0) return false;
    const long long t0 = paged_run(T, W, w), t1 = paged_run(T, W, w + 1);
    run.T = T; run.W = W; run.left = t1 - t0;
    if (t0 >= t1) return false;                              // (more runs than tiles)
    if (sub == 0 && t0 >= end - own && t0 < end) {
        long long rem = t0 - (end - own);
        int b = b0;
        long long of = mine;
        if (per > 1)
            for (; b < b1; ++b) {
                Span s;
                of = 0;
                if (paged_span(a.s, b, s)) {
                    const int nb = paged_blocks(s, a.rows);
                    for (int j = 0; j < nb; ++j) { int u0, u1; paged_tiles(s, a.rows, a.window, tile_shift, j, u0, u1); of += u1 - u0; }
                }
                if (rem < of * a.s.n_kv) break;
                rem -= of * a.s.n_kv;
            }
        sh[4] = b; sh[5] = rem; sh[6] = of;
    }
    __syncthreads();
    PagedItem &it = run.at;
    it.b = (int)sh[4];
    long long rem = sh[5];
    const long long of = sh[6];
    (void)paged_span(a.s, it.b, it.s);
    it.n_blk = paged_blocks(it.s, a.rows);
    it.kvh = (int)(rem / of);
    rem -= it.kvh * of;
    // the block, by every wave: a lane sums a run of blocks
    const int each = (it.n_blk + 63) / 64, j0 = min(lane * each, it.n_blk), j1 = min(j0 + each, it.n_blk);
    long long sum = 0;
    for (int j = j0; j < j1; ++j) { int u0, u1; paged_tiles(it.s, a.rows, a.window, tile_shift, j, u0, u1); sum += u1 - u0; }
    long long upto = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const long long u = __shfl_up(upto, o, RS_WAVE); if (lane >= o) upto += u; }
    const int who = __ffsll((unsigned long long)__ballot(rem < upto)) - 1;             // (rem < of: some lane has it)
    rem -= __shfl(upto - sum, who, RS_WAVE);
    int j = who * each, u0, u1;
    for (;; ++j) {
        paged_tiles(it.s, a.rows, a.window, tile_shift, j, u0, u1);
        if (rem < u1 - u0) break;
        rem -= u1 - u0;
    }
    it.blk = __builtin_amdgcn_readfirstlane(j);
    run.ta = __builtin_amdgcn_readfirstlane(u0 + (int)rem);
    return true;
}

// The item after `it` (there is one).
__device__ __forceinline__ void paged_next(const PagedAttnArgs &a, PagedItem &it) {
    if (++it.blk < it.n_blk) return;
    it.blk = 0;
    if (++it.kvh < a.s.n_kv) return;
    it.kvh = 0;
    do { ++it.b; } while (!paged_span(a.s, it.b, it.s) || it.s.m == 0);
    it.n_blk = paged_blocks(it.s, a.rows);
}

// If item `it`, of which this run w starts at tile ta > t0 and reaches the end, has been cut: who joins it.
__device__ __forceinline__ void paged_note_cut(const PagedAttnArgs &a, const PagedRun &run, const PagedItem &it, int w, int ta, int t0) {
    if (threadIdx.x == 0) a.cuts[w] = make_int4(it.b, it.kvh, it.blk, paged_run_of(run.T, run.W, paged_run(run.T, run.W, w) - (ta - t0)));
}

// Pages of the positions pos .. pos + n - 1 (one page's), of which lo .. hi - 1 are needed: its number, or some page where none is needed or there is none.
__device__ __forceinline__ int paged_page(const PagedAttnArgs &a, const PagedItem &it, int pos, int n, int lo, int hi) {
    if (pos >= hi || pos + n <= lo) return 0;
    const int page = a.s.table[(size_t)it.s.slot * a.s.max_pages + (pos >> a.s.page_shift)];
    if (page >= 0 && page < a.s.n_pages) return page;
    paged_flag(a.s, it.b);
    return 0;
}

// 8 values of q as PL bf16 planes (PL 1: they are bf16)
template <int PL>
__device__ __forceinline__ void paged_load_q(const void *q, size_t at, bool valid, bf16x8_t (&out)[PL]) {
    if constexpr (PL == 1) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (valid) v = *reinterpret_cast<const uint4 *>((const uint16_t *)q + at);
        out[0] = __builtin_bit_cast(bf16x8_t, v);
    } else {
        float x[8] = {};
        if (valid) RowVec<float, 8>::load((const float *)q + at, x);
        split3(x, out);
    }
}
template <int PL>
__device__ __forceinline__ void paged_planes(const float (&p)[8], bf16x8_t (&out)[PL]) {
    if constexpr (PL == 1)
        out[0] = __builtin_bit_cast(bf16x8_t, make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])));
    else split3(p, out);
}

// ---------------------------------------------------------------- infinities and NaN among eight bf16 values
// the first n of them, zeros behind (n <= 0: none)
__device__ __forceinline__ uint32_t paged_first(uint32_t x, int n) { return n >= 2 ? x : n == 1 ? x & 0xffffu : 0u; }
__device__ __forceinline__ uint4 paged_first(const uint4 &v, int n) { return make_uint4(paged_first(v.x, n), paged_first(v.y, n - 2), paged_first(v.z, n - 4), paged_first(v.w, n - 6)); }
// one value: KIND 0: itself, 0 if it is odd; 1 / 2 / 3: one if it is +inf / -inf / NaN, else 0
template <int KIND>
__device__ __forceinline__ uint32_t paged_pick1(uint32_t x) {
    const bool odd = (x & 0x7f80u) == 0x7f80u;
    if (KIND == 0) return odd ? 0u : x;
    return (KIND == 1 ? x == 0x7f80u : KIND == 2 ? x == 0xff80u : odd && (x & 0x7fu)) ? 0x3f80u : 0u;
}
template <int KIND>
__device__ __forceinline__ uint32_t paged_pick(uint32_t x) { return paged_pick1<KIND>(x & 0xffffu) | paged_pick1<KIND>(x >> 16) << 16; }
template <int KIND>
__device__ __forceinline__ bf16x8_t paged_pick(const uint4 &v) {
    return __builtin_bit_cast(bf16x8_t, make_uint4(paged_pick<KIND>(v.x), paged_pick<KIND>(v.y), paged_pick<KIND>(v.z), paged_pick<KIND>(v.w)));
}
// four consecutive channels of a row
template <int PL>
__device__ __forceinline__ void paged_store4(void *out, size_t at, float x, float y, float z, float w) {
    if constexpr (PL == 1) *reinterpret_cast<uint2 *>((uint16_t *)out + at) = make_uint2(pack_bf16x2(x, y), pack_bf16x2(z, w));
    else *reinterpret_cast<float4 *>((float *)out + at) = make_float4(x, y, z, w);
}

// What a lane of 32 columns holds: channels 32 d + 8 (i / 4) + 4 hh + i % 4 of its column; to the row (part < 0) or to a piece.
template <int HD, int PL>
__device__ __forceinline__ void paged_store_cols(const PagedAttnArgs &a, int row, int head, int c, int cols, int part, int hh, float m, float l, const f32x16_t (&o)[HD / 32]) {
    if (part < 0) {
        const float inv = 1.f / l;
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                paged_store4<PL>(a.out, (size_t)row * a.out_stride + (size_t)head * HD + 32 * d + 2 * i + 4 * hh, o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv);
        if (hh == 0 && a.lse) a.lse[(size_t)row * a.n_q + head] = (m * a.c + __log2f(l)) * 0.69314718055994531f;
    } else {
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<float4 *>(a.part_o + ((size_t)part * cols + c) * HD + 32 * d + 2 * i + 4 * hh) = make_float4(o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]);
        if (hh == 0) { a.part_ml[(size_t)part * 2 * cols + c] = m; a.part_ml[((size_t)part * 2 + 1) * cols + c] = l; }
    }
}

// Columns c_from .. c_to - 1 of c0 .. c0 + 31 of an item, by one wave, for items whose sums hold a NaN: V's
// infinities and NaN stay out of the products and reach the columns that see them by being counted.  Operands come straight from the pages.
template <int HD, int PL>
__device__ __forceinline__ void paged_careful(const PagedAttnArgs &a, const PagedItem &it, int c0, int c_from, int c_to) {
    constexpr int NS = HD / 16, ND = HD / 32;
    const int lane = threadIdx.x & 63, col = lane & 31, hh = lane >> 5, c = c0 + col, row = c / a.group, head = it.kvh * a.group + c - row * a.group;
    const int r0 = it.blk * a.rows, nr = min(a.rows, it.s.m - r0);
    const bool valid = c < nr * a.group;
    int lo, hi, see_lo, see_hi;
    paged_seen(it.s, r0, r0 + nr, a.window, lo, hi);
    paged_seen(it.s, r0 + row, r0 + row + 1, a.window, see_lo, see_hi);
    if (!valid) see_hi = 0;
    const int k_row = 16 * ((col >> 4) & 1) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3), in_page = (1 << a.s.page_shift) - 1;
    const size_t q_at = (size_t)(it.s.first + r0 + row) * a.q_stride + (size_t)head * HD + 8 * hh;
    float m = -INFINITY, l = 0.f;
    f32x16_t o[ND], zero;
#pragma unroll
    for (int i = 0; i < 16; ++i) zero[i] = 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] = zero;
    for (int first = lo & ~31; first < hi; first += 32) {
        const size_t kp = ((size_t)paged_page(a, it, first + (k_row & 16), 16, lo, hi) * a.s.n_kv + it.kvh) << a.s.page_shift;
        f32x16_t sc = zero;
        for (int s = 0; s < NS; ++s) {
            const bf16x8_t A = *reinterpret_cast<const bf16x8_t *>(a.kc + (kp + ((first + k_row) & in_page)) * HD + 16 * s + 8 * hh);
            bf16x8_t q[PL];
            paged_load_q<PL>(a.q, q_at + 16 * s, valid, q);
#pragma unroll
            for (int pl = PL - 1; pl >= 0; --pl) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, q[pl], sc, 0, 0, 0);
        }
        float p[16], see[16], mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at = first + 16 * (i >> 3) + 8 * hh + (i & 7);
            see[i] = at >= see_lo && at < see_hi ? 1.f : 0.f;
            p[i] = see[i] > 0.f ? sc[i] : -INFINITY;
            mx = fmaxf(mx, p[i]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32, RS_WAVE));
        const float m_new = fmaxf(m, mx), mc = m_new == -INFINITY ? 0.f : m_new * a.c, alpha = __builtin_amdgcn_exp2f(fmaf(m, a.c, -mc));
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int i = 0; i < 16; ++i) { p[i] = __builtin_amdgcn_exp2f(fmaf(p[i], a.c, -mc)); l += p[i]; }
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            float p8[8], see8[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) { p8[i] = p[8 * s + i]; see8[i] = see[8 * s + i]; }
            bf16x8_t pb8[PL], sb[1];
            paged_planes<PL>(p8, pb8);
            paged_planes<1>(see8, sb);
            const int at = first + 16 * s + 8 * hh;
            const size_t vp = ((size_t)paged_page(a, it, at, 8, lo, hi) * a.s.n_kv + it.kvh) * HD;
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const uint4 v = *reinterpret_cast<const uint4 *>(a.vc + ((vp + 32 * d + col) << a.s.page_shift) + (at & in_page));
#pragma unroll
                for (int pl = PL - 1; pl >= 0; --pl) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(paged_pick<0>(v), pb8[pl], o[d], 0, 0, 0);
                const f32x16_t up = __builtin_amdgcn_mfma_f32_32x32x16_bf16(paged_pick<1>(v), sb[0], zero, 0, 0, 0);
                const f32x16_t down = __builtin_amdgcn_mfma_f32_32x32x16_bf16(paged_pick<2>(v), sb[0], zero, 0, 0, 0);
                const f32x16_t nan = __builtin_amdgcn_mfma_f32_32x32x16_bf16(paged_pick<3>(v), sb[0], zero, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    o[d][i] += (up[i] > 0.f ? INFINITY : 0.f) + (down[i] > 0.f ? -INFINITY : 0.f) + (nan[i] > 0.f ? __uint_as_float(0x7fc00000u) : 0.f);
            }
        }
    }
    l += __shfl_xor(l, 32, RS_WAVE);
    if (valid && c >= c_from && c < c_to) paged_store_cols<HD, PL>(a, it.s.first + r0 + row, head, c, 0, -1, hh, m, l, o);
}

// ------------------------------------------------------------------------------------------------
// k_paged_narrow: up to 16 NB columns a block (decode steps, spans of a few rows).  grid: runs, block 256.  Bound by the cache's bytes: K and V go
// from the pages straight to registers in operand layout, each wave takes every fourth tile (32 positions) of the run with a softmax
// state of its own, the four states of an item meet in LDS.
// ------------------------------------------------------------------------------------------------
template <int HD, int NB>
__host__ __device__ constexpr size_t paged_narrow_lds() { return (size_t)4 * 16 * NB * (HD + 4) * 4 + 2 * 4 * 16 * NB * 4; }

template <int HD, int PL, int NB>
__global__ void __launch_bounds__(256, PL * NB > 3 ? 1 : 2) k_paged_narrow(PagedAttnArgs a) {
    constexpr int NS = HD / 32, ND = HD / 16, COLS = 16 * NB, PITCH = HD + 4;
    extern __shared__ __align__(16) unsigned char smem[];
    float *o_sh = reinterpret_cast<float *>(smem), *m_sh = o_sh + 4 * COLS * PITCH, *l_sh = m_sh + 4 * COLS;      // [wave][column]
    __shared__ long long run_sh[PAGED_RUN_LDS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, hq = lane >> 4, w = blockIdx.x, ps = 1 << a.s.page_shift;
    PagedRun run;
    const bool some = paged_find_run(a, PAGED_NARROW_TILE, PAGED_NARROW_RUNS, PAGED_NARROW_LEAST, w, run_sh, run);
    if (tid == 0) { a.cuts[w] = make_int4(-1, 0, 0, 0); a.odd[w] = 0; }
    if (!some) return;
    PagedItem it = run.at;
    int ta = run.ta;
    unsigned int odd = 0;
    for (int n_items = 0;; ++n_items) {
        int t0, t1;
        paged_tiles(it.s, a.rows, a.window, PAGED_NARROW_TILE, it.blk, t0, t1);
        const int tb = (int)min((long long)t1, ta + run.left);
        const int r0 = it.blk * a.rows, nr = min(a.rows, it.s.m - r0), n_col = nr * a.group;
        int lo, hi;
        paged_seen(it.s, r0, r0 + nr, a.window, lo, hi);
        // ---- this lane's columns
        int see_lo[NB], see_hi[NB];                                   // positions that the column sees
        bf16x8_t q[NB][NS][PL];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int c = 16 * nb + col, r = c / a.group, h = it.kvh * a.group + c - r * a.group;
            const bool valid = c < n_col;
            paged_seen(it.s, r0 + r, r0 + r + 1, a.window, see_lo[nb], see_hi[nb]);
            if (!valid) see_hi[nb] = 0;
            const size_t at = (size_t)(it.s.first + r0 + r) * a.q_stride + (size_t)h * HD + 8 * hq;
#pragma unroll
            for (int s = 0; s < NS; ++s) paged_load_q<PL>(a.q, at + 32 * s, valid, q[nb][s]);
        }
        float m[NB], l[NB];
        f32x4_t o[NB][ND];
        // K: the lane's row col of block blk is position 8 (col / 4) + 4 blk + col % 4 of the tile; V: channel col, positions 8 hq ..
        const int k_pos = 8 * (col >> 2), v_pos = 8 * hq;
        const size_t page_size = (size_t)a.s.n_kv << a.s.page_shift, head = (size_t)it.kvh << a.s.page_shift;
        uint4 k[2][NS], v[ND];
        int kpage = 0, vpage = 0;
        auto pages = [&](int t) __attribute__((always_inline)) { kpage = paged_page(a, it, 32 * t + k_pos, 8, lo, hi); vpage = paged_page(a, it, 32 * t + v_pos, 8, lo, hi); };
        auto load_k = [&](int t, int page) __attribute__((always_inline)) {
            const uint16_t *p = a.kc + (page * page_size + head + ((32 * t + k_pos + (col & 3)) & (ps - 1))) * HD + 8 * hq;
#pragma unroll
            for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                for (int s = 0; s < NS; ++s) k[blk][s] = *reinterpret_cast<const uint4 *>(p + blk * 4 * HD + 32 * s);
        };
        auto load_v = [&](int t, int page) __attribute__((always_inline)) {
            const uint16_t *p = a.vc + (page * page_size + head) * HD + ((size_t)col << a.s.page_shift) + ((32 * t + v_pos) & (ps - 1));
#pragma unroll
            for (int d = 0; d < ND; ++d) v[d] = *reinterpret_cast<const uint4 *>(p + ((size_t)(16 * d) << a.s.page_shift));
        };
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m[nb] = -INFINITY; l[nb] = 0.f;
#pragma unroll
            for (int d = 0; d < ND; ++d) o[nb][d] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
        }
        int t = ta + wave;
        if (t < tb) {
            pages(t);
            load_k(t, kpage); load_v(t, vpage);
            if (t + 4 < tb) pages(t + 4);
        }
        for (; t < tb; t += 4) {
            const bool more = t + 4 < tb;
            const int first = 32 * t + 8 * hq;                                        // position of the lane's scores
            f32x4_t sc[NB][2];
#pragma unroll
            for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    sc[nb][blk] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s < NS; ++s)
#pragma unroll
                        for (int pl = PL - 1; pl >= 0; --pl)
                            sc[nb][blk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k[blk][s]), q[nb][s][pl], sc[nb][blk], 0, 0, 0);
                }
            // (K's registers are free: the next tile's arrives while this one's V is multiplied, and the other way round)
            const int next_v = vpage;
            if (more) load_k(t + 4, kpage);
            if (t + 8 < tb) pages(t + 8);
            if (32 * t + 32 > hi)
#pragma unroll
                for (int d = 0; d < ND; ++d) v[d] = paged_first(v[d], hi - first);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float p[8], mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[i] = first + i >= see_lo[nb] && first + i < see_hi[nb] ? sc[nb][i >> 2][i & 3] : -INFINITY;
                    mx = fmaxf(mx, p[i]);
                }
                mx = fmaxf(mx, __shfl_xor(mx, 16, RS_WAVE));
                mx = fmaxf(mx, __shfl_xor(mx, 32, RS_WAVE));
                const float m_new = fmaxf(m[nb], mx), mc = m_new == -INFINITY ? 0.f : m_new * a.c;
                const float alpha = __builtin_amdgcn_exp2f(fmaf(m[nb], a.c, -mc));            // (no score so far: 0)
                m[nb] = m_new;
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) { p[i] = __builtin_amdgcn_exp2f(fmaf(p[i], a.c, -mc)); sum += p[i]; }
                l[nb] = l[nb] * alpha + sum;
#pragma unroll
                for (int d = 0; d < ND; ++d) { o[nb][d][0] *= alpha; o[nb][d][1] *= alpha; o[nb][d][2] *= alpha; o[nb][d][3] *= alpha; }
                bf16x8_t pb[PL];
                paged_planes<PL>(p, pb);
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int pl = PL - 1; pl >= 0; --pl)
                        o[nb][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v[d]), pb[pl], o[nb][d], 0, 0, 0);
            }
            if (more) load_v(t + 4, next_v);
        }
        float poison = 0.f;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int d = 0; d < ND; ++d) poison += 16 * nb + col < n_col ? (o[nb][d][0] + o[nb][d][1]) + (o[nb][d][2] + o[nb][d][3]) : 0.f;
        // ---- the four waves' states meet: each leaves its own, then four channels of a column a thread
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            l[nb] += __shfl_xor(l[nb], 16, RS_WAVE);
            l[nb] += __shfl_xor(l[nb], 32, RS_WAVE);
            const int at = wave * COLS + 16 * nb + col;
            if (hq == 0) { m_sh[at] = m[nb]; l_sh[at] = l[nb]; }
            if (16 * nb + col < n_col)
#pragma unroll
                for (int d = 0; d < ND; ++d) *reinterpret_cast<float4 *>(o_sh + at * PITCH + 16 * d + 4 * hq) = make_float4(o[nb][d][0], o[nb][d][1], o[nb][d][2], o[nb][d][3]);
        }
        const bool again = __syncthreads_or(poison != poison);
        const bool whole = ta == t0 && tb == t1;
        const int part = whole ? -1 : 2 * w + (ta == t0);
        if (again && whole) odd |= 1u << (n_items & 31);
        for (int i = tid; i < n_col * (HD / 4); i += 256) {
            const int c = i / (HD / 4), d = 4 * (i - c * (HD / 4));
            float mw[4], M = -INFINITY, L = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) { mw[k] = m_sh[k * COLS + c]; M = fmaxf(M, mw[k]); }
            const float Mc = M == -INFINITY ? 0.f : M * a.c;
            float x[4] = {};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float e = __builtin_amdgcn_exp2f(fmaf(mw[k], a.c, -Mc));
                const float4 y = *reinterpret_cast<const float4 *>(o_sh + (k * COLS + c) * PITCH + d);
                L = fmaf(l_sh[k * COLS + c], e, L);
                x[0] = fmaf(y.x, e, x[0]); x[1] = fmaf(y.y, e, x[1]); x[2] = fmaf(y.z, e, x[2]); x[3] = fmaf(y.w, e, x[3]);
            }
            if (whole) {
                const int r = c / a.group, h = it.kvh * a.group + c - r * a.group;
                const size_t row = (size_t)(it.s.first + r0 + r);
                const float inv = 1.f / L;
                paged_store4<PL>(a.out, row * a.out_stride + (size_t)h * HD + d, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
                if (d == 0 && a.lse) a.lse[row * a.n_q + h] = (Mc + __log2f(L)) * 0.69314718055994531f;
            } else {
                *reinterpret_cast<float4 *>(a.part_o + ((size_t)part * COLS + c) * HD + d) = make_float4(x[0], x[1], x[2], x[3]);
                if (d == 0) { a.part_ml[(size_t)part * 2 * COLS + c] = M; a.part_ml[((size_t)part * 2 + 1) * COLS + c] = L; }
            }
        }
        if (ta > t0 && tb == t1) paged_note_cut(a, run, it, w, ta, t0);
        run.left -= tb - ta;
        if (run.left <= 0) break;
        paged_next(a, it);
        int n1;
        paged_tiles(it.s, a.rows, a.window, PAGED_NARROW_TILE, it.blk, ta, n1);
        __syncthreads();
    }
    if (tid == 0) a.odd[w] = odd;
}

// ------------------------------------------------------------------------------------------------
// k_paged_wide: blocks of 128 columns (chunks of a prompt).  grid: runs, block 256.  Bound by the matrix cores: a tile of 64 positions goes to LDS
// once for all columns, by direct loads that are one tile ahead (two buffers); a wave has 32 columns.  Rows of a buffer are
// 16-byte pieces in an order that differs from row to row, since a direct load cannot pad them and the operand reads (32 rows, one
// piece) would meet in the same banks.
// ------------------------------------------------------------------------------------------------
template <int HD> __device__ __forceinline__ int wide_k_swizzle(int row) { return HD == 128 ? row & 15 : HD == 64 ? (row >> 1) & 7 : (row >> 2) & 3; }

typedef const __attribute__((address_space(1))) unsigned char paged_global;
typedef __attribute__((address_space(3))) unsigned char paged_local;

template <int HD, int PL>
__global__ void __launch_bounds__(256, 2) k_paged_wide(PagedAttnArgs a) {
    constexpr int NS = HD / 16, ND = HD / 32, COLS = PAGED_COLS, KB = 64 * HD * 2, RPI = 1024 / (HD * 2);      // rows of K a load fetches
    constexpr int RB = PL == 1 ? 2 : 1;                                   // blocks of 32 positions whose scores are held at a time
    __shared__ __align__(16) unsigned char k0[KB], k1[KB], v0[KB], v1[KB];
    __shared__ long long run_sh[PAGED_RUN_LDS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, hh = lane >> 5, w = blockIdx.x, ps = 1 << a.s.page_shift;
    PagedRun run;
    const bool some = paged_find_run(a, PAGED_WIDE_TILE, PAGED_WIDE_RUNS, 1, w, run_sh, run);
    if (tid == 0) { a.cuts[w] = make_int4(-1, 0, 0, 0); a.odd[w] = 0; }
    if (!some) return;
    PagedItem it = run.at;
    int ta = run.ta;
    const size_t page_bytes = ((size_t)a.s.n_kv << a.s.page_shift) * HD * 2;
    // this lane's part of a load of K (rows 16 wave + RPI i + kr) and of V (channels 8 (4 i + wave) + lane / 8; one piece of eight positions)
    const int kr = lane / (HD / 8), v_piece = (lane & 7) ^ (lane >> 3);
    // operand reads: row of K that lane % 32 stands for
    const int k_row = 16 * ((col >> 4) & 1) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
    unsigned int odd = 0;
    for (int n_items = 0;; ++n_items) {
        int t0, t1;
        paged_tiles(it.s, a.rows, a.window, PAGED_WIDE_TILE, it.blk, t0, t1);
        const int tb = (int)min((long long)t1, ta + run.left);
        const int r0 = it.blk * a.rows, nr = min(a.rows, it.s.m - r0), n_col = nr * a.group;
        int lo, hi;
        paged_seen(it.s, r0, r0 + nr, a.window, lo, hi);
        const int c = 32 * wave + col, row = c / a.group, head = it.kvh * a.group + c - row * a.group;
        const bool valid = c < n_col, busy = 32 * wave < n_col;
        int see_lo, see_hi;
        paged_seen(it.s, r0 + row, r0 + row + 1, a.window, see_lo, see_hi);
        if (!valid) see_hi = 0;
        bf16x8_t q[NS][PL];
        {
            const size_t at = (size_t)(it.s.first + r0 + row) * a.q_stride + (size_t)head * HD + 8 * hh;
#pragma unroll
            for (int s = 0; s < NS; ++s) paged_load_q<PL>(a.q, at + 16 * s, valid, q[s]);
        }
        float m, l;
        f32x16_t o[ND];
        const unsigned char *kh = (const unsigned char *)a.kc + (((size_t)it.kvh << a.s.page_shift) * HD) * 2;
        const unsigned char *vh = (const unsigned char *)a.vc + (((size_t)it.kvh << a.s.page_shift) * HD) * 2;
        int kpage, vpage;
        auto pages = [&](int t) __attribute__((always_inline)) {
            kpage = paged_page(a, it, 64 * t + 16 * wave, 16, lo, hi);
            vpage = paged_page(a, it, 64 * t + 8 * v_piece, 8, lo, hi);
        };
        auto fetch = [&](int t, unsigned char *kb, unsigned char *vb) __attribute__((always_inline)) {
            const unsigned char *kp = kh + kpage * page_bytes + (size_t)((64 * t + 16 * wave) & (ps - 1)) * (HD * 2);
#pragma unroll
            for (int i = 0; i < 16 / RPI; ++i) {
                const int r = RPI * i + kr;                                              // of the wave's 16 rows
                const int piece = (lane & (HD / 8 - 1)) ^ wide_k_swizzle<HD>(16 * wave + r);
                __builtin_amdgcn_global_load_lds((paged_global *)(kp + r * (HD * 2) + piece * 16), (paged_local *)(kb + (16 * wave + RPI * i) * (HD * 2)), 16, 0, 0);
            }
            const unsigned char *vp = vh + vpage * page_bytes + (size_t)((64 * t + 8 * v_piece) & (ps - 1)) * 2;
#pragma unroll
            for (int i = 0; i < HD / 32; ++i) {
                const int ch = 8 * (4 * i + wave);
                __builtin_amdgcn_global_load_lds((paged_global *)(vp + ((size_t)(ch + (lane >> 3)) << (a.s.page_shift + 1))), (paged_local *)(vb + ch * 128), 16, 0, 0);
            }
        };
        // RB blocks of 32 positions from `first` on, which lie from row 32 rb0 of the buffers on
        auto block = [&](int first, int rb0, const unsigned char *kb, const unsigned char *vb) __attribute__((always_inline)) {
            f32x16_t sc[RB];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[rb][i] = 0.f;
                const int r = 32 * (rb0 + rb) + k_row;
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const bf16x8_t A = *reinterpret_cast<const bf16x8_t *>(kb + r * (HD * 2) + ((2 * s + hh) ^ wide_k_swizzle<HD>(r)) * 16);
#pragma unroll
                    for (int pl = PL - 1; pl >= 0; --pl) sc[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, q[s][pl], sc[rb], 0, 0, 0);
                }
            }
            // score i of block rb is position first + 32 rb + 16 (i / 8) + 8 hh + i % 8
            const bool edge = first + 32 * RB > it.s.p0 + r0 + 1 || (a.window > 0 && first < it.s.p0 + r0 + nr - a.window) || n_col < 32 * wave + 32;
            if (edge)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int at = first + 32 * rb + 16 * (i >> 3) + 8 * hh + (i & 7);
                        if (!(at >= see_lo && at < see_hi)) sc[rb][i] = -INFINITY;
                    }
            float mx = -INFINITY;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[rb][i]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, RS_WAVE));
            // the maximum that p is relative to may lag behind by 2^8: the sums have room, and most tiles rescale nothing
            if (__any((mx - m) * a.c > 8.f || (m == -INFINITY && mx > -INFINITY))) {
                const float m_new = fmaxf(m, mx), alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_new) * a.c);
                m = m_new;
                l *= alpha;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
            }
            const float mc = m == -INFINITY ? 0.f : m * a.c;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int i = 0; i < 16; ++i) { sc[rb][i] = __builtin_amdgcn_exp2f(fmaf(sc[rb][i], a.c, -mc)); l += sc[rb][i]; }
            auto v_at = [&](int s, int d) __attribute__((always_inline)) { return vb + (32 * d + col) * 128 + ((4 * rb0 + 2 * s + hh) ^ (col & 7)) * 16; };
#pragma unroll
            for (int s = 0; s < 2 * RB; ++s) {
                float p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = sc[s >> 1][8 * (s & 1) + i];
                bf16x8_t pb[PL];
                paged_planes<PL>(p, pb);
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const bf16x8_t A = *reinterpret_cast<const bf16x8_t *>(v_at(s, d));
#pragma unroll
                    for (int pl = PL - 1; pl >= 0; --pl) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, pb[pl], o[d], 0, 0, 0);
                }
            }
        };
        auto compute = [&](int t, const unsigned char *kb, const unsigned char *vb) __attribute__((always_inline)) {
#pragma unroll
            for (int rb = 0; rb < 2; rb += RB) block(64 * t + 32 * rb, rb, kb, vb);
        };
        // positions at or past hi of the item's last tile
        auto clear_end = [&](int t, unsigned char *vb) __attribute__((always_inline)) {
            if (64 * t + 64 <= hi) return;
            for (int i = tid; i < HD * 8; i += 256) {
                const int ch = i >> 3, piece = i & 7, n = hi - 64 * t - 8 * piece;
                uint4 *at = reinterpret_cast<uint4 *>(vb + ch * 128 + (piece ^ (ch & 7)) * 16);
                if (n < 8) *at = paged_first(*at, n);
            }
            __syncthreads();
        };
        // ---- tiles ta .. tb - 1: one is multiplied while the next one arrives
        m = -INFINITY; l = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        pages(ta);
        fetch(ta, k0, v0);
        pages(ta + 1);
        for (int t = ta; t < tb; t += 2) {
            __builtin_amdgcn_s_waitcnt(0x0f70);                                   // vmcnt(0): this wave's share of tile t has arrived
            __syncthreads();
            clear_end(t, v0);
            if (t + 1 < tb) { fetch(t + 1, k1, v1); pages(t + 2); }
            if (busy) compute(t, k0, v0);
            if (t + 1 >= tb) break;
            __builtin_amdgcn_s_waitcnt(0x0f70);
            __syncthreads();
            clear_end(t + 1, v1);
            if (t + 2 < tb) { fetch(t + 2, k0, v0); pages(t + 3); }
            if (busy) compute(t + 1, k1, v1);
        }
        l += __shfl_xor(l, 32, RS_WAVE);
        float poison = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) poison += o[d][i];
        const int part = ta == t0 && tb == t1 ? -1 : 2 * w + (ta == t0);
        if (__syncthreads_or(valid && poison != poison) && part < 0) odd |= 1u << (n_items & 31);
        if (valid) paged_store_cols<HD, PL>(a, it.s.first + r0 + row, head, c, COLS, part, hh, m, l, o);
        if (ta > t0 && tb == t1) paged_note_cut(a, run, it, w, ta, t0);
        run.left -= tb - ta;
        if (run.left <= 0) break;
        paged_next(a, it);
        int n1;
        paged_tiles(it.s, a.rows, a.window, PAGED_WIDE_TILE, it.blk, ta, n1);
    }
    if (tid == 0) a.odd[w] = odd;
}

// ------------------------------------------------------------------------------------------------
// k_paged_join: the pieces of a cut item, in the order of their runs.  grid (runs, column groups), block 256: HD / 4 threads a column.
// And the items, whole or cut, whose sums hold a NaN, once more.
// ------------------------------------------------------------------------------------------------
template <int HD, int PL, int COLS>
__global__ void __launch_bounds__(256) k_paged_join(PagedAttnArgs a) {
    __shared__ long long run_sh[PAGED_RUN_LDS];
    const int w = blockIdx.x, wave = threadIdx.x >> 6;
    const int4 cut = a.cuts[w];
    const unsigned int odd = blockIdx.y == 0 ? a.odd[w] : 0;
    if (cut.x < 0 && !odd) return;
    PagedItem it;
    if (cut.x >= 0) {
        it.b = cut.x; it.kvh = cut.y; it.blk = cut.z;
        (void)paged_span(a.s, cut.x, it.s);
        const int r0 = it.blk * a.rows, n_col = min(a.rows, it.s.m - r0) * a.group, n = w - cut.w + 1;
        constexpr int TPC = HD / 4, CPW = 256 / TPC;                               // threads a column, columns at a time
        const int c = blockIdx.y * CPW + threadIdx.x / TPC, d = 4 * (threadIdx.x % TPC);
        bool nan = false;
        if (c < n_col) {
            // piece i is the start of run cut.w + i, except the first one, which is the end of its run
            auto part = [&](int i) __attribute__((always_inline)) { return 2 * (size_t)(cut.w + i) + (i == 0); };
            float M = -INFINITY, L = 0.f, x[4] = {};
            for (int i = 0; i < n; ++i) M = fmaxf(M, a.part_ml[part(i) * 2 * COLS + c]);
            const float Mc = M == -INFINITY ? 0.f : M * a.c;
#pragma unroll 4
            for (int i = 0; i < n; ++i) {
                const float e = __builtin_amdgcn_exp2f(fmaf(a.part_ml[part(i) * 2 * COLS + c], a.c, -Mc));
                const float4 y = *reinterpret_cast<const float4 *>(a.part_o + (part(i) * COLS + c) * HD + d);
                L = fmaf(a.part_ml[(part(i) * 2 + 1) * COLS + c], e, L);
                x[0] = fmaf(y.x, e, x[0]); x[1] = fmaf(y.y, e, x[1]); x[2] = fmaf(y.z, e, x[2]); x[3] = fmaf(y.w, e, x[3]);
            }
            const int r = c / a.group, h = it.kvh * a.group + c - r * a.group;
            const size_t row = (size_t)(it.s.first + r0 + r);
            const float inv = 1.f / L, all = (x[0] + x[1]) + (x[2] + x[3]);
            nan = all != all;
            paged_store4<PL>(a.out, row * a.out_stride + (size_t)h * HD + d, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
            if (d == 0 && a.lse) a.lse[row * a.n_q + h] = (Mc + __log2f(L)) * 0.69314718055994531f;
        }
        if (__syncthreads_or(nan)) {
            const int from = blockIdx.y * CPW, c0 = (from & ~31) + 32 * wave;
            if (c0 < min(from + CPW, n_col)) paged_careful<HD, PL>(a, it, c0, from, from + CPW);
        }
    }
    if (!odd) return;
    PagedRun run;
    constexpr bool WIDE = COLS == PAGED_COLS;
    constexpr int SHIFT = WIDE ? PAGED_WIDE_TILE : PAGED_NARROW_TILE;
    if (!paged_find_run(a, SHIFT, WIDE ? PAGED_WIDE_RUNS : PAGED_NARROW_RUNS, WIDE ? 1 : PAGED_NARROW_LEAST, w, run_sh, run)) return;
    it = run.at;
    for (int k = 0, ta = run.ta;; ++k) {
        int t0, t1;
        paged_tiles(it.s, a.rows, a.window, SHIFT, it.blk, t0, t1);
        if (odd >> (k & 31) & 1 && ta == t0 && run.left >= t1 - t0 && 32 * wave < COLS) paged_careful<HD, PL>(a, it, 32 * wave, 0, COLS);
        run.left -= t1 - ta;
        if (run.left <= 0) return;
        paged_next(a, it);
        paged_tiles(it.s, a.rows, a.window, SHIFT, it.blk, ta, t1);
    }
}

}  // namespace rs
