// Attention of new tokens over a cache in pages (rs_paged_attention).
//
// out = sum_j p_j v_j / sum_j p_j with p_j = 2^(c q.k_j - m), c = scale log2 e, over the positions that the row sees, in one
// pass with m the running maximum of c q.k_j, rounded: m is the number itself that p is relative to, so that sums stay as they are where no larger score follows, and
// are multiplied by 2^(m - m') where m' does.  (A running maximum of q.k_j does not do: its product with c is rounded in one place and not in the other, and every tile
// brings that difference again.  lse of 16000 equal scores of 4000 was 0.02 off.)  Both products run on the matrix cores, transposed, so that a lane follows one (row, query head):
//   scores[position, column] = sum_d K[position, d] q[column, d]       A = K, B = q
//   out[d, column]           = sum_j V[j, d] p[column, j]              A = V, which the pages hold by channel, B = p
// The accumulators of the first product are the B operand of the second as they lie: which position a row of A stands for is free, and
// is chosen so that the lane that needs k slots 8 h .. 8 h + 7 holds the scores of eight consecutive positions.  With fp32 q both q
// and p are three bf16 planes (exact: 3 x 8 significant bits).  With bf16 q, q is one plane and p two (16 bits: what is left out is 2^-16 of a term), except in spans
// of several blocks of k_paged_wide (more than 128 columns), where the matrix cores are the bound: there p is rounded to bf16, half a step (2^-8 of a term) at most, as the
// output is.  Errors from 64 bits: 128 sequences of a token 1.7e-3, as the output's rounding alone (with p of one plane 2.2e-3); chunks of 2048 rows, p of one plane, 2.0e-3
// (the output's rounding alone 1.5e-3).
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
constexpr int PAGED_TILE = 6;                  // log2 positions of a tile
// Runs of a call, at most: as many as the CUs hold at a time with head size 128, where a SIMD's 512 registers are two waves of k_paged_wide with one plane of q (252 each), or one
// with three (390; RUNS3), or one of k_paged_narrow.  Smaller head sizes leave room for more wide ones: bf16, 64 tokens, 4000 positions, 8 KV heads, 512 / 768 / 1024 runs: 101 /
// 130 / 111 us with 64 channels, 73 / 62 / 80 with 32; 701 rows of 33 spans, 64 channels, behind a window 30 / 35 / 38.
constexpr int PAGED_WIDE_RUNS = 512, PAGED_WIDE_RUNS3 = 256, PAGED_NARROW_RUNS = 1024;

struct PagedAttnArgs {
    PagedSpans s;
    const uint16_t *kc, *vc;
    const void *q; void *out; float *lse;
    size_t q_stride, out_stride;
    int n_q, group, window, rows, runs;        // rows: of a block of columns; runs: workgroups of the call
    float c;                                   // scale log2 e
    int rsh;                                   // >= 0: fp32 output in operand order with blocks of 1 << rsh rows (frag_index) in the place of rows
    // What is left for k_paged_join: by item, if the call has no more of them than max_items, else by run, the cut item that ends in it.
    int max_items;                             // 0: k_paged_narrow, or more items than runs
    int *entries;                              // how many there are, by item; -1: by run
    int4 *cuts;                                // {first row, KV head, columns, first run | runs << 16}, first row < 0: nothing to do; no runs: whole, with a NaN in its sums
    int2 *cut_of;                              // its {sequence, block}
    unsigned int *odd;                         // by run: bit k % 32: its item k is whole and its sums hold a NaN
    float *part_ml, *part_o;                   // [2 runs][2][columns], [2 runs][columns][head_dim]
};

struct PagedItem { int b, kvh, blk, n_blk; Span s; };
struct PagedRun { PagedItem at; int ta, W, item, n_items; long long left, T; };       // first item, first tile of it; its number, items of the call (-1: too many to have entries); tiles of the run, of the call

// Sum over this lane and those before it: in 32 bits without LDS where no sum passes them.
__device__ __forceinline__ long long wave_prefix(long long v) {
    if (!__any(v >= 1 << 24)) {
        int x = (int)v;
        x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);      // row_shr 1, 2, 4, 8: within rows of 16 lanes
        x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
        x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
        x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
        x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // row_bcast15 into rows 1 and 3
        x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);      // row_bcast31 into rows 2 and 3
        return x;
    }
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const long long u = __shfl_up(v, o, RS_WAVE); if (lane >= o) v += u; }
    return v;
}
__device__ __forceinline__ long long lane_value(long long v, int lane) {
    return (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) | (unsigned)__builtin_amdgcn_readlane((int)v, lane));
}

constexpr int PAGED_RUN_LDS = 16;              // long long

// What run w has to do; false: nothing.  All NT threads of the workgroup get the same.  sh: PAGED_RUN_LDS long long (one wave: not used).
template <int NT>
__device__ __forceinline__ bool paged_find_run(const PagedAttnArgs &a, int w, long long *sh, PagedRun &run) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.s.n_seqs;
    // tiles per KV head of a few sequences a thread, or, where there are many rows, of one sequence by several threads
    int share = 1;
    if (a.s.n_rows > 64 * a.rows) while (share < 64 && 2 * share * n <= NT) share *= 2;
    const int per = (n * share + NT - 1) / NT, b0 = min(tid / share * per, n), b1 = min(b0 + per, n), sub = tid % share;
    Span s;
    s.first = s.m = s.slot = s.p0 = 0;
    auto tiles = [&](int b, int from, int by) __attribute__((always_inline)) {
        long long sum = 0;
        if (!paged_span(a.s, b, s)) { s.m = 0; if (blockIdx.x == 0 && from == 0) paged_flag(a.s, b); }
        else {
            const int nb = paged_blocks(s, a.rows);
            for (int j = from; j < nb; j += by) { int t0, t1; paged_tiles(s, a.rows, a.window, PAGED_TILE, j, t0, t1); sum += t1 - t0; }
        }
        return sum;
    };
    long long mine = 0;
    int blocks = 0;
    for (int b = b0; b < b1; ++b) { mine += tiles(b, sub, share); if (NT > 64) blocks += paged_blocks(s, a.rows); }
    for (int o = 1; o < share; o <<= 1) mine += __shfl_xor(mine, o, RS_WAVE);
    const long long own = sub == 0 ? mine * a.s.n_kv : 0;
    const int own_items = sub == 0 && a.max_items > 0 ? blocks * a.s.n_kv : 0;     // (max_items bounds the rows of a call, so that these stay small)
    long long end = wave_prefix(own), T;
    int items = 0;
    if constexpr (NT == 64) T = lane_value(end, 63);
    else {
        if (a.max_items > 0) items = (int)wave_prefix(own_items);
        if (lane == 63) { sh[wave] = end; sh[12 + wave] = items; }
        __syncthreads();
        T = 0; run.n_items = 0;
        for (int i = 0; i < NT / 64; ++i) { if (i < wave) { end += sh[i]; items += (int)sh[12 + i]; } T += sh[i]; run.n_items += (int)sh[12 + i]; }
    }
    items -= own_items;
    if (NT == 64 || a.max_items == 0 || run.n_items > a.max_items) run.n_items = -1;           // (spans that are no partition of the rows may bring more items than those do)
    const int W = T < a.runs ? (int)T : a.runs;              // (a tile a run at least)
    if (w >= W) return false;
    const long long t0 = paged_run(T, W, w);
    run.T = T; run.W = W; run.left = paged_run(T, W, w + 1) - t0;
    long long rem = 0, of = 0;
    int b = 0;
    const bool found = sub == 0 && t0 >= end - own && t0 < end;
    if (found) {
        rem = t0 - (end - own);
        of = mine; b = b0;
        if (per > 1)
            for (;; ++b) {                                     // (one of the thread's sequences has it)
                of = tiles(b, 0, 1);
                if (rem < of * a.s.n_kv) break;
                rem -= of * a.s.n_kv;
                if (NT > 64) items += paged_blocks(s, a.rows) * a.s.n_kv;
            }
    }
    PagedItem &it = run.at;
    if constexpr (NT == 64) {
        const int who = __ffsll((unsigned long long)__ballot(found)) - 1;
        it.b = __builtin_amdgcn_readlane(b, who); rem = lane_value(rem, who); of = lane_value(of, who);
        it.s.first = __builtin_amdgcn_readlane(s.first, who); it.s.m = __builtin_amdgcn_readlane(s.m, who);
        it.s.slot = __builtin_amdgcn_readlane(s.slot, who); it.s.p0 = __builtin_amdgcn_readlane(s.p0, who);
    } else {
        if (found) { sh[11] = items; sh[4] = b; sh[5] = rem; sh[6] = of; sh[7] = s.first; sh[8] = s.m; sh[9] = s.slot; sh[10] = s.p0; }
        __syncthreads();
        auto value = [&](int i) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane((int)sh[i]); };
        it.b = value(4); rem = lane_value(sh[5], 0); of = lane_value(sh[6], 0);
        it.s.first = value(7); it.s.m = value(8); it.s.slot = value(9); it.s.p0 = value(10);
        run.item = value(11);
    }
    it.n_blk = paged_blocks(it.s, a.rows);
    it.kvh = rem >> 31 == 0 && of >> 31 == 0 ? (int)((unsigned)rem / (unsigned)of) : (int)(rem / of);
    rem -= it.kvh * of;
    int j = 0, u0, u1;
    if (it.n_blk > 1) {
        // the block, by every wave: a lane sums a run of blocks
        const int each = (it.n_blk + 63) / 64, j0 = min(lane * each, it.n_blk), j1 = min(j0 + each, it.n_blk);
        long long sum = 0;
        for (int i = j0; i < j1; ++i) { paged_tiles(it.s, a.rows, a.window, PAGED_TILE, i, u0, u1); sum += u1 - u0; }
        const long long upto = wave_prefix(sum);
        const int who = __ffsll((unsigned long long)__ballot(rem < upto)) - 1;             // (rem < of: some lane has it)
        rem -= lane_value(upto - sum, who);
        j = who * each;
    }
    for (;; ++j) {
        paged_tiles(it.s, a.rows, a.window, PAGED_TILE, j, u0, u1);
        if (rem < u1 - u0) break;
        rem -= u1 - u0;
    }
    it.blk = __builtin_amdgcn_readfirstlane(j);
    run.ta = __builtin_amdgcn_readfirstlane(u0 + (int)rem);
    if (NT > 64) run.item += it.kvh * it.n_blk + it.blk;
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

// Item `it`, number `item`, ends in run w, which has it from tile ta of t0 .. on: what is left for the joining kernel, if anything.  odd: its sums hold a NaN.
__device__ __forceinline__ void paged_note_end(const PagedAttnArgs &a, const PagedRun &run, const PagedItem &it, int w, int item, int ta, int t0, bool odd) {
    if (threadIdx.x != 0) return;
    const bool by_item = run.n_items >= 0;
    const int at = by_item ? item : w, r0 = it.blk * a.rows;
    if (ta == t0 && !(odd && by_item)) { if (by_item) a.cuts[at] = make_int4(-1, 0, 0, 0); return; }
    const int first = ta > t0 ? paged_run_of(run.T, run.W, paged_run(run.T, run.W, w) - (ta - t0)) : 0, pieces = ta > t0 ? w - first + 1 : 0;
    a.cuts[at] = make_int4(it.s.first + r0, it.kvh, min(a.rows, it.s.m - r0) * a.group, first | pieces << 16);
    a.cut_of[at] = make_int2(it.b, it.blk);
}
// Before the first item of run w, also of one that has none.
__device__ __forceinline__ void paged_note_start(const PagedAttnArgs &a, const PagedRun &run, int w) {
    if (threadIdx.x != 0) return;
    if (a.max_items > 0 && w == 0) *a.entries = run.n_items;
    if (run.n_items < 0) { a.cuts[w] = make_int4(-1, 0, 0, 0); a.odd[w] = 0; }
}

// Page table entry of position pos, or of the position nearest to it among the needed ones, lo .. hi - 1; asked for ahead of its use, which checks it:
__device__ __forceinline__ int paged_entry(const PagedAttnArgs &a, const Span &s, int pos, int lo, int hi) {
    return a.s.table[(size_t)s.slot * a.s.max_pages + (min(max(pos, lo), hi - 1) >> a.s.page_shift)];
}
// a page of the cache, whatever the entry holds.
__device__ __forceinline__ int paged_page(const PagedAttnArgs &a, int b, int entry) {
    if ((unsigned)entry < (unsigned)a.s.n_pages) return entry;
    paged_flag(a.s, b);
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
    if constexpr (PL == 3) split3(p, out);
    else {
        float rest[8];
#pragma unroll
        for (int pl = 0; pl < PL; ++pl) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float x = pl ? rest[2 * k] : p[2 * k], y = pl ? rest[2 * k + 1] : p[2 * k + 1];
                w[k] = pack_bf16x2(x, y);
                rest[2 * k] = x - bf16_lo(w[k]); rest[2 * k + 1] = y - bf16_hi(w[k]);
            }
            out[pl] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
        }
    }
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
// four consecutive channels of a row's head
template <int HD, int PL>
__device__ __forceinline__ void paged_store4(const PagedAttnArgs &a, int row, int head, int channel, float x, float y, float z, float w) {
    const int k = head * HD + channel;
    if constexpr (PL == 1) *reinterpret_cast<uint2 *>((uint16_t *)a.out + (size_t)row * a.out_stride + k) = make_uint2(pack_bf16x2(x, y), pack_bf16x2(z, w));
    else *reinterpret_cast<float4 *>((float *)a.out + (a.rsh >= 0 ? frag_index(row, k, a.n_q * HD, a.rsh) : (size_t)row * a.out_stride + k)) = make_float4(x, y, z, w);
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
                paged_store4<HD, PL>(a, row, head, 32 * d + 2 * i + 4 * hh, o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv);
        if (hh == 0 && a.lse) a.lse[(size_t)row * a.n_q + head] = (m + __log2f(l)) * 0.69314718055994531f;
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
// infinities and NaN stay out of the products and reach the columns that see them by being counted, at the end: a sum that had one would be multiplied by the 0 that a much
// higher score makes of the factor, which is a NaN.  Operands come straight from the pages, 32
// channels of the result at a time: few registers, so that the kernel it is part of starts fast when there is nothing of the kind.
template <int HD, int PL>
__device__ __forceinline__ void paged_careful(const PagedAttnArgs &a, const PagedItem &it, int c0, int c_from, int c_to) {
    const int lane = threadIdx.x & 63, col = lane & 31, hh = lane >> 5, c = c0 + col, row = c / a.group, head = it.kvh * a.group + c - row * a.group;
    const int r0 = it.blk * a.rows, nr = min(a.rows, it.s.m - r0);
    const bool valid = c < nr * a.group;
    int lo, hi, see_lo, see_hi;
    paged_seen(it.s, r0, r0 + nr, a.window, lo, hi);
    paged_seen(it.s, r0 + row, r0 + row + 1, a.window, see_lo, see_hi);
    if (!valid) see_hi = 0;
    const int k_row = 16 * ((col >> 4) & 1) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3), in_page = (1 << a.s.page_shift) - 1;
    const size_t q_at = (size_t)(it.s.first + r0 + row) * a.q_stride + (size_t)head * HD + 8 * hh;
#pragma unroll 1
    for (int d = 0; d < HD / 32; ++d) {
        float m = -INFINITY, l = 0.f;
        f32x16_t o;
        unsigned int plus = 0, minus = 0, nan = 0;             // bit i: channel i's column sees one
#pragma unroll
        for (int i = 0; i < 16; ++i) o[i] = 0.f;
#pragma unroll 1
        for (int first = lo & ~31; first < hi; first += 32) {
            const size_t kp = ((size_t)paged_page(a, it.b, paged_entry(a, it.s, first + k_row, lo, hi)) * a.s.n_kv + it.kvh) << a.s.page_shift;
            f32x16_t sc;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll 1
            for (int s = 0; s < HD / 16; ++s) {
                const bf16x8_t A = *reinterpret_cast<const bf16x8_t *>(a.kc + (kp + ((first + k_row) & in_page)) * HD + 16 * s + 8 * hh);
                bf16x8_t q[PL];
                paged_load_q<PL>(a.q, q_at + 16 * s, valid, q);
#pragma unroll
                for (int pl = PL - 1; pl >= 0; --pl) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, q[pl], sc, 0, 0, 0);
            }
            float mx = -INFINITY;
            auto sees = [&](int i) __attribute__((always_inline)) { const int at = first + 16 * (i >> 3) + 8 * hh + (i & 7); return at >= see_lo && at < see_hi; };
#pragma unroll
            for (int i = 0; i < 16; ++i) { sc[i] = sees(i) ? sc[i] : -INFINITY; mx = fmaxf(mx, sc[i]); }
            mx = fmaxf(mx, __shfl_xor(mx, 32, RS_WAVE));
            const float m_new = fmaxf(m, mx * a.c), mc = m_new == -INFINITY ? 0.f : m_new, alpha = __builtin_amdgcn_exp2f(m - mc);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int i = 0; i < 16; ++i) { sc[i] = __builtin_amdgcn_exp2f(fmaf(sc[i], a.c, -mc)); l += sc[i]; o[i] *= alpha; }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float p8[8], see8[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) { p8[i] = sc[8 * s + i]; see8[i] = sees(8 * s + i) ? 1.f : 0.f; }
                bf16x8_t pb[PL], sb[1];
                paged_planes<PL>(p8, pb);
                paged_planes<1>(see8, sb);
                const int at = first + 16 * s + 8 * hh;
                const size_t vp = ((size_t)paged_page(a, it.b, paged_entry(a, it.s, at, lo, hi)) * a.s.n_kv + it.kvh) * HD;
                const uint4 v = *reinterpret_cast<const uint4 *>(a.vc + ((vp + 32 * d + col) << a.s.page_shift) + (at & in_page));
#pragma unroll
                for (int pl = PL - 1; pl >= 0; --pl) o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(paged_pick<0>(v), pb[pl], o, 0, 0, 0);
#pragma unroll 1
                for (int kind = 1; kind < 4; ++kind) {
                    f32x16_t n;
#pragma unroll
                    for (int i = 0; i < 16; ++i) n[i] = 0.f;
                    n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kind == 1 ? paged_pick<1>(v) : kind == 2 ? paged_pick<2>(v) : paged_pick<3>(v), sb[0], n, 0, 0, 0);
                    unsigned int hit = 0;
#pragma unroll
                    for (int i = 0; i < 16; ++i) hit |= n[i] > 0.f ? 1u << i : 0u;
                    (kind == 1 ? plus : kind == 2 ? minus : nan) |= hit;
                }
            }
        }
        l += __shfl_xor(l, 32, RS_WAVE);
        if (valid && c >= c_from && c < c_to) {
            const size_t at = (size_t)(it.s.first + r0 + row);
            const float inv = 1.f / l;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                o[i] = o[i] * inv + (plus >> i & 1 ? INFINITY : 0.f) + (minus >> i & 1 ? -INFINITY : 0.f) + (nan >> i & 1 ? __uint_as_float(0x7fc00000u) : 0.f);
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                paged_store4<HD, PL>(a, (int)at, head, 32 * d + 2 * i + 4 * hh, o[i], o[i + 1], o[i + 2], o[i + 3]);
            if (d == 0 && hh == 0 && a.lse) a.lse[at * a.n_q + head] = (m + __log2f(l)) * 0.69314718055994531f;
        }
    }
}

// K and V tiles in LDS: rows of K (positions), rows of V (channels, 64 positions), in 16-byte pieces whose order differs from row to row, since a direct load
// cannot pad them and the operand reads (one piece of 16 rows at a time) would meet in the same banks.  A load fetches a contiguous kilobyte's worth of whole
// rows: 128 bytes and more of a row side by side, where operands straight from the pages would be pieces of 64.
// The 16 rows of K that a read takes together are consecutive (wide, rows = 32) or 0 .. 3, 8 .. 11, 16 .. 19, 24 .. 27 (narrow, rows = 16).
template <int HD, int ROWS>
__device__ __forceinline__ unsigned paged_k_swizzle(unsigned row) {
    if (ROWS == 32) return HD == 128 ? row & 15 : HD == 64 ? (row >> 1) & 7 : (row >> 2) & 3;
    return HD == 128 ? (row & 3) | ((row >> 1) & 12) : HD == 64 ? ((row >> 1) & 1) | ((row >> 2) & 6) : (row >> 3) & 3;
}
__device__ __forceinline__ unsigned paged_v_swizzle(unsigned channel) { return (channel >> 1) & 7; }

typedef const __attribute__((address_space(1))) unsigned char paged_global;
typedef __attribute__((address_space(3))) unsigned char paged_local;

template <int N>
__device__ __forceinline__ void paged_wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// The wave's LDS reads have arrived: what they read may be overwritten by a load.
__device__ __forceinline__ void paged_wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// A buffer over what lies behind `at` (uniform): loads from it take a 32-bit place a lane, in one register, and what they have in common in a scalar one.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t paged_buffer(const void *at) { return __builtin_amdgcn_make_buffer_rsrc((void *)at, 0, 0x7fffffff, 0x00027000); }

// The larger of a lane's value and that of the lane 32 further or before.
__device__ __forceinline__ float paged_max_halves(float x) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}

// Rows 16 g .. 16 g + 15 of a tile of K at `at` (uniform: its first row in its page) into kb.
template <int HD, int ROWS>
__device__ __forceinline__ void paged_fetch_k(const void *at, unsigned char *kb, int g) {
    constexpr int RPI = 512 / HD;                             // rows a load fetches
    const unsigned lane = threadIdx.x & 63, kr = lane / (HD / 8);
    const __amdgpu_buffer_rsrc_t buf = paged_buffer(at);
#pragma unroll
    for (int i = 0; i < 16 / RPI; ++i) {
        const unsigned r = RPI * i + kr, piece = (lane & (HD / 8 - 1)) ^ paged_k_swizzle<HD, ROWS>(16 * g + r);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (paged_local *)(kb + (16 * g + RPI * i) * (HD * 2)), 16, kr * (HD * 2) + piece * 16, RPI * i * (HD * 2), 0, 0);
    }
}
// The piece of eight positions that a lane fetches of channels 8 i + lane / 8.
__device__ __forceinline__ int paged_v_piece(int i) { const unsigned lane = threadIdx.x & 63; return (lane & 7) ^ paged_v_swizzle(8 * i + (lane >> 3)); }

// Channels 8 i .. 8 i + 7 of a tile of V, for i = i0, i0 + STEP ..  `page`: of the positions 16 g .. of the tile in lane g.
// (A page of 64 positions and more holds the whole tile; the pieces of smaller ones lie in pages that differ from lane to lane.)
template <int HD, int STEP>
__device__ __forceinline__ void paged_fetch_v(const PagedAttnArgs &a, int t, int kvh, int page, unsigned char *vb, int i0) {
    const unsigned lane = threadIdx.x & 63, in_page = (1u << a.s.page_shift) - 1, pitch = a.s.page_shift + 1;
    if (a.s.page_shift >= PAGED_TILE) {
        const size_t at = ((((size_t)__builtin_amdgcn_readfirstlane(page) * a.s.n_kv + kvh) * HD) << a.s.page_shift) + (64 * t & in_page);
        const __amdgpu_buffer_rsrc_t buf = paged_buffer(a.vc + at);
#pragma unroll
        for (int i = 0; i < HD / 8; i += STEP)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (paged_local *)(vb + (i + i0) * 1024), 16, ((lane >> 3) << pitch) + 16 * paged_v_piece(i + i0), (8 * (i + i0)) << pitch, 0, 0);
    } else {
        // (every second load of a lane takes the same piece)
        constexpr int KINDS = STEP % 2 ? 2 : 1;
        const unsigned char *at[KINDS];
#pragma unroll
        for (int k = 0; k < KINDS; ++k) {
            const int piece = paged_v_piece(i0 + k);
            const size_t first = ((((size_t)__shfl(page, piece >> 1, RS_WAVE) * a.s.n_kv + kvh) * HD) << a.s.page_shift) + ((64 * t + 8 * piece) & in_page);
            at[k] = (const unsigned char *)(a.vc + first) + (size_t)((8 * (i0 + k) + (lane >> 3)) << pitch);
        }
#pragma unroll
        for (int i = 0; i < HD / 8; i += STEP) {
            const unsigned char *&p = at[i % 2 % KINDS];
            __builtin_amdgcn_global_load_lds((paged_global *)p, (paged_local *)(vb + (i + i0) * 1024), 16, 0, 0);
            p += (size_t)(8 * STEP * KINDS) << pitch;
        }
    }
}

// ------------------------------------------------------------------------------------------------
// k_paged_narrow: up to 16 NB columns a block (decode steps, spans of a few rows).  grid: runs, block 64: a wave by itself, four of them on a CU, each
// with one tile of K and one of V in LDS.  Bound by the cache's bytes where there are many, by the chain of loads where there are few: K of the next tile
// is on its way while V of this one is multiplied, and the other way round, also from one item to the next, so that a CU has about 100 KB under way.
// One fp32 token: 12 heads on 2, 200 positions 8.5 us; 28 heads on 4, 4561 positions (9.4 MB) 9.3 us: a launch, the search for
// the run, page table, K, V and the stores one after the other.
// ------------------------------------------------------------------------------------------------
template <int HD, int PL, int NB>
__global__ void __launch_bounds__(64, 1) k_paged_narrow(PagedAttnArgs a) {
    constexpr int NS = HD / 32, ND = HD / 16, COLS = 16 * NB, NL = HD / 8;             // NL: loads of a tile of K, and of V
    constexpr int PP = PL == 1 ? 2 : PL;                              // planes of p: the matrix cores have time, and with one the error of p alone is that of the output's rounding
    __shared__ __align__(16) unsigned char kb[64 * HD * 2], vb[64 * HD * 2];
    const int lane = threadIdx.x, col = lane & 15, hq = lane >> 4, w = blockIdx.x, ps = 1 << a.s.page_shift;
    PagedRun run;
    const bool some = paged_find_run<64>(a, w, nullptr, run);
    paged_note_start(a, run, w);
    if (!some) return;
    // ---- the tile that is fetched next: `left` tiles of the run from it on, positions lo .. hi - 1 of its item are needed
    PagedItem fit = run.at;
    int ft = run.ta, f_t0, f_t1, f_lo, f_hi;
    long long left = run.left;
    auto look = [&]() __attribute__((always_inline)) {
        const int r0 = fit.blk * a.rows;
        paged_seen(fit.s, r0, min(r0 + a.rows, fit.s.m), a.window, f_lo, f_hi);
        f_t0 = f_lo >> PAGED_TILE; f_t1 = ((f_hi - 1) >> PAGED_TILE) + 1;
    };
    auto ask = [&]() __attribute__((always_inline)) { return paged_entry(a, fit.s, 64 * ft + 16 * (lane & 3), f_lo, f_hi); };
    auto fetch_k = [&](int t, int kvh, int page) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const size_t at = (((size_t)__builtin_amdgcn_readlane(page, g) * a.s.n_kv + kvh) << a.s.page_shift) + ((64 * t + 16 * g) & (ps - 1));
            paged_fetch_k<HD, 16>(a.kc + at * HD, kb, g);
        }
    };
    auto fetch_v = [&](int t, int kvh, int page) __attribute__((always_inline)) { paged_fetch_v<HD, 1>(a, t, kvh, page, vb, 0); };
    auto step = [&]() __attribute__((always_inline)) {
        --left; ++ft;
        if (left > 0 && ft == f_t1) { paged_next(a, fit); look(); ft = f_t0; }
    };
    int see_lo[NB], see_hi[NB], n_col = 0;                                // positions that the lane's columns see
    bf16x8_t q[NB][NS][PL];
    float m[NB], l[NB];
    f32x4_t o[NB][ND];
    auto begin = [&](const PagedItem &it) __attribute__((always_inline)) {
        const int r0 = it.blk * a.rows;
        n_col = min(a.rows, it.s.m - r0) * a.group;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int c = 16 * nb + col, r = c / a.group, h = it.kvh * a.group + c - r * a.group;
            const bool valid = c < n_col;
            paged_seen(it.s, r0 + r, r0 + r + 1, a.window, see_lo[nb], see_hi[nb]);
            if (!valid) see_hi[nb] = 0;
            const size_t at = (size_t)(it.s.first + r0 + r) * a.q_stride + (size_t)h * HD + 8 * hq;
#pragma unroll
            for (int s = 0; s < NS; ++s) paged_load_q<PL>(a.q, at + 32 * s, valid, q[nb][s]);
            m[nb] = -INFINITY; l[nb] = 0.f;
#pragma unroll
            for (int d = 0; d < ND; ++d) o[nb][d] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
        }
    };
    look();
    int entry = ask();
    begin(fit);                                                           // (q on its way with the page, ahead of the tiles)
    int page = paged_page(a, fit.b, entry);
    fetch_k(ft, fit.kvh, page);
    fetch_v(ft, fit.kvh, page);
    // ---- the tile that is multiplied
    PagedItem it = fit;
    int t = ft, t0 = f_t0, t1 = f_t1, hi = f_hi, ta = ft, n_items = 0;
    step();
    if (left > 0) entry = ask();
    unsigned int odd = 0;
    while (true) {
        // ---- scores: register i of block 2 s32 + blk is position 64 t + 32 s32 + 8 hq + 4 blk + i of column col
        paged_wait_loads<NL>();                                           // all but V of this tile
        // (operands first, then products that do not wait for each other)
        f32x4_t sc[NB][4];
        bf16x8_t kf[4][NS];
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int kbk = 0; kbk < 4; ++kbk) {
                const int r = 32 * (kbk >> 1) + 8 * (col >> 2) + 4 * (kbk & 1) + (col & 3);
                kf[kbk][s] = *reinterpret_cast<const bf16x8_t *>(kb + r * (HD * 2) + ((4 * s + hq) ^ paged_k_swizzle<HD, 16>(r)) * 16);
            }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int kbk = 0; kbk < 4; ++kbk) sc[nb][kbk] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int pl = PL - 1; pl >= 0; --pl)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int kbk = 0; kbk < 4; ++kbk) sc[nb][kbk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kbk][s], q[nb][s][pl], sc[nb][kbk], 0, 0, 0);
        // ---- the next tile's K goes where this one's was
        const bool more = left > 0;
        PagedItem nit = fit;
        int nt = ft, n_t0 = f_t0, n_t1 = f_t1, n_hi = f_hi;
        if (more) {
            page = paged_page(a, fit.b, entry);
            step();
            if (left > 0) entry = ask();
            paged_wait_reads();
            fetch_k(nt, nit.kvh, page);
        }
        // ---- softmax
        const int first = 64 * t + 8 * hq;
        const bool all = 64 * t + 64 <= it.s.p0 + it.blk * a.rows + 1 && a.window == 0;             // every column sees the whole tile
        bf16x8_t pb[NB][2][PP];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float p[16], mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int at = first + 32 * (i >> 3) + (i & 7);
                p[i] = all || (at >= see_lo[nb] && at < see_hi[nb]) ? sc[nb][i >> 2][i & 3] : -INFINITY;
                mx = fmaxf(mx, p[i]);
            }
            mx = fmaxf(mx, __shfl_xor(mx, 16, RS_WAVE));
            mx = fmaxf(mx, __shfl_xor(mx, 32, RS_WAVE));
            const float m_new = fmaxf(m[nb], mx * a.c), mc = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m[nb] - mc);                           // (no score so far: 0)
            m[nb] = m_new;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) { p[i] = __builtin_amdgcn_exp2f(fmaf(p[i], a.c, -mc)); sum += p[i]; }
            l[nb] = l[nb] * alpha + sum;
#pragma unroll
            for (int d = 0; d < ND; ++d) { o[nb][d][0] *= alpha; o[nb][d][1] *= alpha; o[nb][d][2] *= alpha; o[nb][d][3] *= alpha; }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float p8[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) p8[i] = p[8 * s + i];
                paged_planes<PP>(p8, pb[nb][s]);
            }
        }
        // ---- P V
        if (more) paged_wait_loads<NL>(); else paged_wait_loads<0>();     // all but K of the next tile
        const bool end = 64 * t + 64 > hi;
        uint4 v[ND][2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                v[d][s] = *reinterpret_cast<const uint4 *>(vb + (16 * d + col) * 128 + ((4 * s + hq) ^ paged_v_swizzle(col)) * 16);
                if (end) v[d][s] = paged_first(v[d][s], hi - first - 32 * s);
            }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int pl = PP - 1; pl >= 0; --pl)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int d = 0; d < ND; ++d)
                        o[nb][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v[d][s]), pb[nb][s][pl], o[nb][d], 0, 0, 0);
        if (more) { paged_wait_reads(); fetch_v(nt, nit.kvh, page); }
        // ---- the item's or the run's last tile
        if (t + 1 == t1 || !more) {
            const bool whole = ta == t0 && t + 1 == t1;
            const int part = 2 * w + (ta == t0), r0 = it.blk * a.rows;
            float poison = 0.f;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                l[nb] += __shfl_xor(l[nb], 16, RS_WAVE);
                l[nb] += __shfl_xor(l[nb], 32, RS_WAVE);
                const int c = 16 * nb + col, r = c / a.group, h = it.kvh * a.group + c - r * a.group;
                if (c >= n_col) continue;
                const size_t row = (size_t)(it.s.first + r0 + r);
                const float inv = 1.f / l[nb];
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const f32x4_t x = o[nb][d];
                    poison += (x[0] + x[1]) + (x[2] + x[3]);
                    if (whole) paged_store4<HD, PL>(a, (int)row, h, 16 * d + 4 * hq, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
                    else *reinterpret_cast<float4 *>(a.part_o + ((size_t)part * COLS + c) * HD + 16 * d + 4 * hq) = make_float4(x[0], x[1], x[2], x[3]);
                }
                if (hq == 0) {
                    if (!whole) { a.part_ml[(size_t)part * 2 * COLS + c] = m[nb]; a.part_ml[((size_t)part * 2 + 1) * COLS + c] = l[nb]; }
                    else if (a.lse) a.lse[row * a.n_q + h] = (m[nb] + __log2f(l[nb])) * 0.69314718055994531f;
                }
            }
            const bool nan = __any(poison != poison);
            if (whole && nan) odd |= 1u << (n_items & 31);
            if (t + 1 == t1) paged_note_end(a, run, it, w, 0, ta, t0, nan);
            if (!more) break;
            ++n_items;
            ta = n_t0;
            begin(nit);
        }
        it = nit; t = nt; t0 = n_t0; t1 = n_t1; hi = n_hi;
    }
    if (lane == 0) a.odd[w] = odd;
}

// ------------------------------------------------------------------------------------------------
// k_paged_wide: blocks of 128 columns (chunks of a prompt).  grid: runs, block 256.  Bound by the matrix cores: a tile of 64 positions goes to LDS
// once for all columns, by direct loads that are one tile ahead (two buffers); a wave has 32 columns.
// Sharing the XCD's L2: neighbouring runs, which read the same K and V, are an XCD's, and they read the same tiles at the same time, because a run begins each item at
// the tile that its count of tiles so far gives, modulo the item's, and goes round.  Begun at the first tile each, runs were spread over the whole context
// and 11 % of the requests met in L2: 8.7 GB at 6 TB/s from beyond it for the four chunks of 2048 rows on up to 14000 positions.  Now 62 % do, which is 2 % of the time
// (1243 -> 1219 us).
// Those chunks (40 bf16 heads of 128 on 8, 1.09 TFLOP): 1196 to 1246 us, 870 to 910 TFLOP/s, 73 % of the rate of a large bf16 product (1226); products and exponentials take turns
// in a wave and two waves a SIMD fill each other's gaps.  With the scores of the next tile computed beside this one's exponentials the registers leave one
// wave a SIMD, 2040 us, or spill, 3680.  128 bf16 tokens of 28 heads on 4, 512 .. 4607 positions each (707 MB): 137 us, 5.2 TB/s.  61 fp32 rows, three planes, one wave a
// SIMD: 60 us (its launch bound is one wave at every head size; of 32 and 64 channels two would fit).  701 bf16 rows of 33 sequences, head size 64, window 1000: 20 us.
// ------------------------------------------------------------------------------------------------
template <int HD, int PL>
__global__ void __launch_bounds__(256, PL == 1 ? 2 : 1) k_paged_wide(PagedAttnArgs a) {
    constexpr int NS = HD / 16, ND = HD / 32, COLS = PAGED_COLS, KB = 64 * HD * 2;
    constexpr int RB = PL == 1 ? 2 : 1;                                   // blocks of 32 positions whose scores are held at a time
    __shared__ __align__(16) unsigned char k0[KB], k1[KB], v0[KB], v1[KB];
    __shared__ long long run_sh[PAGED_RUN_LDS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, hh = lane >> 5, ps = 1 << a.s.page_shift;
    const int w = (blockIdx.x & 7) * (a.runs / 8) + (blockIdx.x >> 3);         // (workgroups go round the eight XCDs)
    PagedRun run;
    const bool some = paged_find_run<256>(a, w, run_sh, run);
    paged_note_start(a, run, w);
    if (!some) return;
    PagedItem it = run.at;
    int ta = run.ta;
    // operand reads: row of K that lane % 32 stands for
    const int k_row = 16 * ((col >> 4) & 1) + 8 * ((col >> 2) & 1) + 4 * ((col >> 3) & 1) + (col & 3);
    unsigned int odd = 0;
    int done = 0;
    for (int n_items = 0;; ++n_items) {
        int t0, t1;
        paged_tiles(it.s, a.rows, a.window, PAGED_TILE, it.blk, t0, t1);
        const int tb = (int)min((long long)t1, ta + run.left);
        const int r0 = it.blk * a.rows, nr = min(a.rows, it.s.m - r0), n_col = nr * a.group;
        int lo, hi;
        paged_seen(it.s, r0, r0 + nr, a.window, lo, hi);
        const int c = 32 * wave + col, row = c / a.group, head = it.kvh * a.group + c - row * a.group;
        const bool valid = c < n_col, busy = 32 * wave < n_col;        // (columns that are none have q = 0; nothing of theirs is stored)
        int see_lo, see_hi;
        paged_seen(it.s, r0 + row, r0 + row + 1, a.window, see_lo, see_hi);
        if (!valid) see_hi = 0;
        // bf16 rows: a second plane of p unless the span has several blocks, so that a row's bits depend on its span alone.  One block, us with two planes / one, in a graph: 128
        // single tokens 144 / 140; 33 spans of up to 32 rows behind a window 28.6 / 27.1; 32 spans of 20 rows, 100 columns, 168 / 165; head size 64, 64 spans of 30 rows 98 / 84.
        // Several: four chunks of 2048 rows 1620 / 1235 (with the choice 1253: the registers it takes).
        const bool two_planes = PL == 1 && it.n_blk == 1;
        bf16x8_t q[NS][PL];
        {
            const size_t at = (size_t)(it.s.first + r0 + row) * a.q_stride + (size_t)head * HD + 8 * hh;
#pragma unroll
            for (int s = 0; s < NS; ++s) paged_load_q<PL>(a.q, at + 16 * s, valid, q[s]);
        }
        float m, l;
        f32x16_t o[ND];
        auto ask = [&](int t) __attribute__((always_inline)) { return paged_entry(a, it.s, 64 * t + 16 * (lane & 3), lo, hi); };
        auto fetch = [&](int t, int entry, unsigned char *kb, unsigned char *vb) __attribute__((always_inline)) {
            const int page = paged_page(a, it.b, entry);
            const size_t k_at = (((size_t)__builtin_amdgcn_readlane(page, wave) * a.s.n_kv + it.kvh) << a.s.page_shift) + ((64 * t + 16 * wave) & (ps - 1));
            paged_fetch_k<HD, 32>(a.kc + k_at * HD, kb, wave);
            paged_fetch_v<HD, 4>(a, t, it.kvh, page, vb, wave);
        };
        // RB blocks of 32 positions from `first` on, which lie from row 32 rb0 of the buffers on
        auto block = [&](int first, int rb0, const unsigned char *kb, const unsigned char *vb) __attribute__((always_inline)) {
            f32x16_t sc[RB];
            // operands are read ahead of the products: those of the first block, then one beside each product
            bf16x8_t kf[RB][NS], vf[2][ND];
            auto v_at = [&](int s, int d) __attribute__((always_inline)) { return *reinterpret_cast<const bf16x8_t *>(vb + (32 * d + col) * 128 + ((4 * rb0 + 2 * s + hh) ^ paged_v_swizzle(col)) * 16); };
            auto read_k = [&](int rb) __attribute__((always_inline)) {
                const int r = 32 * (rb0 + rb) + k_row;
#pragma unroll
                for (int s = 0; s < NS; ++s) kf[rb][s] = *reinterpret_cast<const bf16x8_t *>(kb + r * (HD * 2) + ((2 * s + hh) ^ paged_k_swizzle<HD, 32>(r)) * 16);
            };
            read_k(0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[rb][i] = 0.f;
                if (rb + 1 < RB) read_k(rb + 1);
                else
#pragma unroll
                    for (int d = 0; d < ND; ++d) vf[0][d] = v_at(0, d);
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int pl = PL - 1; pl >= 0; --pl) sc[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[rb][s], q[s][pl], sc[rb], 0, 0, 0);
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);           // one LDS read,
                    __builtin_amdgcn_sched_group_barrier(0x008, PL, 0);          // the products of one operand
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // score i of block rb is position first + 32 rb + 16 (i / 8) + 8 hh + i % 8
            const bool edge = first + 32 * RB > it.s.p0 + r0 + 1 || (a.window > 0 && first < it.s.p0 + r0 + nr - a.window);
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
            mx = paged_max_halves(mx) * a.c;
            // the maximum that p is relative to may lag behind by 2^8, and most tiles rescale nothing: l has room, o while |V| times the positions is below 2^119
            if (__any(mx - m > 8.f)) {                     // (no score so far: the difference is infinite, or no number where this tile has none either)
                const float m_new = fmaxf(m, mx), alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
                m = m_new;
                l *= alpha;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
            }
            const float mc = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int i = 0; i < 16; ++i) { sc[rb][i] = __builtin_amdgcn_exp2f(fmaf(sc[rb][i], a.c, -mc)); l += sc[rb][i]; }
#pragma unroll
            for (int s = 0; s < 2 * RB; ++s) {
                float p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = sc[s >> 1][8 * (s & 1) + i];
                bf16x8_t pb[PL];
                paged_planes<PL>(p, pb);
                if (s + 1 < 2 * RB) {
#pragma unroll
                    for (int d = 0; d < ND; ++d) vf[(s + 1) & 1][d] = v_at(s + 1, d);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int pl = PL - 1; pl >= 0; --pl) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[s & 1][d], pb[pl], o[d], 0, 0, 0);
                if (two_planes) {
                    bf16x8_t both[2];
                    paged_planes<2>(p, both);
#pragma unroll
                    for (int d = 0; d < ND; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[s & 1][d], both[1], o[d], 0, 0, 0);
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
                uint4 *at = reinterpret_cast<uint4 *>(vb + ch * 128 + (piece ^ paged_v_swizzle(ch)) * 16);
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
        // (a whole item from the tile on at which a run that has multiplied as many tiles as this one stands, and round: see above)
        const int n = tb - ta, from = n == t1 - t0 ? done % n : 0;
        auto tile = [&](int i) __attribute__((always_inline)) { i += from; return ta + (i >= n ? i - n : i); };
        fetch(tile(0), ask(tile(0)), k0, v0);
        int entry = ask(tile(1));
        for (int i = 0; i < n; i += 2) {
            __builtin_amdgcn_s_waitcnt(0x0f70);                                   // vmcnt(0): this wave's share of tile i has arrived
            __syncthreads();
            clear_end(tile(i), v0);
            if (i + 1 < n) { fetch(tile(i + 1), entry, k1, v1); entry = ask(tile(i + 2)); }
            if (busy) compute(tile(i), k0, v0);
            if (i + 1 >= n) break;
            __builtin_amdgcn_s_waitcnt(0x0f70);
            __syncthreads();
            clear_end(tile(i + 1), v1);
            if (i + 2 < n) { fetch(tile(i + 2), entry, k0, v0); entry = ask(tile(i + 3)); }
            if (busy) compute(tile(i + 1), k1, v1);
        }
        done += n;
        l += __shfl_xor(l, 32, RS_WAVE);
        float poison = 0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) poison += o[d][i];
        const int part = ta == t0 && tb == t1 ? -1 : 2 * w + (ta == t0);
        const bool nan = __syncthreads_or(valid && poison != poison);
        if (nan && part < 0) odd |= 1u << (n_items & 31);
        if (valid) paged_store_cols<HD, PL>(a, it.s.first + r0 + row, head, c, COLS, part, hh, m, l, o);
        if (tb == t1) paged_note_end(a, run, it, w, run.item + n_items, ta, t0, nan);
        run.left -= tb - ta;
        if (run.left <= 0) break;
        paged_next(a, it);
        int n1;
        paged_tiles(it.s, a.rows, a.window, PAGED_TILE, it.blk, ta, n1);
    }
    if (tid == 0 && run.n_items < 0) a.odd[w] = odd;
}

// ------------------------------------------------------------------------------------------------
// k_paged_join: the pieces of a cut item, in the order of their runs, and the items, whole or cut, whose sums hold a NaN, once more.
// grid (runs, shares) or, by item, (entries * shares), block 256: HD / 4 threads a column and, with narrow blocks, whose pieces are many, four such groups that
// share them (of two and four groups with wide blocks 26 and 45 us in the place of 19).  Every piece is read once, eight at a time; what bounds it are the loads'
// time of flight (one fp32 token of 28 heads over 4561 positions: 4 us) and its workgroups, 2.7 ns for one that has no work.  Hence an entry per item where
// a wide call has few: 61 rows of 40 query heads on 8 behind 9001 positions, 24 entries of 16 shares in the place of 256: 19.4 -> 6.0 us.
// At least three waves a SIMD: chunks of 8192 rows 27 us, two (180 registers, the NaN's part) 34.
// ------------------------------------------------------------------------------------------------
template <int HD, int COLS>
__host__ __device__ constexpr int join_groups() { return COLS == PAGED_COLS ? 1 : 4; }                     // threads that share a column's pieces between them: many pieces where blocks are small
template <int HD, int COLS>
__host__ __device__ constexpr int join_cols() { return 1024 / HD / join_groups<HD, COLS>(); }            // columns a workgroup

template <int HD, int PL, int COLS>
__global__ void __launch_bounds__(256, 3) k_paged_join(PagedAttnArgs a) {
    constexpr int TPC = HD / 4, G = join_groups<HD, COLS>(), CPW = join_cols<HD, COLS>(), BATCH = 8;
    __shared__ long long run_sh[PAGED_RUN_LDS];
    __shared__ float o_sh[G > 1 ? G : 1][CPW][HD + 4];
    const int wave = threadIdx.x >> 6;
    int w = blockIdx.x, part = blockIdx.y, share = gridDim.y, n_items = -1;               // workgroup `part` of `share` of entry w
    if (COLS == PAGED_COLS && a.max_items > 0) {
        n_items = *a.entries;
        const unsigned entries = n_items < 0 ? a.runs : n_items;
        if (entries == 0) return;
        share = gridDim.x / entries; w = blockIdx.x % entries; part = blockIdx.x / entries;
        if (part >= share) return;
    }
    const int4 cut = a.cuts[w];
    const unsigned int odd = part == 0 && n_items < 0 ? a.odd[w] : 0;
    if (cut.x < 0 && !odd) return;
    if (cut.x >= 0) {
        const int kvh = cut.y, n_col = cut.z, first = cut.w & 0xffff, n = cut.w >> 16;
        const int unit = threadIdx.x / TPC, g = unit / CPW, lc = unit % CPW, d = 4 * (threadIdx.x % TPC);
        for (int from = part * CPW; from < n_col; from += share * CPW) {
        const int c = from + lc;
        bool nan = n == 0;
        float M = -INFINITY, L = 0.f, x[4] = {};
        if (c < n_col) {
            // piece i is the start of run first + i, except the first one, which is the end of its run.  A batch's loads are under way together.
            for (int i0 = g; i0 < n; i0 += G * BATCH) {
                float m[BATCH], l[BATCH];
                float4 y[BATCH];
#pragma unroll
                for (int k = 0; k < BATCH; ++k) {
                    const int i = i0 + G * k;
                    m[k] = -INFINITY; l[k] = 0.f; y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (i >= n) continue;
                    const size_t at = 2 * (size_t)(first + i) + (i == 0);
                    m[k] = a.part_ml[at * 2 * COLS + c]; l[k] = a.part_ml[(at * 2 + 1) * COLS + c];
                    y[k] = *reinterpret_cast<const float4 *>(a.part_o + (at * COLS + c) * HD + d);
                }
                float top = M;
#pragma unroll
                for (int k = 0; k < BATCH; ++k) top = fmaxf(top, m[k]);
                const float tc = top == -INFINITY ? 0.f : top, e0 = __builtin_amdgcn_exp2f(M - tc);
                M = top; L *= e0; x[0] *= e0; x[1] *= e0; x[2] *= e0; x[3] *= e0;
#pragma unroll
                for (int k = 0; k < BATCH; ++k) {
                    const float e = __builtin_amdgcn_exp2f(m[k] - tc);
                    L = fmaf(l[k], e, L);
                    x[0] = fmaf(y[k].x, e, x[0]); x[1] = fmaf(y[k].y, e, x[1]); x[2] = fmaf(y[k].z, e, x[2]); x[3] = fmaf(y[k].w, e, x[3]);
                }
            }
        }
        if constexpr (G > 1) {
            *reinterpret_cast<float4 *>(&o_sh[g][lc][d]) = make_float4(x[0], x[1], x[2], x[3]);
            if (d == 0) { o_sh[g][lc][HD] = M; o_sh[g][lc][HD + 1] = L; }
            __syncthreads();
            float top = -INFINITY;
#pragma unroll
            for (int k = 0; k < G; ++k) top = fmaxf(top, o_sh[k][lc][HD]);
            const float tc = top == -INFINITY ? 0.f : top;
            M = top; L = 0.f; x[0] = x[1] = x[2] = x[3] = 0.f;
#pragma unroll
            for (int k = 0; k < G; ++k) {
                const float e = __builtin_amdgcn_exp2f(o_sh[k][lc][HD] - tc);
                const float4 y = *reinterpret_cast<const float4 *>(&o_sh[k][lc][d]);
                L = fmaf(o_sh[k][lc][HD + 1], e, L);
                x[0] = fmaf(y.x, e, x[0]); x[1] = fmaf(y.y, e, x[1]); x[2] = fmaf(y.z, e, x[2]); x[3] = fmaf(y.w, e, x[3]);
            }
        }
        if (c < n_col && g == 0 && n > 0) {
            const int r = c / a.group, h = kvh * a.group + c - r * a.group;
            const size_t row = (size_t)(cut.x + r);
            const float inv = 1.f / L, all = (x[0] + x[1]) + (x[2] + x[3]);
            nan = all != all;
            paged_store4<HD, PL>(a, (int)row, h, d, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
            if (d == 0 && a.lse) a.lse[row * a.n_q + h] = ((M == -INFINITY ? 0.f : M) + __log2f(L)) * 0.69314718055994531f;
        }
        if (__syncthreads_or(nan)) {
            const int c0 = (from & ~31) + 32 * wave;
            PagedItem it;
            it.b = a.cut_of[w].x; it.blk = a.cut_of[w].y; it.kvh = kvh;
            (void)paged_span(a.s, it.b, it.s);
            if (c0 < min(from + CPW, n_col)) paged_careful<HD, PL>(a, it, c0, from, from + CPW);
        }
        }
    }
    if (!odd) return;
    PagedRun run;
    if (!paged_find_run<256>(a, w, run_sh, run)) return;
    PagedItem it = run.at;
    for (int k = 0, ta = run.ta;; ++k) {
        int t0, t1;
        paged_tiles(it.s, a.rows, a.window, PAGED_TILE, it.blk, t0, t1);
        if (odd >> (k & 31) & 1 && ta == t0 && run.left >= t1 - t0 && 32 * wave < COLS) paged_careful<HD, PL>(a, it, 32 * wave, 0, COLS);
        run.left -= t1 - ta;
        if (run.left <= 0) return;
        paged_next(a, it);
        paged_tiles(it.s, a.rows, a.window, PAGED_TILE, it.blk, ta, t1);
    }
}

}  // namespace rs
