// Rotary rows and the writing of a cache in pages (rs_rope_rows, rs_paged_append).
//
// A rotation by the angle position * frequency turns the pair (a, b) into A (a cos - b sin, b cos + a sin).  The angle is a
// product in double, reduced in double to a quarter turn, so that far positions lose nothing; sine and cosine of what is left are
// fp32.  One evaluation serves all heads of a row: a workgroup puts those of its rows into LDS first.
// Both kernels move bytes: every value is read and written once, 16 bytes a lane.
#pragma once

#include "device_utils.h"
#include "paged_plan.h"

namespace rs {

__device__ __forceinline__ void paged_flag(const PagedSpans &a, int b) {
    if (a.flags) atomicOr(a.flags + b, RS_FLAG_BADARG);
}

// ---------------------------------------------------------------- angles
// cos and sin of pos * f, times amplitude.  pi/2 in two doubles; quarter turns are counted in double (at most 2^31 radians).
__device__ __forceinline__ float2 rope_turn(int pos, double f, float amplitude) {
    const double x = (double)pos * f, n = __builtin_rint(x * 0.63661977236758134308);
    const double r = fma(-n, 6.123233995736766036e-17, fma(-n, 1.57079632679489661923, x));
    float s, c;
    sincosf((float)r, &s, &c);
    const int q = (int)((long long)n & 3);
    const float cc = q & 1 ? s : c, ss = q & 1 ? c : s;
    return make_float2(((q + 1) & 2 ? -cc : cc) * amplitude, (q & 2 ? -ss : ss) * amplitude);
}

// ---------------------------------------------------------------- 4 or 8 values of a row
template <typename T, int N> struct RowVec;
template <> struct RowVec<float, 4> {
    static __device__ __forceinline__ void load(const float *p, float (&x)[4]) {
        const float4 v = *reinterpret_cast<const float4 *>(p);
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    }
    static __device__ __forceinline__ void store(float *p, const float (&x)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]); }
};
template <> struct RowVec<uint16_t, 4> {
    static __device__ __forceinline__ void load(const uint16_t *p, float (&x)[4]) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
    }
    static __device__ __forceinline__ void store(uint16_t *p, const float (&x)[4]) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
    }
};
template <> struct RowVec<uint16_t, 8> {
    static __device__ __forceinline__ void load(const uint16_t *p, float (&x)[8]) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
        x[4] = bf16_lo(v.z); x[5] = bf16_hi(v.z); x[6] = bf16_lo(v.w); x[7] = bf16_hi(v.w);
    }
    static __device__ __forceinline__ void store(uint16_t *p, const float (&x)[8]) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
    }
};
template <typename T> struct RowVec<T, 8> {
    static __device__ __forceinline__ void load(const T *p, float (&x)[8]) {
        float lo[4], hi[4];
        RowVec<T, 4>::load(p, lo); RowVec<T, 4>::load(p + 4, hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = lo[i]; x[4 + i] = hi[i]; }
    }
    static __device__ __forceinline__ void store(T *p, const float (&x)[8]) {
        const float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
        RowVec<T, 4>::store(p, lo); RowVec<T, 4>::store(p + 4, hi);
    }
};

// Unit u of a head: VEC pairs (u < half / VEC), or 8 channels behind the rotated ones.
// turns: {cos, sin} of the row's pairs.
template <int VEC>
__device__ __forceinline__ int rope_units(int half, int head_dim) { return half / VEC + (head_dim - 2 * half) / 8; }

template <typename TI, typename TO, int VEC>
__device__ __forceinline__ void rope_unit(const TI *x, TO *y, int u, int half, bool interleaved, const float2 *turns) {
    const int rot_units = half / VEC;
    if (u >= rot_units) {
        const int c = 2 * half + 8 * (u - rot_units);
        float v[8];
        RowVec<TI, 8>::load(x + c, v);
        RowVec<TO, 8>::store(y + c, v);
        return;
    }
    const int i = u * VEC;
    float a[VEC], b[VEC];
    if (interleaved) {
        RowVec<TI, VEC>::load(x + 2 * i, a);
        RowVec<TI, VEC>::load(x + 2 * i + VEC, b);
#pragma unroll
        for (int k = 0; k < VEC / 2; ++k) {
            const float2 t = turns[i + k], w = turns[i + VEC / 2 + k];
            const float p = a[2 * k], q = a[2 * k + 1], r = b[2 * k], s = b[2 * k + 1];
            a[2 * k] = fmaf(p, t.x, -(q * t.y)); a[2 * k + 1] = fmaf(q, t.x, p * t.y);
            b[2 * k] = fmaf(r, w.x, -(s * w.y)); b[2 * k + 1] = fmaf(s, w.x, r * w.y);
        }
        RowVec<TO, VEC>::store(y + 2 * i, a);
        RowVec<TO, VEC>::store(y + 2 * i + VEC, b);
    } else {
        RowVec<TI, VEC>::load(x + i, a);
        RowVec<TI, VEC>::load(x + half + i, b);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const float2 t = turns[i + k];
            const float p = a[k], q = b[k];
            a[k] = fmaf(p, t.x, -(q * t.y)); b[k] = fmaf(q, t.x, p * t.y);
        }
        RowVec<TO, VEC>::store(y + i, a);
        RowVec<TO, VEC>::store(y + half + i, b);
    }
}

// The units of `rows` rows of `heads` heads, by a workgroup of 256: a thread keeps its unit of a head and walks the heads, row after row (no divisions on the way).
// f(row, head, unit)
template <typename F>
__device__ __forceinline__ void rope_walk(int rows, int heads, int units, F f) {
    const int at_once = 256 / units, slot = threadIdx.x / units, u = threadIdx.x - slot * units;         // (a head of 1024 channels has 128 units)
    if (slot >= at_once) return;
    const int dr = at_once / heads, dh = at_once - dr * heads;
    for (int r = slot / heads, h = slot - r * heads; r < rows;) {
        f(r, h, u);
        r += dr; h += dh;
        if (h >= heads) { h -= heads; ++r; }
    }
}

// ---------------------------------------------------------------- rs_rope_rows
struct RopeRowsArgs {
    const void *x; void *out; size_t x_stride, out_stride;
    const int *pos; const double *inv_freq; float amplitude;
    int n_rows, n_heads, head_dim, half, interleaved, inverse, rows_wg;
};

// grid row blocks, LDS rows_wg * half float2.  A workgroup has all heads of its rows, so that an angle is computed once.
// Bound by bytes: 16384 bf16 rows of 40 heads of 128 (336 MB read and written) 65 us, 5.2 TB/s, as a large copy (5.1); 128 fp32 rows of 28 heads 3.4 us,
// of which 1.7 are a launch.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) k_rope_rows(RopeRowsArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    float2 *turns = reinterpret_cast<float2 *>(smem);
    const int tid = threadIdx.x, r0 = blockIdx.x * a.rows_wg, n = min(a.rows_wg, a.n_rows - r0);
    for (int i = tid; i < n * a.half; i += 256) {
        const int r = i / a.half;
        float2 t = rope_turn(a.pos[r0 + r], a.inv_freq[i - r * a.half], a.amplitude);
        if (a.inverse) t.y = -t.y;
        turns[i] = t;
    }
    __syncthreads();
    rope_walk(n, a.n_heads, rope_units<VEC>(a.half, a.head_dim), [&](int r, int h, int u) __attribute__((always_inline)) {
        const T *x = (const T *)a.x + (size_t)(r0 + r) * a.x_stride + (size_t)h * a.head_dim;
        T *y = (T *)a.out + (size_t)(r0 + r) * a.out_stride + (size_t)h * a.head_dim;
        rope_unit<T, T, VEC>(x, y, u, a.half, a.interleaved, turns + r * a.half);
    });
}

// ---------------------------------------------------------------- rs_paged_append
struct AppendArgs {
    PagedSpans s;
    uint16_t *kc, *vc;
    const void *q, *k, *v; void *q_out;
    size_t q_stride, k_stride, v_stride, q_out_stride;
    const double *inv_freq; float amplitude;
    int n_q, head_dim, half, interleaved, heads_wg, rope_wgs;
};

constexpr int APPEND_V_PITCH = 2;                                  // spare values of a row of V in LDS
__host__ __device__ __forceinline__ size_t append_lds_bytes(int half, int head_dim) {
    const size_t turns = (size_t)APPEND_BLOCK * half * 8, v = (size_t)APPEND_BLOCK * (head_dim + APPEND_V_PITCH) * 2;
    return turns > v ? turns : v;
}

// grid (blocks of positions, at most; rope_wgs blocks of q and k heads and then a V head each).  A block is 64 aligned positions of one sequence, so that V,
// which turns from rows into channels in LDS, is written in pieces of 16 bytes and a channel's 128 bytes lie side by side; q and k pass through
// registers.  Bound by bytes: chunks of 8192 bf16 rows of 40 + 8 + 8 heads (235 MB) 47 us, 5.0 TB/s, as a large copy; single calls by their launch and the
// search for the block: one fp32 row 4.8 us, 128 sequences of one bf16 row 6.0, 517 fp32 rows of nine sequences 11.2.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) k_paged_append(AppendArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int found[4], wave_n[4], page_of[APPEND_BLOCK];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // ---- the sequence and the block of this workgroup: blocks are counted over the sequences, a few sequences a thread
    if (tid == 0) found[0] = -1;
    const int per = (a.s.n_seqs + 255) / 256, b0 = min(tid * per, a.s.n_seqs), b1 = min(b0 + per, a.s.n_seqs);
    int n = 0;
    for (int b = b0; b < b1; ++b) {
        Span s;
        if (!paged_span(a.s, b, s)) { if (blockIdx.x == 0 && blockIdx.y == 0) paged_flag(a.s, b); }
        else n += append_blocks_of(s);
    }
    int before = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int u = __shfl_up(before, o, RS_WAVE); if (lane >= o) before += u; }
    if (lane == 63) wave_n[wave] = before;
    __syncthreads();
    before -= n;
    for (int w = 0; w < wave; ++w) before += wave_n[w];
    if ((int)blockIdx.x >= before && (int)blockIdx.x < before + n) {
        for (int b = b0; b < b1; ++b) {
            Span s;
            if (!paged_span(a.s, b, s)) continue;
            const int nb = append_blocks_of(s);
            if ((int)blockIdx.x < before + nb) { found[0] = b; found[1] = blockIdx.x - before; break; }
            before += nb;
        }
    }
    __syncthreads();
    const int b = found[0];
    if (b < 0) return;
    Span s;
    (void)paged_span(a.s, b, s);
    const int base = (s.p0 / APPEND_BLOCK + found[1]) * APPEND_BLOCK;                    // (within 2^30)
    const int lo = max(s.p0, base), hi = min(s.p0 + s.m, base + APPEND_BLOCK), rows = hi - lo, r0 = s.first + lo - s.p0;
    const int ps = 1 << a.s.page_shift;
    if (tid < APPEND_BLOCK) {
        int page = -1;
        if (base + tid >= lo && base + tid < hi) {
            page = a.s.table[(size_t)s.slot * a.s.max_pages + ((base + tid) >> a.s.page_shift)];
            if (page < 0 || page >= a.s.n_pages) { page = -1; paged_flag(a.s, b); }
        }
        page_of[tid] = page;
    }
    if ((int)blockIdx.y < a.rope_wgs) {
        float2 *turns = reinterpret_cast<float2 *>(smem);
        for (int i = tid; i < rows * a.half; i += 256) {
            const int r = i / a.half;
            turns[i] = rope_turn(lo + r, a.inv_freq[i - r * a.half], a.amplitude);
        }
        __syncthreads();
        const int h0 = blockIdx.y * a.heads_wg, nh = min(a.heads_wg, a.n_q + a.s.n_kv - h0);
        rope_walk(rows, nh, rope_units<VEC>(a.half, a.head_dim), [&](int r, int hl, int u) __attribute__((always_inline)) {
            const int h = h0 + hl, page = page_of[lo - base + r];
            if (page < 0) return;
            if (h < a.n_q) {
                const T *x = (const T *)a.q + (size_t)(r0 + r) * a.q_stride + (size_t)h * a.head_dim;
                rope_unit<T, T, VEC>(x, (T *)a.q_out + (size_t)(r0 + r) * a.q_out_stride + (size_t)h * a.head_dim, u, a.half, a.interleaved, turns + r * a.half);
            } else {
                const T *x = (const T *)a.k + (size_t)(r0 + r) * a.k_stride + (size_t)(h - a.n_q) * a.head_dim;
                uint16_t *y = a.kc + ((((size_t)page * a.s.n_kv + h - a.n_q) << a.s.page_shift) + ((lo + r) & (ps - 1))) * a.head_dim;
                rope_unit<T, uint16_t, VEC>(x, y, u, a.half, a.interleaved, turns + r * a.half);
            }
        });
        return;
    }
    // ---- V: a head's rows go to LDS and come back by channel
    uint16_t *tile = reinterpret_cast<uint16_t *>(smem);
    const int pitch = a.head_dim + APPEND_V_PITCH, h = blockIdx.y - a.rope_wgs, pieces = a.head_dim / 8;
    for (int i = tid; i < rows * pieces; i += 256) {
        const int r = i / pieces, c = 8 * (i - r * pieces);
        float x[8];
        RowVec<T, 8>::load((const T *)a.v + (size_t)(r0 + r) * a.v_stride + (size_t)h * a.head_dim + c, x);
        uint32_t *t = reinterpret_cast<uint32_t *>(tile + (size_t)(lo - base + r) * pitch + c);
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = pack_bf16x2(x[2 * k], x[2 * k + 1]);
    }
    __syncthreads();
    for (int i = tid; i < a.head_dim * (APPEND_BLOCK / 8); i += 256) {
        const int c = i / (APPEND_BLOCK / 8), o = 8 * (i % (APPEND_BLOCK / 8)), page = page_of[min(max(o, lo - base), hi - 1 - base)];
        if (page < 0 || base + o + 8 <= lo || base + o >= hi) continue;                // (eight places are one page's)
        uint16_t *y = a.vc + ((((size_t)page * a.s.n_kv + h) * a.head_dim + c) << a.s.page_shift) + ((base + o) & (ps - 1));
        if (base + o >= lo && base + o + 8 <= hi) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = tile[(size_t)(o + 2 * k) * pitch + c] | (uint32_t)tile[(size_t)(o + 2 * k + 1) * pitch + c] << 16;
            *reinterpret_cast<uint4 *>(y) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            for (int k = max(0, lo - base - o); k < min(8, hi - base - o); ++k) y[k] = tile[(size_t)(o + k) * pitch + c];
        }
    }
}

}  // namespace rs
