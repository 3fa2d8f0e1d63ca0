// Selection over beams and vocabulary (rs_beam_select).
//
// The continuation of beam b by token t is worth score_b + (x_t - ln Z_b), x = scale * logits, Z = sum e^x.  Neighbours in the order of a vocabulary,
// and more so across beams, may be nearer than fp32 sums can tell, so the sum of exponentials and all that is compared across beams are double; within a
// row the order is that of the logits themselves.
#pragma once

#include "device_utils.h"
#include "../../include/rstitch.h"

namespace rs {

struct BeamArgs {
    const void *logits; size_t stride;
    const float *scale, *score;
    const int *last, *len;
    int eos, n_groups, n_beams, vocab, n_out;
    double alpha;
    int *parent, *token, *len_out;
    float *score_out;
    unsigned int *flags;
    unsigned long long *keys;                                      // [row][n_out] best logits of a row, in order
    double *log_z;                                                 // [row]
};

// 2^d for d <= 0, to 1.1e-12: 2^n p(d - n), n the nearest integer, p of degree eight through 2^f at the Chebyshev nodes of [-1/2, 1/2].
// Below 2^-1000 it is 2^-1000.
__device__ __forceinline__ double exp2_sum(double d) {
    d = fmax(d, -1000.0);
    const double n = __builtin_rint(d), f = d - n;
    double p = 1.3255224887502117e-06;
    p = fma(p, f, 1.531007940254368e-05); p = fma(p, f, 0.0001540345585240991); p = fma(p, f, 0.0013333450567999414); p = fma(p, f, 0.009618129159402628);
    p = fma(p, f, 0.05550410941205934); p = fma(p, f, 0.2402265069581299); p = fma(p, f, 0.6931471805459335); p = fma(p, f, 1.0);
    return __builtin_ldexp(p, (int)n);
}

// A logit and its token as one number: larger for a larger logit, and for a lower token among equals (-0 and 0 are equal).  0: no candidate.
__device__ __forceinline__ unsigned long long beam_key(float x, int token) {
    const uint32_t u = __float_as_uint(x + 0.f), o = u >> 31 ? ~u : u | 0x80000000u;
    return x > -INFINITY ? (unsigned long long)o << 32 | (uint32_t)~token : 0;
}
__device__ __forceinline__ float key_logit(unsigned long long key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int key_token(unsigned long long key) { return (int)~(uint32_t)key; }

__device__ __forceinline__ float beam_logit(const float *x, int i) { return x[i]; }
__device__ __forceinline__ float beam_logit(const uint16_t *x, int i) { return bf16_to_f32(x[i]); }

// What a row takes part with: its vocabulary, its end, or nothing.
enum { BEAM_NONE, BEAM_ENDED, BEAM_RUNS };
__device__ __forceinline__ int beam_row(const BeamArgs &a, int row, unsigned int &flag) {
    const float score = a.score[row], scale = a.scale ? a.scale[row] : 1.f;
    flag = 0;
    if (!(score < INFINITY) || (a.len && a.len[row] < 0)) { flag = RS_FLAG_BADARG; return BEAM_NONE; }
    if (score == -INFINITY) return BEAM_NONE;
    if (a.last && a.eos >= 0 && a.last[row] == a.eos) return BEAM_ENDED;
    if (!(scale > 0.f && scale < INFINITY)) { flag = RS_FLAG_BADARG; return BEAM_NONE; }
    return BEAM_RUNS;
}

// ---------------------------------------------------------------- one row
// grid rows, block 1024: ln Z, then the n_out best logits one after the other
template <typename T>
__global__ void __launch_bounds__(1024) k_beam_row(BeamArgs a) {
    __shared__ float sh_m[16];
    __shared__ double sh_z[16];
    __shared__ unsigned long long sh_key[16];
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    unsigned long long *keys = a.keys + (size_t)row * a.n_out;
    unsigned int flag;
    const int what = beam_row(a, row, flag);
    if (flag && tid == 0 && a.flags) atomicOr(a.flags + row, flag);
    if (what != BEAM_RUNS) {
        for (int k = tid; k < a.n_out; k += 1024) keys[k] = 0;
        return;
    }
    const T *x = (const T *)a.logits + (size_t)row * a.stride;
    const double c = (a.scale ? a.scale[row] : 1.f) * 1.4426950408889634074;
    float m = -INFINITY;
    int bad = 0;
    for (int i = tid; i < a.vocab; i += 1024) {
        const float v = beam_logit(x, i);
        bad |= !(v < INFINITY);
        m = fmaxf(m, v);
    }
    m = wave_max(m);
    if (lane == 0) sh_m[wave] = m;
    bad = __syncthreads_or(bad);
    for (int w = 0; w < 16; ++w) m = fmaxf(m, sh_m[w]);
    if (bad || !(m > -INFINITY)) {
        if (bad && tid == 0 && a.flags) atomicOr(a.flags + row, RS_FLAG_NONFINITE);
        for (int k = tid; k < a.n_out; k += 1024) keys[k] = 0;
        return;
    }
    double z = 0.0;
    for (int i = tid; i < a.vocab; i += 1024) z += exp2_sum(((double)beam_logit(x, i) - (double)m) * c);
    for (int o = 32; o; o >>= 1) z += __shfl_xor(z, o, RS_WAVE);
    if (lane == 0) sh_z[wave] = z;
    __syncthreads();
    if (tid == 0) {
        z = 0.0;
        for (int w = 0; w < 16; ++w) z += sh_z[w];
        a.log_z[row] = log(z) + (double)m * (a.scale ? a.scale[row] : 1.f);
    }
    unsigned long long before = ~0ull;
    for (int k = 0; k < a.n_out; ++k) {
        unsigned long long best = 0;
        for (int i = tid; i < a.vocab; i += 1024) {
            const unsigned long long key = beam_key(beam_logit(x, i), i);
            if (key < before && key > best) best = key;
        }
        for (int o = 32; o; o >>= 1) { const unsigned long long u = __shfl_xor(best, o, RS_WAVE); best = u > best ? u : best; }
        __syncthreads();
        if (lane == 0) sh_key[wave] = best;
        __syncthreads();
        for (int w = 0; w < 16; ++w) best = sh_key[w] > best ? sh_key[w] : best;
        if (tid == 0) keys[k] = best;
        before = best;
        if (!best) { for (int j = k + 1 + tid; j < a.n_out; j += 1024) keys[j] = 0; break; }
    }
}

// ---------------------------------------------------------------- one group
struct BeamCandidate { double rank, value; int beam, at, token, len; };
__device__ __forceinline__ bool beam_before(const BeamCandidate &a, const BeamCandidate &b) {      // a is taken before b; beam < 0: none
    if (b.beam < 0) return a.beam >= 0;
    if (a.beam < 0) return false;
    return a.rank > b.rank || (a.rank == b.rank && (a.beam < b.beam || (a.beam == b.beam && a.at < b.at)));
}

// grid groups, block 256
__global__ void __launch_bounds__(256) k_beam_group(BeamArgs a) {
    __shared__ BeamCandidate sh[256];
    const int g = blockIdx.x, tid = threadIdx.x;
    BeamCandidate last{INFINITY, 0.0, 0, -1, 0, 0};
    float out_score = 0.f;
    int out_parent = -1, out_token = -1, out_len = 0;
    for (int k = 0; k < a.n_out; ++k) {
        BeamCandidate best{0.0, 0.0, -1, 0, 0, 0};
        for (int i = tid; i < a.n_beams * a.n_out; i += 256) {
            const int b = i / a.n_out, at = i - b * a.n_out, row = g * a.n_beams + b;
            unsigned int flag;
            const int what = beam_row(a, row, flag);
            BeamCandidate c{0.0, 0.0, -1, at, 0, 0};
            const int len = a.len ? a.len[row] : 0;
            if (what == BEAM_ENDED && at == 0) { c.beam = b; c.token = a.eos; c.value = a.score[row]; c.len = len; }
            const unsigned long long key = what == BEAM_RUNS ? a.keys[(size_t)row * a.n_out + at] : 0;
            if (key) {
                c.beam = b; c.token = key_token(key); c.len = len + 1;
                c.value = (double)a.score[row] + ((double)key_logit(key) * (a.scale ? a.scale[row] : 1.f) - a.log_z[row]);
            }
            if (c.beam < 0) continue;
            c.rank = a.alpha > 0.0 ? c.value / pow((double)max(c.len, 1), a.alpha) : c.value;
            if (beam_before(last, c) && beam_before(c, best)) best = c;
        }
        __syncthreads();
        sh[tid] = best;
        __syncthreads();
        for (int o = 128; o; o >>= 1) {
            if (tid < o && beam_before(sh[tid + o], sh[tid])) sh[tid] = sh[tid + o];
            __syncthreads();
        }
        best = sh[0];
        if (tid == k) {
            out_parent = best.beam; out_token = best.beam < 0 ? -1 : best.token; out_len = best.len;
            out_score = best.beam < 0 ? -INFINITY : (float)best.value;
        }
        if (best.beam < 0) { if (tid > k && tid < a.n_out) out_score = -INFINITY; break; }
        last = best;
    }
    __syncthreads();                                               // (outputs may be the inputs' places)
    if (tid < a.n_out) {
        const size_t o = (size_t)g * a.n_out + tid;
        a.parent[o] = out_parent; a.token[o] = out_token; a.score_out[o] = out_score;
        if (a.len_out) a.len_out[o] = out_len;
    }
}

}  // namespace rs
