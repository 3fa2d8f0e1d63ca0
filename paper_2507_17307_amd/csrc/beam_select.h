// Selection over beams and vocabulary (rs_beam_select).
//
// The continuation of beam b by token t is worth score_b + (x_t - ln Z_b), x = scale * logits, Z = sum e^x.  Neighbours in the order of a vocabulary,
// and more so across beams, may be nearer than fp32 sums can tell, so the sum of exponentials and all that is compared across beams are double; within a
// row the order is that of the logits themselves.  The scores that go from call to call are double or fp32, as the caller holds them: fp32 ones are rounded
// once a call, which adds up over a search.
//
// k_beam_scan makes one pass over the logits.  A wave takes 1024 of them at a time, 16 a lane: their exponentials go into its sum, the largest of each lane's 16
// into LDS.  After eight batches it sets a border that n_out of its values at least reach, from what the lanes had as their largest, and only lanes
// with something at or above it read their 16 values again (from the cache) and put those into a short list of the wave in LDS; a list that fills up is cut to
// its n_out best.  The workgroup joins its waves' lists and leaves n_out keys and a sum; k_beam_join joins those of a group.  Lists are ordered
// by counting, for each member, how many come before it.
#pragma once

#include <cfloat>

#include "beam_plan.h"
#include "device_utils.h"
#include "../../include/rstitch.h"

namespace rs {

struct BeamSum { double z; float m; int bad; };                    // sum of 2^((x - m) c) over what was seen, its largest logit, NaN or +inf seen

struct BeamArgs {
    const void *logits; size_t stride;
    const float *scale;
    const void *score;                                             // double if `wide`, else float; so is score_out
    const int *last, *len;
    int eos, n_beams, vocab, n_out, parts;                         // parts * n_beams * n_out <= BEAM_KEYS
    double alpha;
    int *parent, *token, *len_out;
    void *score_out;
    int wide;                                                      // 0 or 1
    unsigned int *flags;
    unsigned long long *keys;                                      // [row][part][n_out]; 0: none
    BeamSum *sums;                                                 // [row][part]
    double *scores;                                                // [row]: as double, whatever the caller's are
};

// 2^f for |f| <= 1/2, to 1.1e-12: degree eight through 2^f at the nine Chebyshev nodes, of which 0 is one.  2^0 is exactly 1, so that a token that makes up
// the whole sum has log probability 0, and equal scores stay equal.  Scores nearer than ln Z's error may change places.  (Degree seven through 1 at 0 is off
// by 1.1e-10: a call on 128 rows of 152064 fp32 logits takes 28.6 us in the place of 29.2.)
__device__ __forceinline__ double exp2_part(double f) {
    double p = 1.3255224887502117e-06;
    p = fma(p, f, 1.531007940254368e-05); p = fma(p, f, 0.0001540345585240991); p = fma(p, f, 0.0013333450567999414); p = fma(p, f, 0.009618129159402628);
    p = fma(p, f, 0.05550410941205934); p = fma(p, f, 0.2402265069581299); p = fma(p, f, 0.6931471805459335); return fma(p, f, 1.0);
}
// p 2^n, p in [0.7, 1.5] and |n| <= 1020: n goes into the exponent
__device__ __forceinline__ double scale_exp(double p, int n) { return __hiloint2double(__double2hiint(p) + (n << 20), __double2loint(p)); }
// Adding this to a number below 2^30 leaves the nearest integer in the low word of the sum.
constexpr double TO_INT = 6755399441055744.0;                      // 1.5 2^52

// 2^d for d <= 1; below 2^-1000 it is 2^-1000.
__device__ __forceinline__ double exp2_sum(double d) {
    d = fmax(d, -1000.0);
    const double s = d + TO_INT;
    return scale_exp(exp2_part(d - (s - TO_INT)), __double2loint(s));
}

// A logit and its token as one number: larger for a larger logit, and for a lower token among equals (-0 and 0 are equal).  0: no candidate.
__device__ __forceinline__ uint32_t beam_order(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ unsigned long long beam_key(float x, int token) {
    return x > -INFINITY ? (unsigned long long)beam_order(x) << 32 | (uint32_t)~token : 0;
}
constexpr uint32_t ORDER_OF_MINUS_INF = 0x007fffffu;
__device__ __forceinline__ float order_logit(uint32_t o) { return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ float key_logit(unsigned long long key) { return order_logit((uint32_t)(key >> 32)); }
__device__ __forceinline__ int key_token(unsigned long long key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ unsigned long long double_order(double x) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double order_double(unsigned long long o) { return __longlong_as_double((long long)(o >> 63 ? o & ~(1ull << 63) : ~o)); }

// Exchanges inside rows of 16 lanes as operands of DPP moves (device_utils.h), step 0 .. 3: with the lane one, two, four and eight away or its mirror image, which
// has the same value by then.
template <int STEP>
__device__ __forceinline__ int row_move(int v) {
    constexpr int CTRL = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 : 0x140;
    return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false);
}
template <int STEP> __device__ __forceinline__ uint32_t row_move(uint32_t v) { return (uint32_t)row_move<STEP>((int)v); }
template <int STEP> __device__ __forceinline__ float row_move(float v) { return __int_as_float(row_move<STEP>(__float_as_int(v))); }
template <int STEP> __device__ __forceinline__ double row_move(double v) { return __hiloint2double(row_move<STEP>(__double2hiint(v)), row_move<STEP>(__double2loint(v))); }
__device__ __forceinline__ int lane_of(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ double lane_of(double v, int lane) { return __hiloint2double(lane_of(__double2hiint(v), lane), lane_of(__double2loint(v), lane)); }

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
    v = max(v, row_move<0>(v)); v = max(v, row_move<1>(v)); v = max(v, row_move<2>(v)); v = max(v, row_move<3>(v));
    return max(max(lane_of(v, 0), lane_of(v, 16)), max(lane_of(v, 32), lane_of(v, 48)));
}
__device__ __forceinline__ double wave_sum_f64(double v) {
    v += row_move<0>(v); v += row_move<1>(v); v += row_move<2>(v); v += row_move<3>(v);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
// f over the 2^shift lanes of each lane's group
template <typename T, typename F>
__device__ __forceinline__ T group_all(T v, int shift, F f) {
    if (shift > 0) v = f(v, row_move<0>(v));
    if (shift > 1) v = f(v, row_move<1>(v));
    if (shift > 2) v = f(v, row_move<2>(v));
    if (shift > 3) v = f(v, row_move<3>(v));
    if (shift > 4) v = f(v, __shfl_xor(v, 16, RS_WAVE));
    if (shift > 5) v = f(v, __shfl_xor(v, 32, RS_WAVE));
    return v;
}

// What a row takes part with: its vocabulary, its end, or nothing.
enum { BEAM_NONE, BEAM_ENDED, BEAM_RUNS };
struct BeamRow { double score; float scale; int last, len; };
__device__ __forceinline__ double beam_score(const BeamArgs &a, int row) {
    // (both words of a double are asked for at once, which for a float are one and the same: no branch before the load)
    const int *word = (const int *)a.score + ((size_t)row << a.wide);
    const int low = word[0], high = word[a.wide];
    return a.wide ? __hiloint2double(high, low) : (double)__int_as_float(low);
}
__device__ __forceinline__ BeamRow beam_row(const BeamArgs &a, int row, double score) {
    return {score, a.scale ? a.scale[row] : 1.f, a.last ? a.last[row] : -2, a.len ? a.len[row] : 0};
}
__device__ __forceinline__ int beam_kind(const BeamRow &r, int eos, unsigned int &flag) {
    flag = 0;
    if (!(r.score < INFINITY) || r.len < 0 || r.len == 0x7fffffff) { flag = RS_FLAG_BADARG; return BEAM_NONE; }
    if (r.score == -INFINITY) return BEAM_NONE;
    if (eos >= 0 && r.last == eos) return BEAM_ENDED;
    if (!(r.scale > 0.f && r.scale < INFINITY)) { flag = RS_FLAG_BADARG; return BEAM_NONE; }
    return BEAM_RUNS;
}

// An order that at least `keep` of 128 reach, two a lane, keep <= 64; ORDER_OF_MINUS_INF if so many are not above that.
// The lanes in 2^k >= keep groups: the least of the groups' largest, 6 steps across lanes.  Of random numbers keep (ln keep + 0.6) reach that;
// beyond eight, or where a group has nothing, halving the way to the largest brings it nearer to keep.
__device__ __forceinline__ uint32_t wave_border(uint32_t x, uint32_t y, int keep) {
    const int lanes = keep > 32 ? 0 : keep > 16 ? 1 : keep > 8 ? 2 : keep > 4 ? 3 : keep > 2 ? 4 : keep > 1 ? 5 : 6;      // log2 of a group's lanes
    uint32_t t = max(x, y), m = t;
    auto step = [&](bool group, uint32_t other_t, uint32_t other_m) { t = group ? max(t, other_t) : min(t, other_t); m = max(m, other_m); };
    step(lanes > 0, row_move<0>(t), row_move<0>(m)); step(lanes > 1, row_move<1>(t), row_move<1>(m));
    step(lanes > 2, row_move<2>(t), row_move<2>(m)); step(lanes > 3, row_move<3>(t), row_move<3>(m));
    auto join = [](uint32_t v, bool sixteen, bool thirty_two) {    // (four rows of 16 lanes; true: the larger)
        const uint32_t a = lane_of(v, 0), b = lane_of(v, 16), c = lane_of(v, 32), d = lane_of(v, 48);
        const uint32_t e = sixteen ? max(a, b) : min(a, b), f = sixteen ? max(c, d) : min(c, d);
        return thirty_two ? max(e, f) : min(e, f);
    };
    uint32_t lo = join(t, lanes > 4, lanes > 5);
    const int halvings = lo <= ORDER_OF_MINUS_INF ? 20 : keep > 8 ? 8 : 0;
    if (halvings > 0) {
        uint32_t hi = join(m, true, true) + 1;
#pragma unroll 1
        for (int k = 0; k < halvings; ++k) {
            const uint32_t mid = lo + (hi - lo) / 2;
            const bool enough = (int)__popcll(__ballot(x >= mid)) + (int)__popcll(__ballot(y >= mid)) >= keep;
            lo = enough ? mid : lo; hi = enough ? hi : mid;
        }
    }
    return lo;
}

// Lane's place among the wave's lanes with `in`, behind *count, which it moves on: one addition for the wave.
__device__ __forceinline__ int wave_place(bool in, int *count) {
    const unsigned long long who = __ballot(in);
    if (!who) return 0;
    int base = 0;
    if ((threadIdx.x & 63) == 0) base = atomicAdd(count, (int)__popcll(who));
    return __builtin_amdgcn_readfirstlane(base) + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
}

// ---------------------------------------------------------------- a wave's list
constexpr int BEAM_LIST = 256;

// Keys above `floor`, of which it has to keep so many (once it was cut, floor is the last of those).
struct WaveList {
    unsigned long long *keys, *spare, floor;                       // spare: room for `keep` keys
    int n, keep;

    __device__ __forceinline__ void cut() {
        const int lane = threadIdx.x & 63;
#pragma unroll 1
        for (int i = lane; i < n; i += 64) {
            const unsigned long long mine = keys[i];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) rank += keys[j] > mine;
            if (rank < keep) spare[rank] = mine;
        }
        __builtin_amdgcn_wave_barrier();
        if (n > keep) n = keep;
        if (lane < n) keys[lane] = spare[lane];
        __builtin_amdgcn_wave_barrier();
        if (n == keep) floor = keys[keep - 1];
    }
    __device__ __forceinline__ void push(unsigned long long key) {
        bool in = key > floor;
        unsigned long long who = __ballot(in);
        if (!who) return;
        if (n + (int)__popcll(who) > BEAM_LIST) {
            cut();
            in = key > floor;
            who = __ballot(in);
        }
        if (in) keys[n + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] = key;
        n += (int)__popcll(who);
    }
};

// ---------------------------------------------------------------- a wave's sum
// Batches whose logits are of an ordinary size are added up as sum 2^(x c - r) for one integer r of the wave, near the largest of its first batch: x c is
// rounded to n, which goes into the exponent, and x c - n is exact in one operation (14 double instructions a logit; counted from the largest logit met so
// far, with its rescaling, 17).  What is 2^1000 times smaller is raised to that.  Other batches, logits beyond 4096 and what towers 2^500 above r, are added
// up by the lanes from their largest.
struct WaveSum {
    double c, z, lane_z;                                           // z: with r; lane_z: with lane_m
    float lane_m, low, high;
    int r;
    bool bad, ready;

    __device__ __forceinline__ void init(float scale) {
        c = (double)scale * 1.4426950408889634074;
        z = lane_z = 0.0; lane_m = low = high = -INFINITY; r = 0; bad = ready = false;
    }
    __device__ __forceinline__ void add(const float (&v)[16], float top) {
        if (!ready) {
            const float m = wave_max(top);
            const double x = (double)m * c;
            if (fabs(x) < 4096.0) {
                r = (int)__builtin_rint(x);
                low = (float)((double)(r - 1000) / c); high = (float)((double)(r + 500) / c);
                ready = low > -INFINITY;                           // (scales under 2^-115 or so: nothing is 2^1000 smaller but masked logits, which the lanes drop)
            }
        }
        if (ready && !__any(top > high)) {
            const double shift = TO_INT - (double)r;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const double x = (double)__builtin_amdgcn_fmed3f(v[k], low, INFINITY), s = fma(x, c, shift);       // (a maximum that takes NaN as it is)
                z += scale_exp(exp2_part(fma(x, c, shift - s)), __double2loint(s));
            }
        } else {
            if (top > lane_m) { lane_z = lane_m > -INFINITY ? lane_z * exp2_sum(((double)lane_m - (double)top) * c) : 0.0; lane_m = top; }
            const double from = lane_m > -INFINITY ? (double)lane_m : 0.0;         // (nothing but masked logits so far: their 2^-1000 are dropped)
#pragma unroll
            for (int k = 0; k < 16; ++k) lane_z += exp2_sum(((double)v[k] - from) * c);
        }
    }
    // the wave's largest logit among those added, given the largest of each lane; z then counts from it
    __device__ __forceinline__ float finish(float lane_top) {
        const float top = wave_max(lane_top);
        double all = lane_m > -INFINITY ? lane_z * exp2_sum(((double)lane_m - (double)top) * c) : 0.0;
        if (ready && top > -INFINITY) all += z * exp2_sum((double)r - (double)top * c);
        z = wave_sum_f64(all);
        return top;
    }
};

// How many of m numbers are above `mine`, and how many equal it.  x: in LDS, 16-byte aligned, with zeros up to a multiple of eight.
__device__ __forceinline__ void count_before(const uint32_t *x, int m, uint32_t mine, int &above, int &equal) {
#pragma unroll 1
    for (int j = 0; j < m; j += 8) {
        const uint4 a = *reinterpret_cast<const uint4 *>(x + j), b = *reinterpret_cast<const uint4 *>(x + j + 4);
        const uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int k = 0; k < 8; ++k) { above += v[k] > mine; equal += v[k] == mine; }
    }
}

// How many of m keys are above hi:lo.  Their halves: in LDS, 16-byte aligned, with zeros up to a multiple of eight.  (Whole keys, since
// bf16 logits have many equal upper halves.)
__device__ __forceinline__ int count_keys_before(const uint32_t *high, const uint32_t *low, int m, uint32_t hi, uint32_t lo) {
    const unsigned long long mine = (unsigned long long)hi << 32 | lo;
    int rank = 0;
#pragma unroll 1
    for (int j = 0; j < m; j += 8) {
        const uint4 a = *reinterpret_cast<const uint4 *>(high + j), b = *reinterpret_cast<const uint4 *>(high + j + 4);
        const uint4 c = *reinterpret_cast<const uint4 *>(low + j), d = *reinterpret_cast<const uint4 *>(low + j + 4);
        const uint32_t h[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}, l[8] = {c.x, c.y, c.z, c.w, d.x, d.y, d.z, d.w};
#pragma unroll
        for (int k = 0; k < 8; ++k) rank += ((unsigned long long)h[k] << 32 | l[k]) > mine;
    }
    return rank;
}

// f(j) for those that equal it.
template <typename F>
__device__ __forceinline__ void for_equal(const uint32_t *x, int m, uint32_t mine, F f) {
#pragma unroll 1
    for (int j = 0; j < m; j += 8) {
        const uint4 a = *reinterpret_cast<const uint4 *>(x + j), b = *reinterpret_cast<const uint4 *>(x + j + 4);
        const uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        uint32_t which = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) which |= (uint32_t)(v[k] == mine) << k;
        for (; which; which &= which - 1) f(j + __ffs(which) - 1);
    }
}

// A number that `keep` and few more of the workgroup's reach (all of them, if there are fewer): down from the largest, `most`, in growing steps, then what lies
// between is divided, four numbers at a time, since each time costs a barrier.  Zeros are none.
constexpr int BORDER_SLACK = 24;                                   // more than `keep` that are not worth another step
constexpr int BORDER_AT_ONCE = 4;
// three times down (2^16, 2^18 .. 2^30, all); then w -> w / 5 + 4 at most, 32 bits in 14 times, and 5 -> 1
constexpr int BORDER_COUNTS = BORDER_AT_ONCE * (3 + 14 + 4);
constexpr int SCAN_SHORT = 96;                                     // keys beyond n_out that are ordered without such a search
template <int N>
__device__ __forceinline__ uint32_t block_border(const uint32_t (&x)[N], uint32_t most, int keep, int *counts) {      // counts: BORDER_COUNTS zeros in LDS, 16-byte aligned
    const int lane = threadIdx.x & 63;
    auto reach = [&](const uint32_t (&t)[BORDER_AT_ONCE], int (&r)[BORDER_AT_ONCE]) __attribute__((always_inline)) {
        int mine = 0;
#pragma unroll
        for (int q = 0; q < BORDER_AT_ONCE; ++q) {
            int c = 0;
#pragma unroll
            for (int k = 0; k < N; ++k) c += (int)__popcll(__ballot(x[k] >= t[q]));
            mine = lane == q ? c : mine;
        }
        if (lane < BORDER_AT_ONCE) atomicAdd(&counts[lane], mine);
        __syncthreads();
        const int4 c = *reinterpret_cast<const int4 *>(counts);
        r[0] = c.x; r[1] = c.y; r[2] = c.z; r[3] = c.w;
        counts += BORDER_AT_ONCE;
    };
    uint32_t border = 1, above = most;
    int reached = -1;
    if (most == 0) return 1;
#pragma unroll 1
    for (int d = 16; reached < 0; d += 2 * BORDER_AT_ONCE) {
        uint32_t t[BORDER_AT_ONCE];
        int r[BORDER_AT_ONCE];
#pragma unroll
        for (int q = 0; q < BORDER_AT_ONCE; ++q) t[q] = d + 2 * q < 32 && most > 1u << (d + 2 * q & 31) ? most - (1u << (d + 2 * q & 31)) : 1;
        reach(t, r);
#pragma unroll
        for (int q = 0; q < BORDER_AT_ONCE; ++q) {
            if (reached >= 0) continue;
            if (r[q] >= keep || t[q] == 1) { border = t[q]; reached = r[q]; } else above = t[q];
        }
    }
#pragma unroll 1
    while (reached > keep + BORDER_SLACK && above - border > 1) {
        const uint32_t step = max((above - border) / (BORDER_AT_ONCE + 1), 1u), last = above - 1;
        uint32_t t[BORDER_AT_ONCE];
        int r[BORDER_AT_ONCE];
#pragma unroll
        for (int q = 0; q < BORDER_AT_ONCE; ++q) t[q] = min(border + (q + 1) * step, last);
        reach(t, r);
#pragma unroll
        for (int q = BORDER_AT_ONCE - 1; q >= 0; --q) {
            if (r[q] < keep) above = t[q];
            else { border = t[q]; reached = r[q]; break; }
        }
    }
    return border;
}

// ---------------------------------------------------------------- a wave's batch
template <typename T> struct BeamUnit;                             // a piece of 16 bytes
template <> struct BeamUnit<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float value(const u32x4_t &q, int i) { return __uint_as_float(q[i]); }
    static __device__ __forceinline__ float one(const float *p) { return *p; }
};
template <> struct BeamUnit<uint16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float value(const u32x4_t &q, int i) { return i & 1 ? bf16_hi(q[i / 2]) : bf16_lo(q[i / 2]); }
    static __device__ __forceinline__ float one(const uint16_t *p) { return bf16_to_f32(*p); }
};

constexpr int BEAM_ROUND = 8;                                      // batches between two looks for candidates

struct ScanShared {
    union {
        unsigned long long list[BEAM_WAVES][BEAM_LIST];
        struct { uint32_t order[BEAM_WAVES * BEAM_LIST + 8], rest[BEAM_WAVES * BEAM_LIST + 8]; } kept;
    };
    union { float of[BEAM_ROUND][64]; unsigned long long spare[BEAM_MAX]; } top[BEAM_WAVES];
    double z[BEAM_WAVES];
    float m[BEAM_WAVES];
    uint32_t border[BEAM_WAVES];
    int bad[BEAM_WAVES], count[BEAM_WAVES], n;
    alignas(16) int counts[BORDER_COUNTS];
};

// grid (parts, rows), block BEAM_THREADS.  Two borders near each other: the 78 MB of 128 rows of 152064 fp32 logits take 12.4 us as a streaming read (6.3 TB/s), and
// some 25 vector operations a logit, 14 of them in double, four cycles each, 12 us.  25 us measured (3.1 TB/s).  The whole call takes
// 29.7 us, 25.1 without candidates and 20.4 without candidates and exponentials: the parts add up, since the workgroups of the one round there is start, read and end
// together.  bf16 with 32 candidates of 384 rows, a sixth of them ended: 74 us, 58 and 30.
template <typename T>
__global__ void __launch_bounds__(BEAM_THREADS) k_beam_scan(BeamArgs a) {
    constexpr int UNIT = BeamUnit<T>::N, PIECES = 16 / UNIT, WAVE_UNITS = 64 * PIECES;
    __shared__ ScanShared sh;
    const int row = blockIdx.y, part = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const BeamRow r = beam_row(a, row, beam_score(a, row));
    unsigned int flag;
    if (part == 0 && tid == 0) a.scores[row] = r.score;
    const int kind = beam_kind(r, a.eos, flag);
    if (flag && part == 0 && tid == 0 && a.flags) atomicOr(a.flags + row, flag);
    if (kind != BEAM_RUNS) return;
    const T *x = (const T *)a.logits + (size_t)row * a.stride;
    const BeamShare share = beam_share((int)((uintptr_t)x % 16), (int)sizeof(T), a.vocab, a.parts, part, wave);
    const int before = share.before, ends = share.ends, unit_0 = share.unit_0, unit_end = share.unit_end, unit_a = unit_0 + lane;
    const u32x4_t *px = reinterpret_cast<const u32x4_t *>(x + before);
    WaveSum sum;
    sum.init(r.scale);
    WaveList list{sh.list[wave], sh.top[wave].spare, 0, 0, a.n_out};
    uint32_t border = 0;
    float v[16], least = -FLT_MAX, lo_top = -INFINITY, hi_top = -INFINITY;
    const int whole = (unit_end - unit_0 + WAVE_UNITS - 1) / WAVE_UNITS, n_batches = whole + (ends > 0);      // (the single values: a batch of their own, one a lane)
    const int end_token = beam_end_token(share, lane);
    const float end_value = lane < ends ? BeamUnit<T>::one(x + end_token) : -INFINITY;
    // this lane's pieces of batch b < whole, and their values
    auto fetch = [&](int b, u32x4_t (&w)[PIECES]) __attribute__((always_inline)) {
        const int u0 = unit_a + b * WAVE_UNITS;
#pragma unroll
        for (int j = 0; j < PIECES; ++j) w[j] = px[min(u0 + 64 * j, unit_end - 1)];
    };
    auto values = [&](int b, const u32x4_t (&w)[PIECES], float (&x16)[16]) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 16; ++k) x16[k] = BeamUnit<T>::value(w[k / UNIT], k % UNIT);
        if (unit_0 + (b + 1) * WAVE_UNITS > unit_end) {
            const int u0 = unit_a + b * WAVE_UNITS;
#pragma unroll
            for (int k = 0; k < 16; ++k) x16[k] = u0 + 64 * (k / UNIT) < unit_end ? x16[k] : -INFINITY;
        }
    };
    u32x4_t next[PIECES];                                          // under way while a batch is added up (two batches ahead was no faster)
    if (whole > 0) fetch(0, next);
    for (int b0 = 0; b0 < n_batches; b0 += BEAM_ROUND) {
        const int n_round = min(BEAM_ROUND, n_batches - b0);
        float best = -INFINITY;
        for (int b = b0; b < b0 + n_round; ++b) {
            if (b < whole) {
                values(b, next, v);
                if (b + 1 < whole) fetch(b + 1, next);
            } else {
#pragma unroll
                for (int k = 1; k < 16; ++k) v[k] = -INFINITY;
                v[0] = end_value;
            }
            float lo = v[0], hi = v[UNIT];                         // (of every other piece: a short batch has some in each)
#pragma unroll
            for (int k = 1; k < 16; ++k) { if (k / UNIT % 2 == 0) lo = fmaxf(lo, v[k]); else if (k != UNIT) hi = fmaxf(hi, v[k]); }
            const float top = fmaxf(lo, hi);
            lo_top = fmaxf(lo_top, lo); hi_top = fmaxf(hi_top, hi); best = fmaxf(best, top);
            sh.top[wave].of[b - b0][lane] = top;
#pragma unroll
            for (int k = 0; k < 16; k += 2) sum.bad |= __builtin_isunordered(v[k], v[k + 1]);
            sum.add(v, top);
        }
        if (__any(best >= least)) {
            border = max(border, wave_border(beam_order(lo_top), beam_order(hi_top), a.n_out));
            least = border > ORDER_OF_MINUS_INF ? order_logit(border) : -FLT_MAX;
            uint32_t in = 0;                                       // the lane's batches with something to take
            for (int k = 0; k < n_round; ++k) in |= (uint32_t)(sh.top[wave].of[k][lane] >= least) << k;
#pragma unroll 1
            while (__any(in != 0)) {
                const int b = b0 + __ffs(in) - 1;                  // (the last one is still there)
                float w[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) w[k] = v[k];
                if (in && b != b0 + n_round - 1) { u32x4_t again[PIECES]; fetch(b, again); values(b, again, w); }
                uint32_t which = 0;
#pragma unroll
                for (int k = 0; k < 16; ++k) which |= (uint32_t)(w[k] >= least) << k;
                if (!in) which = 0;
                const int first = b < whole ? before + (unit_a + b * WAVE_UNITS) * UNIT : end_token;
#pragma unroll 1
                while (__any(which != 0)) {                        // a lane's next one
                    const int k = __ffs(which) - 1;
                    // (chosen by bits: a choice between two elements of an array becomes one between their addresses)
                    const uint32_t eight = 0u - (k >> 3 & 1), four = 0u - (k >> 2 & 1), two = 0u - (k >> 1 & 1), one = 0u - (k & 1);
                    uint32_t q[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) q[e] = (__float_as_uint(w[8 + e]) & eight) | (__float_as_uint(w[e]) & ~eight);
#pragma unroll
                    for (int e = 0; e < 4; ++e) q[e] = (q[4 + e] & four) | (q[e] & ~four);
                    q[0] = (q[2] & two) | (q[0] & ~two); q[1] = (q[3] & two) | (q[1] & ~two);
                    list.push(which ? beam_key(__uint_as_float((q[1] & one) | (q[0] & ~one)), first + (k / UNIT) * (64 * UNIT) + k % UNIT) : 0);
                    which &= which - 1;
                }
                in &= in - 1;
            }
        }
    }
    const float lane_top = fmaxf(lo_top, hi_top);
    // ---- the waves' sums and lists
    const float top = sum.finish(lane_top);
    const int bad = __any(sum.bad || !(lane_top < INFINITY));
    if (lane == 0) { sh.z[wave] = sum.z; sh.m[wave] = top; sh.bad[wave] = bad; sh.count[wave] = list.n; sh.border[wave] = border; }
    if (tid < BORDER_COUNTS) sh.counts[tid] = 0;
    if (tid == 0) sh.n = 0;
    __syncthreads();
    if (tid == 0) {
        float m = sh.m[0];
        int any = sh.bad[0];
#pragma unroll
        for (int w = 1; w < BEAM_WAVES; ++w) { m = fmaxf(m, sh.m[w]); any |= sh.bad[w]; }
        double all = 0.0;
#pragma unroll 1
        for (int w = 0; w < BEAM_WAVES; ++w) all += sh.m[w] > -INFINITY && !any ? sh.z[w] * exp2_sum(((double)sh.m[w] - (double)m) * sum.c) : 0.0;
        a.sums[(size_t)row * a.parts + part] = {all, m, any};
    }
    unsigned long long mine[BEAM_LIST / 64];
    uint32_t order[BEAM_LIST / 64], most = 0, least_kept = 1;
    int total = 0;
#pragma unroll
    for (int w = 0; w < BEAM_WAVES; ++w) { total += sh.count[w]; most = max(most, sh.m[w] > -INFINITY ? beam_order(sh.m[w]) : 0u); least_kept = max(least_kept, sh.border[w]); }
#pragma unroll
    for (int k = 0; k < BEAM_LIST / 64; ++k) {
        mine[k] = lane + 64 * k < list.n ? list.keys[lane + 64 * k] : 0;
        order[k] = (uint32_t)(mine[k] >> 32);
    }
    // (n_out keys at least reach each of the waves' borders, so the highest of them does for short lists)
    if (total > a.n_out + SCAN_SHORT) least_kept = block_border(order, most, a.n_out, sh.counts);
    __syncthreads();
    unsigned long long *to = a.keys + ((size_t)row * a.parts + part) * a.n_out;
#pragma unroll
    for (int k = 0; k < BEAM_LIST / 64; ++k) {
        const bool in = order[k] >= least_kept;
        const int at = wave_place(in, &sh.n);
        if (in) { sh.kept.order[at] = order[k]; sh.kept.rest[at] = (uint32_t)mine[k]; }
    }
    __syncthreads();
    const int m = sh.n;
    if (tid < 8) sh.kept.order[m + tid] = sh.kept.rest[m + tid] = 0;
    __syncthreads();
    for (int i = tid; i < m; i += BEAM_THREADS) {
        const uint32_t order = sh.kept.order[i], rest = sh.kept.rest[i];
        const int rank = m <= a.n_out ? i : count_keys_before(sh.kept.order, sh.kept.rest, m, order, rest);      // (few: in any order)
        if (rank < a.n_out) to[rank] = (unsigned long long)order << 32 | rest;
    }
    for (int k = m + tid; k < a.n_out; k += BEAM_THREADS) to[k] = 0;
}

// ---------------------------------------------------------------- the join of a group
constexpr int JOIN_EACH = 4;                                       // keys a thread
constexpr int JOIN_KEPT = 1024;                                    // items that are kept for ordering

struct alignas(16) JoinRow { double score, top, z, div; float scale; int kind, len; };      // (side by side: three reads of 16 bytes an item)

struct JoinShared {
    uint32_t high[JOIN_KEPT + 8];                                  // upper halves of the values
    unsigned long long value[JOIN_KEPT], key[JOIN_KEPT], edge_value, edge_key;
    uint32_t beam[JOIN_KEPT], edge_beam, most;
    alignas(16) int counts[BORDER_COUNTS];
    JoinRow row[BEAM_MAX];
    int n;
};

// The order of items: larger values first, of equals the lower beam, in one beam the larger key.
__device__ __forceinline__ bool item_before(unsigned long long v, uint32_t b, unsigned long long k, unsigned long long v2, uint32_t b2, unsigned long long k2) {
    return v > v2 || (v == v2 && (b < b2 || (b == b2 && k > k2)));
}

// grid groups, block 256, 512 or 1024: JOIN_EACH keys a thread.  Bound by the chain of its steps (keys and sums, logarithm, values, border, order): 5.8 us of 608 to
// 1024 keys a group, 11 of 2560.
__global__ void __launch_bounds__(1024) k_beam_join(BeamArgs a) {
    __shared__ JoinShared sh;
    const int g = blockIdx.x, tid = threadIdx.x, threads = blockDim.x, lane = tid & 63, parts = a.parts;
    const int per_row = parts * a.n_out, n = a.n_beams * per_row;
    const unsigned long long *keys = a.keys + (size_t)g * a.n_beams * per_row;
    unsigned long long value[JOIN_EACH], key[JOIN_EACH];
#pragma unroll
    for (int k = 0; k < JOIN_EACH; ++k) key[k] = tid + threads * k < n ? keys[tid + threads * k] : 0;      // (of rows that do not run: anything)
    // ---- ln Z of the rows: as many lanes a row as it has parts, up to the next power of two
    const int shift = parts <= 1 ? 0 : 32 - __clz(parts - 1), rows_at_once = threads >> shift, sub = lane & ((1 << shift) - 1);
    for (int b0 = 0; b0 < a.n_beams; b0 += rows_at_once) {
        const int b = b0 + (tid >> shift), row = g * a.n_beams + min(b, a.n_beams - 1);
        const BeamRow r = beam_row(a, row, a.scores[row]);
        const BeamSum s = a.sums[(size_t)row * parts + min(sub, parts - 1)];       // (of rows that do not run: anything)
        unsigned int flag;
        int kind = beam_kind(r, a.eos, flag);
        const bool has = kind == BEAM_RUNS && sub < parts;
        const float m = has ? s.m : -INFINITY, top = group_all(m, shift, [](float x, float y) { return fmaxf(x, y); });
        const int bad = group_all(has ? s.bad : 0, shift, [](int x, int y) { return x | y; });
        const double z = group_all(m > -INFINITY ? s.z * exp2_sum(((double)m - (double)top) * ((double)r.scale * 1.4426950408889634074)) : 0.0, shift,
                                   [](double x, double y) { return x + y; });
        if (sub == 0 && b < a.n_beams) {
            if (bad && a.flags) atomicOr(a.flags + row, RS_FLAG_NONFINITE);
            if (kind == BEAM_RUNS && (bad || !(top > -INFINITY))) kind = BEAM_NONE;
            const int len = r.len + (kind == BEAM_RUNS);
            sh.row[b] = {r.score, kind == BEAM_RUNS ? (double)top * (double)r.scale : 0.0, kind == BEAM_RUNS ? z : 1.0, 1.0, r.scale, kind, len};
        }
    }
    if (tid == 0) { sh.n = 0; sh.most = 0; }
    if (tid < BORDER_COUNTS) sh.counts[tid] = 0;
    __syncthreads();
    // ln Z = ln z + top.  With double scores top is taken from a logit first, so that ln z is kept however large the logits are; with fp32 scores ln Z is one
    // double, in which ln z is off by 2^-53 of top: less than their own rounding for logits up to 2^29 times the score.
    if (tid < a.n_beams) {
        const double top = sh.row[tid].top, ln_z = log(sh.row[tid].z);
        sh.row[tid].top = a.wide ? top : 0.0;
        sh.row[tid].z = a.wide ? ln_z : ln_z + top;
        if (a.alpha > 0.0) sh.row[tid].div = pow((double)max(sh.row[tid].len, 1), a.alpha);
    }
    __syncthreads();
    auto worth = [](const JoinRow &r, unsigned long long item) __attribute__((always_inline)) {
        const double v = r.score + (((double)key_logit(item) * (double)r.scale - r.top) - r.z);
        return r.kind == BEAM_RUNS ? v : r.score;
    };
    // ---- the items' values
    unsigned long long best = 0;
#pragma unroll
    for (int k = 0; k < JOIN_EACH; ++k) {
        const int i = tid + threads * k, b = min(i / per_row, a.n_beams - 1);
        const JoinRow r = sh.row[b];
        const int kind = i < n ? r.kind : BEAM_NONE;
        value[k] = 0;
        const double v = worth(r, key[k]);
        if (kind == BEAM_ENDED) key[k] = i == b * per_row ? 1ull << 32 | (uint32_t)~a.eos : 0;
        if (kind != BEAM_NONE && key[k]) value[k] = double_order(a.alpha > 0.0 ? v / r.div : v);
        best = value[k] > best ? value[k] : best;
    }
    const uint32_t wave_most = wave_max_u32((uint32_t)(best >> 32));
    if (lane == 0) atomicMax(&sh.most, wave_most);
    __syncthreads();
    uint32_t high[JOIN_EACH];
#pragma unroll
    for (int k = 0; k < JOIN_EACH; ++k) high[k] = (uint32_t)(value[k] >> 32);
    const uint32_t border = block_border(high, sh.most, a.n_out, sh.counts);
    auto keep = [&](int k, bool in) __attribute__((always_inline)) {
        const int at = wave_place(in, &sh.n);
        if (in && at < JOIN_KEPT) { sh.high[at] = (uint32_t)(value[k] >> 32); sh.value[at] = value[k]; sh.key[at] = key[k]; sh.beam[at] = (tid + threads * k) / per_row; }
    };
#pragma unroll
    for (int k = 0; k < JOIN_EACH; ++k) keep(k, value[k] && (uint32_t)(value[k] >> 32) >= border);
    __syncthreads();
    if (sh.n > JOIN_KEPT) {
        // more than a thousand equals: the border is the n_out-th of the threads' first items, which leaves items of n_out threads
        unsigned long long v = 0, x = 0;
        uint32_t b = 0;
#pragma unroll
        for (int k = 0; k < JOIN_EACH; ++k) {
            const uint32_t bk = (tid + threads * k) / per_row;
            if (value[k] && (!v || item_before(value[k], bk, key[k], v, b, x))) { v = value[k]; x = key[k]; b = bk; }
        }
        __syncthreads();
        sh.value[tid] = v; sh.key[tid] = x; sh.beam[tid] = b;
        if (tid == 0) { sh.n = 0; sh.edge_value = 0; sh.edge_key = 0; sh.edge_beam = 0; }
        __syncthreads();
        int rank = 0;
        for (int j = 0; j < threads; ++j) rank += item_before(sh.value[j], sh.beam[j], sh.key[j], v, b, x);
        if (v && rank == a.n_out - 1) { sh.edge_value = v; sh.edge_key = x; sh.edge_beam = b; }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < JOIN_EACH; ++k)
            keep(k, value[k] && !item_before(sh.edge_value, sh.edge_beam, sh.edge_key, value[k], (tid + threads * k) / per_row, key[k]));
        __syncthreads();
    }
    // ---- in order (all rows were read: outputs may be their places)
    const size_t o = (size_t)g * a.n_out;
    const int m = sh.n;
    if (tid < 8) sh.high[m + tid] = 0;
    __syncthreads();
    for (int i = tid; i < m; i += threads) {
        const unsigned long long v = sh.value[i], x = sh.key[i];
        const uint32_t b = sh.beam[i], high = sh.high[i];
        int rank = 0, equal = 0;
        count_before(sh.high, m, high, rank, equal);
        if (equal > 1)
            for_equal(sh.high, m, high, [&](int j) { rank += item_before(sh.value[j], sh.beam[j], sh.key[j], v, b, x); });
        if (rank < a.n_out) {
            // (where lengths count: not the quotient times the divisor, so that an ended beam's score stays as it is, bit by bit)
            const double score = a.alpha > 0.0 ? worth(sh.row[b], x) : order_double(v);
            a.parent[o + rank] = (int)b; a.token[o + rank] = key_token(x);
            if (a.wide) ((double *)a.score_out)[o + rank] = score; else ((float *)a.score_out)[o + rank] = (float)score;
            if (a.len_out) a.len_out[o + rank] = sh.row[b].len;
        }
    }
    for (int k = m + tid; k < a.n_out; k += threads) {
        a.parent[o + k] = -1; a.token[o + k] = -1;
        if (a.wide) ((double *)a.score_out)[o + k] = -INFINITY; else ((float *)a.score_out)[o + k] = -INFINITY;
        if (a.len_out) a.len_out[o + k] = 0;
    }
}

}  // namespace rs
