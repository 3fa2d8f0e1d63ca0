// A pool of pages that sequences share (rs_pages_reserve, rs_pages_release, rs_pages_fork, rs_pages_copy, rs_pages_compact).
//
// All state is the page table and, for each page, how many of its entries name it; a page that none names is free, and a call
// that needs pages takes the free ones of the lowest indices in order.  So a call's result depends on the state before it alone, and no atomic's order shows:
// counts are sums, and whoever takes the k-th free page is fixed by the order of the call's rows.
#pragma once

#include "device_utils.h"
#include "../../include/rstitch.h"

namespace rs {

constexpr int POOL_ROWS = 1024;                                    // rows of a call, at most
constexpr int POOL_THREADS = 1024, POOL_WAVES = POOL_THREADS / 64;

struct Pool {
    uint16_t *k, *v;
    int *table, *ref;
    int n_layers, n_pages, page_shift, n_slots, max_pages, n_kv, head_dim;
    unsigned int *flags;                                           // may be null
};

__device__ __forceinline__ bool is_page(const Pool &p, int page) { return page >= 0 && page < p.n_pages; }
__device__ __forceinline__ void pool_flag(const Pool &p, int row, unsigned int flag) { if (p.flags) atomicOr(p.flags + row, flag); }

// Counts are changed by atomics, which act in the L2, and read past the vector caches; a thread's atomics have acted once it has waited for them.
__device__ __forceinline__ int ref_load(const int *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void ref_store(int *p, int v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void ref_add(int *p, int v) { (void)__hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void refs_settled() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

__device__ __forceinline__ int wave_scan(int v) {                  // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int u = __shfl_up(v, o, RS_WAVE); if (lane >= o) v += u; }
    return v;
}
// Sum of v over the threads before this one; total: over all.  sh: POOL_WAVES ints of LDS.
__device__ __forceinline__ int block_scan(int v, int *sh, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in = wave_scan(v);
    __syncthreads();                                               // sh may still be read from the last call
    if (lane == 63) sh[wave] = in;
    __syncthreads();
    int before = in - v;
    total = 0;
#pragma unroll
    for (int w = 0; w < POOL_WAVES; ++w) { if (w < wave) before += sh[w]; total += sh[w]; }
    return before;
}

// found(i, rank) for those i of 0 .. n - 1, in order, whose number load(i) passes test(), until at least `enough` have.  Returns how many have.
// ORDERED_EACH numbers a thread at once, POOL_THREADS apart, so that they are requested together and side by side.
constexpr int ORDERED_EACH = 8, ORDERED_COUNTS = ORDERED_EACH * POOL_WAVES;
static_assert(ORDERED_COUNTS == 128, "two counts a lane");
template <typename L, typename T, typename F>
__device__ __forceinline__ int ordered(int n, int enough, int *sh, L load, T test, F found) {       // sh: ORDERED_COUNTS ints of LDS
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int STEP = POOL_THREADS * ORDERED_EACH;
    int rank = 0, next[ORDERED_EACH];
#pragma unroll
    for (int u = 0; u < ORDERED_EACH; ++u) next[u] = n > 0 ? load(min(POOL_THREADS * u + tid, n - 1)) : 0;
    for (int i0 = 0; i0 < n && rank < enough; i0 += STEP) {
        int x[ORDERED_EACH];
#pragma unroll
        for (int u = 0; u < ORDERED_EACH; ++u) {
            x[u] = next[u];
            if (i0 + STEP < n) next[u] = load(min(i0 + STEP + POOL_THREADS * u + tid, n - 1));
        }
        uint32_t in = 0;
        int before[ORDERED_EACH];
        __syncthreads();                                           // sh may still be read from the last time round
#pragma unroll
        for (int u = 0; u < ORDERED_EACH; ++u) {
            const bool yes = i0 + POOL_THREADS * u + tid < n && test(x[u]);
            const unsigned long long who = __ballot(yes);
            in |= (uint32_t)yes << u;
            before[u] = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
            if (lane == 0) sh[u * POOL_WAVES + wave] = (int)__popcll(who);
        }
        __syncthreads();
        const int a = sh[lane], b = sh[64 + lane], to_a = wave_scan(a), all_a = __shfl(to_a, 63, RS_WAVE), to_b = wave_scan(b) + all_a;
#pragma unroll
        for (int u = 0; u < ORDERED_EACH; ++u) {
            const int c = u * POOL_WAVES + wave, at = c < 64 ? __shfl(to_a - a, c & 63, RS_WAVE) : __shfl(to_b - b, c & 63, RS_WAVE);
            if (in >> u & 1) found(i0 + POOL_THREADS * u + tid, rank + at + before[u]);
        }
        rank += __shfl(to_b, 63, RS_WAVE);
    }
    return rank;
}

// Which row names a number first: a table of twice as many places as there can be rows.
struct FirstRow { int key[2 * POOL_ROWS], row[2 * POOL_ROWS]; };
__device__ __forceinline__ void first_clear(FirstRow &f) {
    for (int i = threadIdx.x; i < 2 * POOL_ROWS; i += POOL_THREADS) { f.key[i] = -1; f.row[i] = POOL_ROWS; }
}
__device__ __forceinline__ int first_enter(FirstRow &f, int key, int row) {          // key >= 0; returns its place
    int h = (int)((uint32_t)key * 2654435761u >> 21);
    for (;;) {
        const int seen = atomicCAS(&f.key[h], -1, key);
        if (seen == -1 || seen == key) break;
        h = (h + 1) & (2 * POOL_ROWS - 1);
    }
    atomicMin(&f.row[h], row);
    return h;
}

// ---------------------------------------------------------------- rs_pages_release
struct RangeArgs { Pool p; const int *slot, *from, *to; int n; int *list; };

// Row r of a call on ranges of positions; false: out of range.
__device__ __forceinline__ bool pool_range(const RangeArgs &a, int r, int &slot, int &from, int &to) {
    slot = a.slot[r];
    from = a.from ? a.from[r] : 0;
    to = a.to[r];
    return slot >= 0 && slot < a.p.n_slots && from >= 0 && to >= from && to <= (long long)a.p.max_pages << a.p.page_shift;
}

// grid n, block 256: the entries whose pages lie wholly in the row's range.  A launch and one chain entry -> count: 1.9 us for a row, 4.7 for 128 rows of up to 125 entries.
__global__ void __launch_bounds__(256) k_pool_release(RangeArgs a) {
    const int r = blockIdx.x, tid = threadIdx.x;
    int slot, from, to;
    const bool ok = pool_range(a, r, slot, from, to);
    int again = 0;
    for (int i = tid; i < r; i += 256) again |= a.slot[i] == slot;
    again = __syncthreads_or(again);
    if (!ok || again) { if (tid == 0) pool_flag(a.p, r, RS_FLAG_BADARG); return; }
    const int ps = 1 << a.p.page_shift, e0 = (from + ps - 1) >> a.p.page_shift, e1 = to >> a.p.page_shift;
    int *entry = a.p.table + (size_t)slot * a.p.max_pages;
    for (int e = e0 + tid; e < e1; e += 256) {
        const int page = entry[e];
        if (is_page(a.p, page)) ref_add(a.p.ref + page, -1);
        entry[e] = -1;
    }
}

// ---------------------------------------------------------------- rs_pages_reserve
// grid 1, block POOL_THREADS.  Counts the entries that lack a page, row by row, with as many lanes a row as take the longest one in at once; finds as
// many free pages; hands them out in the same walk.  One workgroup: what a decode step needs is a chain of four dependent reads, not bytes (1 row 3 us,
// 128 rows that need 8 pages behind 35800 held ones 19, 1000 rows that need 63 behind 44000 31).  Where a call wants thousands it is bound by one CU's stores: 10149 pages
// for 128 rows 24 us.
constexpr int RESERVE_EACH = 8;                                    // entries a lane looks at together
__global__ void __launch_bounds__(POOL_THREADS) k_pool_reserve(RangeArgs a) {
    __shared__ FirstRow first;
    __shared__ int sh[ORDERED_COUNTS], slot_of[POOL_ROWS], entry_of[POOL_ROWS], len_of[POOL_ROWS], lack_of[POOL_ROWS], longest, taken;
    const int tid = threadIdx.x, lane = tid & 63, n = a.n, ps = 1 << a.p.page_shift;
    int slot = -1, from = 0, to = 0, len = 0, place = 0;
    const bool ok = tid < n && pool_range(a, tid, slot, from, to);
    first_clear(first);
    if (tid == 0) longest = taken = 0;
    __syncthreads();
    if (tid < n && slot >= 0) place = first_enter(first, slot, tid);
    __syncthreads();
    if (tid < n) {
        if (!ok || first.row[place] != tid) pool_flag(a.p, tid, RS_FLAG_BADARG);
        else if (to > from) len = ((to + ps - 1) >> a.p.page_shift) - (from >> a.p.page_shift);
        slot_of[tid] = slot; entry_of[tid] = from >> a.p.page_shift; len_of[tid] = len;
        if (len) atomicMax(&longest, len);
    }
    __syncthreads();
    if (!longest) return;
    int shift = 0;
    while (shift < 6 && RESERVE_EACH << shift < longest) ++shift;
    const int lanes = 1 << shift, sub = lane & (lanes - 1), base = lane - sub;
    const unsigned long long mates = (lanes == 64 ? ~0ull : (1ull << lanes) - 1) << base;
    // f(entry, which, ranks): bit u of `which` says that entry[lanes * u] lacks a page, the ranks[u]-th of the row's that do; returns how many do
    auto walk = [&](int r, auto f) __attribute__((always_inline)) {
        int *row = a.p.table + (size_t)slot_of[r] * a.p.max_pages + entry_of[r], rank = 0;
        const int m = len_of[r];
        for (int e0 = 0; e0 < m; e0 += lanes * RESERVE_EACH) {
            int page[RESERVE_EACH];
#pragma unroll
            for (int u = 0; u < RESERVE_EACH; ++u) page[u] = row[min(e0 + lanes * u + sub, m - 1)];
            uint32_t which = 0;
            int ranks[RESERVE_EACH];
#pragma unroll
            for (int u = 0; u < RESERVE_EACH; ++u) {
                const bool lacks = e0 + lanes * u + sub < m && !is_page(a.p, page[u]);
                const unsigned long long who = __ballot(lacks) & mates;
                which |= (uint32_t)lacks << u;
                ranks[u] = rank + (int)__popcll(who & ((1ull << lane) - 1));
                rank += (int)__popcll(who);
            }
            f(row + e0 + sub, which, ranks);
        }
        return rank;
    };
    for (int r = tid >> shift; r < n; r += POOL_THREADS >> shift) {
        const int lack = walk(r, [](int *, uint32_t, const int (&)[RESERVE_EACH]) {});
        if (sub == 0) lack_of[r] = lack;
    }
    __syncthreads();
    int wanted;
    const int mine = tid < n ? lack_of[tid] : 0, before = block_scan(mine, sh, wanted);
    if (!wanted) return;
    // (a page is counted where it is found, side by side with its neighbours, which entries are not)
    const int have = ordered(a.p.n_pages, wanted, sh, [&](int i) { return a.p.ref[i]; }, [](int count) { return count == 0; },
                             [&](int i, int rank) { if (rank < wanted) { a.list[rank] = i; a.p.ref[i] = 1; } });
    if (tid < n) {
        const bool served = before + mine <= have;
        if (mine && !served) { pool_flag(a.p, tid, RS_FLAG_NO_PAGE); len_of[tid] = 0; }
        if (mine && served) atomicMax(&taken, before + mine);
        lack_of[tid] = before;
    }
    refs_settled();
    for (int i = taken + tid; i < min(have, wanted); i += POOL_THREADS) a.p.ref[__hip_atomic_load(a.list + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)] = 0;
    for (int r = tid >> shift; r < n; r += POOL_THREADS >> shift) {
        const int at = lack_of[r];
        walk(r, [&](int *entry, uint32_t which, const int (&ranks)[RESERVE_EACH]) __attribute__((always_inline)) {
            int page[RESERVE_EACH];                                // (requested together, not one after the other behind a branch each)
#pragma unroll
            for (int u = 0; u < RESERVE_EACH; ++u) page[u] = ref_load(a.list + min(at + ranks[u], a.p.n_pages - 1));
#pragma unroll
            for (int u = 0; u < RESERVE_EACH; ++u) if (which >> u & 1) entry[lanes * u] = page[u];
        });
    }
}

// ---------------------------------------------------------------- moving pages
// What a move of one page is: `part` places (a multiple of 8) from page src to page dst, in all layers.
struct alignas(16) PageMove { int src, dst, part; };

struct CopyArgs {
    Pool to;
    const uint16_t *k, *v;                                         // the pages to read from, to.n_layers of from_pages pages each
    int from_pages;
    const PageMove *moves; const int *n_moves;                     // on the device; or
    const int *src, *dst; int n;                                   // pairs of the caller
    const int *map;                                                // not null: table entries follow it (k_pool_compact)
    int pieces;                                                    // of a page's K or V of one layer, COPY_UNITS * 256 units each
};

constexpr int COPY_UNITS = 4;                                      // 16-byte units a thread
// Places of a channel of V that are written together: 128 bytes.  Writing part of such a line costs more than twice as much as all of it, so the places
// behind the part are read from where they go to and written again (a fork with 70 parts of pages of the 7B shape, 8 / 16 / 24 / 40 / 56 of 64 places: the part
// alone 163 / 166 / 137 / 137 / 149 us, whole halves of a line 144 / 149 / 153 / 121 / 141, whole lines 99 / 101 / 105 / 117 / 136; 70 whole pages copied 104).
constexpr int COPY_BLOCK = 64;

// grid (pieces * 2 * layers, any): a workgroup has its piece of every gridDim.y-th move.  Bound by HBM: 24 pages of 64 positions of the 14B shape, 604 MB read and
// written, 124 us (4.9 TB/s, a large copy's 4.78); 90 of the 7B shape 136.  A fork's parts move more than they hold, since V goes by whole lines that are read at both
// ends: parts of the 7B shape of 122 MB, read and written, 51 us; V's whole lines, read at both ends and written, make some 243 MB of it, 51 us at a copy's rate.
// A part of a page: of K the first `part` places of every head, of V the first `part` places of every channel.
__global__ void __launch_bounds__(256) k_pool_copy(CopyArgs a) {
    const Pool &p = a.to;
    const int tid = threadIdx.x, ps = 1 << p.page_shift;
    if (a.map) {
        const long long entries = (long long)p.n_slots * p.max_pages, threads = (long long)gridDim.x * gridDim.y * 256;
        for (long long i = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 256 + tid; i < entries; i += threads) {
            const int page = p.table[i];
            if (is_page(p, page)) p.table[i] = a.map[page];
        }
    }
    const int piece = blockIdx.x % a.pieces, half = blockIdx.x / a.pieces, layer = half >> 1;
    const bool is_v = half & 1;
    const size_t page_values = (size_t)p.n_kv * p.head_dim << p.page_shift;
    const u32x4_t *from = reinterpret_cast<const u32x4_t *>((is_v ? a.v : a.k) + (size_t)layer * a.from_pages * page_values);
    u32x4_t *to = reinterpret_cast<u32x4_t *>((is_v ? p.v : p.k) + (size_t)layer * p.n_pages * page_values);
    const int gap = is_v ? ps / 8 : ps / 8 * p.head_dim, rows = is_v ? p.n_kv * p.head_dim : p.n_kv, n = a.moves ? *a.n_moves : a.n;
    for (int m = blockIdx.y; m < n; m += gridDim.y) {
        PageMove mv;
        if (a.moves) mv = a.moves[m];
        else {
            mv = {a.src[m], a.dst[m], ps};
            if (mv.src < 0 || mv.src >= a.from_pages || !is_page(p, mv.dst)) { if (blockIdx.x == 0 && tid == 0) pool_flag(p, m, RS_FLAG_BADARG); continue; }
        }
        const u32x4_t *x = from + (size_t)mv.src * (page_values / 8);
        u32x4_t *y = to + (size_t)mv.dst * (page_values / 8);
        const int own = mv.part / 8, row = is_v ? min(ps, (mv.part + COPY_BLOCK - 1) / COPY_BLOCK * COPY_BLOCK) / 8 : own * p.head_dim;
        const int units = rows * row, u0 = piece * (256 * COPY_UNITS) + tid;
        if (piece * (256 * COPY_UNITS) >= units || x == y) continue;
        u32x4_t w[COPY_UNITS];
        int at[COPY_UNITS];
#pragma unroll
        for (int i = 0; i < COPY_UNITS; ++i) {
            const int u = min(u0 + 256 * i, units - 1), r = row == gap ? 0 : u / row;
            at[i] = u + r * (gap - row);
            w[i] = (is_v && (row == gap ? u % gap : u - r * row) >= own ? y : x)[at[i]];
        }
#pragma unroll
        for (int i = 0; i < COPY_UNITS; ++i) if (u0 + 256 * i < units) y[at[i]] = w[i];
    }
}

// ---------------------------------------------------------------- rs_pages_fork
struct ForkArgs { Pool p; const int *slot, *parent, *pos; int *pos_out; int n_groups, n_beams; PageMove *moves; int *n_moves; };

// grid 1, block POOL_THREADS.  Reads everything before it writes a table entry: whether all rows are in range, the counts after the call, the rows that
// need a page, the pages they get.  FORK_EACH: table entries that a thread requests together, and holds between reading and writing them: FORK_FEW where the
// rows have FORK_FEW_ENTRIES at most together, 8 otherwise.  us of a call without copies by 2 / by 8, rows whose entries all change: 4 rows of 64 entries 7.1 / 8.6, 128 of 16
// 8.6 / 9.9, 4096 entries (4 to 512 rows) 9.9 to 10.2 / 10.8 to 11.1, 8192 (4 to 512 rows) 13.0 to 13.4 / 13.2 to 13.5, 1000 rows of 8 14.9 / 14.0, 128 of 128 19.8 / 18.6, 1000 of
// 64 92 / 51.  Bound by the chain of its steps, each a read that depends on the last (slot, position,
// table, count, page, table), in one workgroup.
constexpr int FORK_FEW = 2, FORK_FEW_ENTRIES = 4096;
template <int FORK_EACH>
__global__ void __launch_bounds__(POOL_THREADS) k_pool_fork(ForkArgs a) {
    __shared__ FirstRow first;
    __shared__ int sh[ORDERED_COUNTS], slot_of[POOL_ROWS], from_of[POOL_ROWS], whole_of[POOL_ROWS], new_page[POOL_ROWS], want_row[POOL_ROWS];
    const Pool &p = a.p;
    const int tid = threadIdx.x, n = a.n_groups * a.n_beams, mp = p.max_pages, ps = 1 << p.page_shift;
    const int slot = tid < n ? a.slot[tid] : -1, parent = tid < n ? a.parent[tid] : -1;
    first_clear(first);
    __syncthreads();
    int place = 0;
    if (tid < n) { slot_of[tid] = slot; if (slot >= 0) place = first_enter(first, slot, tid); }
    __syncthreads();
    // ---- a thread a row: its parent's slot and positions
    int bad = 0, from = -1, pos = 0, tail = 0, whole = 0, page = -1;
    if (tid < n) {
        bad = slot < 0 || slot >= p.n_slots || parent >= a.n_beams || first.row[place] != tid;
        if (!bad && parent >= 0) {
            const int q = tid / a.n_beams * a.n_beams + parent;
            from = slot_of[q]; pos = a.pos[q];
            if (from < 0 || from >= p.n_slots || pos < 0 || pos > (long long)mp << p.page_shift) { bad = 1; from = -1; pos = 0; }
        }
        whole = pos >> p.page_shift; tail = pos & (ps - 1);
        if (bad) pool_flag(p, tid, RS_FLAG_BADARG);
    }
    if (__syncthreads_or(bad)) { if (tid == 0) *a.n_moves = 0; return; }
    if (tid < n) {
        if (from >= 0 && tail) { page = p.table[(size_t)from * mp + whole]; if (!is_page(p, page)) page = -1; }
        from_of[tid] = from; whole_of[tid] = whole;
    }
    first_clear(first);                                            // (all have read it before the last barrier)
    __syncthreads();
    if (page >= 0) place = first_enter(first, page, tid);
    // ---- counts: what the rows held goes, the whole pages of their parents come
    // entries of a thread are POOL_THREADS apart in the rows one behind the other, FORK_EACH of them requested together
    const int jump_r = POOL_THREADS / mp, jump_j = POOL_THREADS - jump_r * mp;
    auto count = [&](int by) __attribute__((always_inline)) {
        int r = tid / mp, j = tid - r * mp;
        while (r < n) {
            int old[FORK_EACH], now[FORK_EACH];
#pragma unroll
            for (int k = 0; k < FORK_EACH; ++k) {
                old[k] = now[k] = -1;
                if (r < n) {
                    const int f = from_of[r];
                    old[k] = p.table[(size_t)slot_of[r] * mp + j];
                    if (f >= 0 && j < whole_of[r]) now[k] = p.table[(size_t)f * mp + j];
                }
                r += jump_r; j += jump_j;
                if (j >= mp) { j -= mp; ++r; }
            }
#pragma unroll
            for (int k = 0; k < FORK_EACH; ++k) {
                if (old[k] == now[k]) continue;
                if (is_page(p, old[k])) ref_add(p.ref + old[k], -by);
                if (is_page(p, now[k])) ref_add(p.ref + now[k], by);
            }
        }
        refs_settled();
    };
    count(1);
    // ---- the last page of a parent: the first row that wants it keeps it if nobody else has it
    const bool keep = page >= 0 && first.row[place] == tid && ref_load(p.ref + page) == 0;
    __syncthreads();                                               // (all have looked before the first count changes)
    if (keep) ref_store(p.ref + page, 1);
    const bool want = page >= 0 && !keep;
    int wanted;
    const int rank = block_scan(want, sh, wanted);
    if (tid < n) new_page[tid] = keep ? page : -1;
    if (want) want_row[rank] = tid;
    refs_settled();
    const int have = ordered(p.n_pages, wanted, sh, [&](int i) { return ref_load(p.ref + i); }, [](int count) { return count == 0; },
                             [&](int i, int k) { if (k < wanted) new_page[want_row[k]] = i; });
    __syncthreads();
    if (have < wanted) {                                           // as before the call
        if (keep) ref_store(p.ref + page, 0);
        refs_settled();
        count(-1);
        if (tid < n) pool_flag(p, tid, RS_FLAG_NO_PAGE);
        if (tid == 0) *a.n_moves = 0;
        return;
    }
    if (want) {
        ref_store(p.ref + new_page[tid], 1);
        a.moves[rank] = {page, new_page[tid], (tail + 7) / 8 * 8};
    }
    if (tid == 0) *a.n_moves = wanted;
    if (a.pos_out && tid < n) a.pos_out[tid] = pos;                // (every row's position was read before)
    // ---- the tables, some columns of all rows at a time: a row may be another one's parent
    const int cols = mp < POOL_THREADS * FORK_EACH / n ? mp : POOL_THREADS * FORK_EACH / n;
    for (int c0 = 0; c0 < mp; c0 += cols) {
        int x[FORK_EACH];
#pragma unroll
        for (int k = 0; k < FORK_EACH; ++k) {
            const int i = tid + POOL_THREADS * k, r = i / cols, j = c0 + i - r * cols;
            x[k] = -1;
            if (r >= n || j >= mp || from_of[r] < 0) continue;
            if (j < whole_of[r]) { x[k] = p.table[(size_t)from_of[r] * mp + j]; if (!is_page(p, x[k])) x[k] = -1; }
            else if (j == whole_of[r]) x[k] = new_page[r];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < FORK_EACH; ++k) {
            const int i = tid + POOL_THREADS * k, r = i / cols, j = c0 + i - r * cols;
            if (r < n && j < mp) p.table[(size_t)slot_of[r] * mp + j] = x[k];
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- rs_pages_compact
struct CompactArgs { Pool p; int *used; PageMove *moves; int *n_moves, *map, *gaps; };

// grid 1, block POOL_THREADS: used pages from the number of used pages on, in order, go to the free ones below it, in order.  Three reads of the counts, of which the first
// is of all: 6.5 us for 400 pages, 7.7 for 4000.
__global__ void __launch_bounds__(POOL_THREADS) k_pool_compact(CompactArgs a) {
    __shared__ int sh[ORDERED_COUNTS];
    const Pool &p = a.p;
    const int tid = threadIdx.x;
    int mine = 0, used;
    for (int i = tid; i < p.n_pages; i += POOL_THREADS) { mine += p.ref[i] != 0; a.map[i] = i; }
    (void)block_scan(mine, sh, used);
    ordered(used, 0x7fffffff, sh, [&](int i) { return p.ref[i]; }, [](int count) { return count == 0; }, [&](int i, int k) { a.gaps[k] = i; });
    refs_settled();
    const int n = ordered(p.n_pages - used, 0x7fffffff, sh, [&](int i) { return p.ref[used + i]; }, [](int count) { return count != 0; }, [&](int i, int k) {
        const int from = used + i, to = __hip_atomic_load(a.gaps + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        a.moves[k] = {from, to, 1 << p.page_shift};
        a.map[from] = to;
        p.ref[to] = p.ref[from];
        p.ref[from] = 0;
    });
    if (tid == 0) { *a.used = used; *a.n_moves = n; }
}

}  // namespace rs
