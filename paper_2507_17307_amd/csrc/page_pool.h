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

// test(i) of i = 0 .. n - 1 in order; found(i, rank) for those that pass, until at least `enough` have.  Returns how many have.
template <typename T, typename F>
__device__ __forceinline__ int ordered(int n, int enough, int *sh, T test, F found) {
    int rank = 0;
    for (int i0 = 0; i0 < n && rank < enough; i0 += POOL_THREADS) {
        const int i = i0 + threadIdx.x;
        const bool yes = i < n && test(i);
        int total;
        const int at = block_scan(yes, sh, total);
        if (yes) found(i, rank + at);
        rank += total;
    }
    return rank;
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

// grid n, block 256: the entries whose pages lie wholly in the row's range
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
// grid 1, block POOL_THREADS: the entries of all rows' ranges that name no page, in order, and the free pages, in order
__global__ void __launch_bounds__(POOL_THREADS) k_pool_reserve(RangeArgs a) {
    __shared__ int sh[POOL_WAVES], slot_of[POOL_ROWS], first_of[POOL_ROWS], start[POOL_ROWS + 1], lack_end[POOL_ROWS];
    const int tid = threadIdx.x, n = a.n;
    // a thread a row: its range of entries
    int slot = -1, from = 0, to = 0, len = 0, total;
    const bool ok = tid < n && pool_range(a, tid, slot, from, to);
    if (tid < n) slot_of[tid] = slot;
    __syncthreads();
    bool again = false;
    for (int i = 0; i < tid && tid < n; ++i) again |= slot_of[i] == slot;
    if (tid < n && (!ok || again)) pool_flag(a.p, tid, RS_FLAG_BADARG);
    const int ps = 1 << a.p.page_shift, e0 = from >> a.p.page_shift;
    if (ok && !again && to > from) len = ((to + ps - 1) >> a.p.page_shift) - e0;
    // (the entries of a call are no more than rows times table entries, below 2^31 as checked on the host)
    const int at = block_scan(len, sh, total);
    if (tid < n) { first_of[tid] = e0; start[tid] = at; lack_end[tid] = 0; }
    if (tid == 0) start[n] = total;
    __syncthreads();
    auto place = [&](int i, int &row) {                             // entry i of the call
        int lo = 0, hi = n;
        while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (start[mid] <= i) lo = mid; else hi = mid; }
        row = lo;
        return a.p.table + (size_t)slot_of[lo] * a.p.max_pages + first_of[lo] + (i - start[lo]);
    };
    // how many entries lack a page, up to the end of each row
    auto lacks = [&](int i) { int row; return !is_page(a.p, *place(i, row)); };
    const int lack = ordered(total, 0x7fffffff, sh, lacks, [&](int i, int rank) { int row; (void)place(i, row); atomicMax(&lack_end[row], rank + 1); });
    if (lack == 0) return;
    __syncthreads();
    const int have = ordered(a.p.n_pages, lack, sh, [&](int i) { return ref_load(a.p.ref + i) == 0; },
                             [&](int i, int rank) { if (rank < lack) __hip_atomic_store(a.list + rank, i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); });
    refs_settled();
    if (tid < n && lack_end[tid] > have) pool_flag(a.p, tid, RS_FLAG_NO_PAGE);
    // (a row's entries are looked at and filled in the same order by the same threads)
    ordered(total, 0x7fffffff, sh, lacks, [&](int i, int rank) {
        int row;
        int *entry = place(i, row);
        if (lack_end[row] > have) return;
        const int page = __hip_atomic_load(a.list + rank, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *entry = page;
        ref_store(a.p.ref + page, 1);
    });
}

// ---------------------------------------------------------------- moving pages
// What a move of one page is: `part` places (a multiple of 8) from page src to page dst, in all layers.
struct PageMove { int src, dst, part, row; };

struct CopyArgs {
    Pool to;
    const uint16_t *k, *v;                                         // the pages to read from, to.n_layers of from_pages pages each
    int from_pages;
    const PageMove *moves; const int *n_moves;                     // on the device; or
    const int *src, *dst; int n;                                   // pairs of the caller
    const int *map;                                                // not null: table entries follow it (k_pool_compact)
};

constexpr int COPY_UNITS = 4;                                      // 16-byte units a thread

// One piece of a page's K or V of one layer: units u0 + tid, ... of 16 bytes.
__device__ __forceinline__ void copy_piece(const Pool &p, const uint16_t *src, uint16_t *dst, int part, bool is_v, int u0) {
    const int ps = 1 << p.page_shift, row = is_v ? part / 8 : part * p.head_dim / 8, gap = is_v ? ps / 8 : ps * p.head_dim / 8;
    const int units = (is_v ? p.n_kv * p.head_dim : p.n_kv) * row;
    uint4 x[COPY_UNITS];
    int at[COPY_UNITS];
#pragma unroll
    for (int i = 0; i < COPY_UNITS; ++i) {
        const int u = u0 + threadIdx.x + 256 * i;
        at[i] = u >= units ? -1 : part == ps ? u : u / row * gap + u % row;
        if (at[i] >= 0) x[i] = reinterpret_cast<const uint4 *>(src)[at[i]];
    }
#pragma unroll
    for (int i = 0; i < COPY_UNITS; ++i)
        if (at[i] >= 0) reinterpret_cast<uint4 *>(dst)[at[i]] = x[i];
}

// grid any, block 256
__global__ void __launch_bounds__(256) k_pool_copy(CopyArgs a) {
    const Pool &p = a.to;
    const int ps = 1 << p.page_shift;
    if (a.map) {
        const size_t entries = (size_t)p.n_slots * p.max_pages;
        for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < entries; i += (size_t)gridDim.x * 256) {
            const int page = p.table[i];
            if (is_page(p, page)) p.table[i] = a.map[page];
        }
    }
    const size_t page_values = (size_t)p.n_kv * p.head_dim << p.page_shift;
    const int pieces = (int)((page_values / 8 + 256 * COPY_UNITS - 1) / (256 * COPY_UNITS));
    const int n = a.moves ? *a.n_moves : a.n;
    const long long items = (long long)n * p.n_layers * 2 * pieces;
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const int piece = (int)(it % pieces), kv = (int)(it / pieces % 2), layer = (int)(it / pieces / 2 % p.n_layers), m = (int)(it / pieces / 2 / p.n_layers);
        PageMove mv;
        if (a.moves) mv = a.moves[m];
        else {
            mv = {a.src[m], a.dst[m], ps, m};
            if (mv.src < 0 || mv.src >= a.from_pages || !is_page(p, mv.dst)) { if (piece == 0 && kv == 0 && layer == 0 && threadIdx.x == 0) pool_flag(p, m, RS_FLAG_BADARG); continue; }
        }
        const uint16_t *src = (kv ? a.v : a.k) + ((size_t)layer * a.from_pages + mv.src) * page_values;
        uint16_t *dst = (kv ? p.v : p.k) + ((size_t)layer * p.n_pages + mv.dst) * page_values;
        if (src != dst) copy_piece(p, src, dst, mv.part, kv, piece * 256 * COPY_UNITS);
    }
}

// ---------------------------------------------------------------- rs_pages_fork
struct ForkArgs { Pool p; const int *slot, *parent, *pos; int *pos_out; int n_groups, n_beams; PageMove *moves; int *n_moves; };

constexpr int FORK_EACH = 8;                                       // table entries a thread holds between reading and writing them

// grid 1, block POOL_THREADS.  Reads everything before it writes a table entry: whether all rows are in range, the counts after the call, the rows that
// need a page, the pages they get.
__global__ void __launch_bounds__(POOL_THREADS) k_pool_fork(ForkArgs a) {
    __shared__ int sh[POOL_WAVES], slot_of[POOL_ROWS], from_of[POOL_ROWS], whole_of[POOL_ROWS], tail_page[POOL_ROWS], new_page[POOL_ROWS], want_row[POOL_ROWS];
    const Pool &p = a.p;
    const int tid = threadIdx.x, n = a.n_groups * a.n_beams, mp = p.max_pages, ps = 1 << p.page_shift;
    if (tid < n) slot_of[tid] = a.slot[tid];
    __syncthreads();
    // ---- a thread a row: its parent's slot and positions
    int bad = 0, from = -1, pos = 0, tail = 0, whole = 0, page = -1;
    if (tid < n) {
        const int slot = slot_of[tid], parent = a.parent[tid];
        bad = slot < 0 || slot >= p.n_slots || parent >= a.n_beams;
        for (int i = 0; i < tid; ++i) bad |= slot_of[i] == slot;
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
        from_of[tid] = from; whole_of[tid] = whole; tail_page[tid] = page;
    }
    __syncthreads();
    // ---- counts: what the rows held goes, the whole pages of their parents come
    const long long entries = (long long)n * mp;
    auto count = [&](int by) {
        for (long long i = tid; i < entries; i += POOL_THREADS) {
            const int r = (int)(i / mp), j = (int)(i - (long long)r * mp), f = from_of[r];
            const int old = p.table[(size_t)slot_of[r] * mp + j], now = f >= 0 && j < whole_of[r] ? p.table[(size_t)f * mp + j] : -1;
            if (old == now) continue;
            if (is_page(p, old)) ref_add(p.ref + old, -by);
            if (is_page(p, now)) ref_add(p.ref + now, by);
        }
        refs_settled();
    };
    count(1);
    // ---- the last page of a parent: the first row that wants it keeps it if nobody else has it
    bool keep = false;
    if (page >= 0) {
        keep = ref_load(p.ref + page) == 0;
        for (int i = 0; i < tid && keep; ++i) keep = tail_page[i] != page;
    }
    __syncthreads();                                               // (all have looked before the first count changes)
    if (keep) ref_store(p.ref + page, 1);
    const bool want = page >= 0 && !keep;
    int wanted;
    const int rank = block_scan(want, sh, wanted);
    if (tid < n) new_page[tid] = keep ? page : -1;
    if (want) want_row[rank] = tid;
    refs_settled();
    const int have = ordered(p.n_pages, wanted, sh, [&](int i) { return ref_load(p.ref + i) == 0; }, [&](int i, int k) { if (k < wanted) new_page[want_row[k]] = i; });
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
        a.moves[rank] = {page, new_page[tid], (tail + 7) / 8 * 8, tid};
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

// grid 1, block POOL_THREADS: used pages from the number of used pages on, in order, go to the free ones below it, in order
__global__ void __launch_bounds__(POOL_THREADS) k_pool_compact(CompactArgs a) {
    __shared__ int sh[POOL_WAVES];
    const Pool &p = a.p;
    const int tid = threadIdx.x;
    int mine = 0, used;
    for (int i = tid; i < p.n_pages; i += POOL_THREADS) { mine += p.ref[i] != 0; a.map[i] = i; }
    (void)block_scan(mine, sh, used);
    ordered(used, 0x7fffffff, sh, [&](int i) { return p.ref[i] == 0; }, [&](int i, int k) { a.gaps[k] = i; });
    refs_settled();
    const int n = ordered(p.n_pages - used, 0x7fffffff, sh, [&](int i) { return p.ref[used + i] != 0; }, [&](int i, int k) {
        const int from = used + i, to = __hip_atomic_load(a.gaps + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        a.moves[k] = {from, to, 1 << p.page_shift, k};
        a.map[from] = to;
        p.ref[to] = p.ref[from];
        p.ref[from] = 0;
    });
    if (tid == 0) { *a.used = used; *a.n_moves = n; }
}

}  // namespace rs
