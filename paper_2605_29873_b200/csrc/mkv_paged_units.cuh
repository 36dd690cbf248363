// The work of an attention launch as one list: units (sequence, KV head, tile of RT rows) in order, each a
// number of blocks of BLK cached tokens.  The list is cut into one contiguous range per CTA; lengths are on
// the device, so every CTA sums them for itself.
#pragma once
#include "mkv_paged.cuh"
#include "mkv_ptx.cuh"

namespace mkv {

// Bounded wait, for a few seconds at most.  The limit is counted in cycles: reading the global timer takes longer than
// most waits do (the kernel for many rows ran KTIME with it).
__device__ inline bool paged_wait(uint32_t bar, uint32_t parity) {
    for (int i = 0; i < 16; ++i)
        if (ptx::mbar_try_wait(bar, parity)) return true;
    const long long t0 = clock64();
    do {
        for (int i = 0; i < 64; ++i)
            if (ptx::mbar_try_wait(bar, parity)) return true;
    } while (clock64() - t0 < (1ll << 32));
    return false;
}

// One (sequence, KV head, row tile), and the part of the block list that is its own.
struct Unit {
    long long base;   // of its first block in the list
    int s, h, rt;
    int tok0, n, len;
    int row0, rows;   // rows [row0, row0 + rows) of the n * group of its sequence and head
    int plo, phi;     // positions of the first and the last row's token
    int blk0, nblk;   // blocks to read; a unit without any counts as one in the list
    __device__ int count() const { return max(nblk, 1); }
    __device__ long long end() const { return base + count(); }
};

template <int RT, int BLK>
__device__ inline void unit_rows(const PagedAttendArgs& a, Unit& u) {
    const int G = a.c.group, R = u.n * G;
    u.row0 = u.rt * RT;
    u.rows = min(RT, R - u.row0);
    u.plo = u.len - u.n + u.row0 / G;
    u.phi = u.len - u.n + (u.row0 + u.rows - 1) / G;
    const int begin = a.window > 0 ? max(0, u.plo - a.window + 1) : 0;
    u.blk0 = begin / BLK;
    u.nblk = u.phi >= begin ? u.phi / BLK - u.blk0 + 1 : 0;
}
template <int RT> __device__ inline int row_tiles(const PagedAttendArgs& a, int n) { return (n * a.c.group + RT - 1) / RT; }

// Blocks of one head of sequence s in the list.
template <int RT, int BLK>
__device__ inline long long blocks_per_head(const PagedAttendArgs& a, const PagedSpan& sp) {
    Unit u;
    u.n = sp.n; u.len = sp.len;
    long long t = 0;
    const int rts = row_tiles<RT>(a, sp.n);
    for (u.rt = 0; u.rt < rts; ++u.rt) { unit_rows<RT, BLK>(a, u); t += u.count(); }
    return t;
}

// Moves u to the next unit that has rows; false behind the last.
template <int RT, int BLK>
__device__ inline bool next_unit(const PagedAttendArgs& a, Unit& u) {
    u.base = u.end();
    if (++u.rt >= row_tiles<RT>(a, u.n)) {
        u.rt = 0;
        if (++u.h >= a.c.kv_heads) {
            u.h = 0;
            do {
                if (++u.s >= a.b.batch) return false;
                const PagedSpan sp = paged_span(a.c, a.b, u.s);
                u.tok0 = sp.tok0; u.n = sp.n; u.len = sp.len;
            } while (u.n == 0);
        }
    }
    unit_rows<RT, BLK>(a, u);
    return true;
}

// Length of the list, and which range of it this CTA has.  Called by all threads of a block of THREADS; the
// thread that finds the first unit leaves it in *first.  `want(total)`: the number of ranges.  Returns false
// where the CTA has no work (for all threads alike).
struct Range {
    long long total, t0, t1;
    int n;   // ranges
    __device__ long long begin_of(int r) const { return total * r / n; }
    __device__ int of(long long t) const {
        int r = (int)(t * n / total);
        while (begin_of(r + 1) <= t) ++r;
        while (begin_of(r) > t) --r;
        return r;
    }
};
template <int RT, int BLK, int THREADS, typename Want>
__device__ inline bool find_range(const PagedAttendArgs& a, Range& r, Unit* first, long long* scan, Want want) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int per = (a.b.batch + THREADS - 1) / THREADS, s0 = min(a.b.batch, tid * per), s1 = min(a.b.batch, s0 + per);
    long long mine = 0;
    for (int s = s0; s < s1; ++s) {
        const PagedSpan sp = paged_span(a.c, a.b, s);
        if (sp.n > a.max_new) paged_fail(a.c, MKV_ERR_CAPACITY);
        mine += blocks_per_head<RT, BLK>(a, sp) * a.c.kv_heads;
    }
    long long before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += x;
    }
    if (lane == 31) scan[warp] = before;
    __syncthreads();
    r.total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) before += scan[w];
        r.total += scan[w];
    }
    before -= mine;
    if (r.total == 0) return false;
    r.n = (int)max(1ll, min((long long)gridDim.x, want(r.total)));
    if (blockIdx.x >= r.n) return false;
    r.t0 = r.begin_of(blockIdx.x);
    r.t1 = r.begin_of(blockIdx.x + 1);
    if (before <= r.t0 && r.t0 < before + mine) {
        Unit u;
        long long base = before;
        for (int s = s0; s < s1; ++s) {
            const PagedSpan sp = paged_span(a.c, a.b, s);
            const long long head = blocks_per_head<RT, BLK>(a, sp), all = head * a.c.kv_heads;
            if (r.t0 < base + all) {
                u.s = s; u.tok0 = sp.tok0; u.n = sp.n; u.len = sp.len;
                u.h = (int)((r.t0 - base) / head);
                u.base = base + u.h * head;
                u.rt = 0;
                unit_rows<RT, BLK>(a, u);
                while (u.end() <= r.t0) { u.base = u.end(); ++u.rt; unit_rows<RT, BLK>(a, u); }
                break;
            }
            base += all;
        }
        *first = u;
    }
    __syncthreads();
    return true;
}

}  // namespace mkv
