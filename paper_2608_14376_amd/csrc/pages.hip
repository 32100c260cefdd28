// pages.hip -- pages of a paged cache given to slots, on the device: fork,
// reorder, cut, grow, free (corun_pages_assign) and compact
// (corun_pages_compact).
//
// Nothing is kept between calls but the table and the slots' counts: which pages
// are in use follows from them.  A plan is made, then carried out:
//  1 clear    every page free
//  2 mark     what each slot takes is checked and its pages are marked; its new row
//             of the table is staged (the old rows are still read)
//  3 plan     one workgroup deals the free pages to the slots in order and lists
//             the copies; it alone decides whether anything is written
//  4 carry    rows of the table, and the copies, 16 KB of a page of a layer's k or
//             v to a workgroup
// Where the marks of all pages fit in LDS and the table is small, 1 to 3 and the
// table's rows are one workgroup's work, and a call is two launches.  Marks are
// integer minima, so their order does not matter.
//
// The plan is latency, barriers above all: 5 to 8 us in one workgroup (twice the
// barriers took 1 to 2 us more), 11 to 13 in three launches.  The copies
// are bound by memory: 148 pages of 1.57 MB (48 layers) moved in 92 to 98 us, 4.8 to
// 5.1 TB/s; 32 part-filled pages of 48 layers in 19 to 21.  Pieces of 16 KB whose loads
// all go out before the stores: one 4 KB head to a workgroup took 24 us there.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include <algorithm>

#include "device.h"
#include "groups.h"

namespace corun {
namespace {

constexpr int FREE = INT_MAX, WHOLE = -1;              // marks of a page; >= 0: the lowest slot with it as its part-filled page

// The workspace.
struct Plan {
    int32_t *head;                                     // [16]
    int32_t *mark;                                     // [pages]; compaction: then a page's new number
    int32_t *list;                                     // [pages] free pages in order
    int32_t *fresh0, *first, *total, *tail;            // [slots] first of its fresh pages, pages it has, pages it shall have, part-filled page taken
    int32_t *from, *to, *count;                        // [max(slots, pages)] copies: pages and tokens
    int32_t *rows;                                     // [slots][width] staged
};
enum { BAD = 0, STATUS, COPIES };                      // of head

__host__ __device__ inline size_t up4(size_t n) { return (n + 3) & ~(size_t)3; }

inline Plan plan_of(void *ws, int slots, int width, int pages)
{
    Plan p;
    int32_t *at = (int32_t *)ws;
    const auto take = [&](size_t n) { int32_t *q = at; at += up4(n); return q; };
    const size_t moves = (size_t)std::max(slots, pages);
    p.head = take(16);
    p.mark = take(pages);
    p.list = take(pages);
    p.fresh0 = take(slots);
    p.first = take(slots);
    p.total = take(slots);
    p.tail = take(slots);
    p.from = take(moves);
    p.to = take(moves);
    p.count = take(moves);
    p.rows = take((size_t)slots * width);
    return p;
}

__global__ __launch_bounds__(256) void k_pages_clear(Plan p, int pages)
{
    if (blockIdx.x == 0 && threadIdx.x < 16) p.head[threadIdx.x] = 0;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < pages; i += gridDim.x * 256) p.mark[i] = FREE;
}

// Assignment: one wavefront to a slot.
__global__ __launch_bounds__(256) void k_pages_mark(PageShape s, Plan p, const int32_t *__restrict__ table,
                                                    const int32_t *__restrict__ held, const int32_t *__restrict__ src,
                                                    const int32_t *__restrict__ keep, const int32_t *__restrict__ hold)
{
    const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (r >= s.slots) return;
    const int from = src[r];
    int nfull = 0, total = 0, tail = -1;
    bool bad = from < -1 || from >= s.slots;
    if (!bad && from >= 0) {
        const int n = keep[r], m = hold == nullptr ? n : hold[r], has = held[from];
        bad = has < 0 || has > s.width || n < 0 || n > (long long)has * s.page_size || m < n ||
              m > (long long)s.width * s.page_size;
        if (!bad) {
            nfull = n / s.page_size;
            total = (int)(((long long)m + s.page_size - 1) / s.page_size);
            const int taken = nfull + (n > nfull * s.page_size);
            for (int i = lane; i < taken; i += 64) {
                const int page = table[(size_t)from * s.width + i];
                if ((unsigned)page >= (unsigned)s.pages) {
                    bad = true;
                    continue;
                }
                p.rows[(size_t)r * s.width + i] = page;
                if (i < nfull) atomicMin(&p.mark[page], WHOLE);
                else {
                    atomicMin(&p.mark[page], r);
                    tail = page;
                }
            }
            const unsigned long long has_tail = __ballot(tail >= 0);
            if (has_tail) tail = __shfl(tail, __ffsll((long long)has_tail) - 1, 64);
        }
    }
    if (bad) p.head[BAD] = 1;
    if (lane == 0) {
        p.first[r] = nfull;
        p.total[r] = total;
        p.tail[r] = tail;
    }
}

// A lane's value from a lane before it: n lanes before in its row of sixteen
// (0x110 + n), the last lane of the row before (0x142), lane 31 (0x143); 0 where
// there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ int from_before(int x)
{
    return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}

// Sums of the workgroup's values before the caller's (exclusive), and of all, by its
// sixteen wavefronts in order.  One barrier: calls take two lds in turn, so that
// whoever still reads one has not reached the barrier before it is written again.
__device__ __forceinline__ int before(int v, int *all, int *lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
    x += from_before<0x111, 0xf>(x);
    x += from_before<0x112, 0xf>(x);
    x += from_before<0x114, 0xf>(x);
    x += from_before<0x118, 0xf>(x);
    x += from_before<0x142, 0xa>(x);                   // rows 1 and 3
    x += from_before<0x143, 0xc>(x);                   // rows 2 and 3
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    int sum = 0, mine = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        mine += w < wave ? lds[w] : 0;
        sum += lds[w];
    }
    *all = sum;
    return mine + x - v;
}

// The most of values >= 0 over the workgroup's sixteen wavefronts: noted, and read
// after a barrier.
__device__ __forceinline__ void note_most(int v, int *lds)
{
    v = max(v, from_before<0x111, 0xf>(v));
    v = max(v, from_before<0x112, 0xf>(v));
    v = max(v, from_before<0x114, 0xf>(v));
    v = max(v, from_before<0x118, 0xf>(v));
    v = max(v, from_before<0x142, 0xa>(v));
    v = max(v, from_before<0x143, 0xc>(v));
    if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = v;
}
__device__ __forceinline__ int most_of(const int *lds)
{
    int v = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) v = max(v, lds[w]);
    return v;
}

// Assignment: deals the free pages.  One workgroup.
__global__ __launch_bounds__(1024) void k_pages_plan(PageShape s, Plan p, const int32_t *__restrict__ keep,
                                                     int32_t *status)
{
    __shared__ int lds[2][16];
    const int tid = threadIdx.x;
    if (p.head[BAD]) {
        if (tid == 0) *status = p.head[STATUS] = -1;
        return;
    }
    long long need = 0;
    int copies = 0;
    for (int r0 = 0; r0 < s.slots; r0 += 1024) {
        const int r = r0 + tid;
        int fresh = 0, copy = 0, have = 0, tail = -1;
        if (r < s.slots) {
            tail = p.tail[r];
            const bool stays = tail >= 0 && p.mark[tail] == r;
            copy = tail >= 0 && !stays;
            have = p.first[r] + stays;
            fresh = p.total[r] - have;
        }
        int all;
        const long long at = need + before(fresh, &all, lds[0]);
        need += all;
        const int c = copies + before(copy, &all, lds[1]);
        copies += all;
        if (r < s.slots) {
            p.fresh0[r] = (int)(at < INT_MAX ? at : INT_MAX);
            p.first[r] = have;
            if (copy) {
                p.from[c] = tail;
                p.to[c] = (int)(at < INT_MAX ? at : INT_MAX);   // a place in the list of free pages, for now
                const int rest = keep[r] % s.page_size;
                p.count[c] = (rest + s.block - 1) / s.block;
            }
        }
    }
    long long found = 0;
    for (int i0 = 0, b = 0; i0 < s.pages && found < need; i0 += 1024, b ^= 1) {
        const int i = i0 + tid;
        const int free = i < s.pages && p.mark[i] == FREE;
        int all;
        const int at = (int)found + before(free, &all, lds[b]);
        if (free) p.list[at] = i;
        found += all;
    }
    __syncthreads();
    const int left = (int)std::min<long long>(need > found ? need - found : 0, INT_MAX);
    if (left == 0)
        for (int c = tid; c < copies; c += 1024) p.to[c] = p.list[p.to[c]];
    if (tid == 0) {
        *status = p.head[STATUS] = left;
        p.head[COPIES] = copies;
    }
}

// Compaction: marks of all held pages, one wavefront to a slot.
__global__ __launch_bounds__(256) void k_pages_held(PageShape s, Plan p, const int32_t *__restrict__ table,
                                                    const int32_t *__restrict__ held)
{
    const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (r >= s.slots) return;
    const int n = held[r];
    bool bad = n < 0 || n > s.width;
    for (int i = lane; !bad && i < n; i += 64) {
        const int page = table[(size_t)r * s.width + i];
        if ((unsigned)page >= (unsigned)s.pages) {
            bad = true;
            break;
        }
        p.mark[page] = WHOLE;
    }
    if (bad) p.head[BAD] = 1;
}

// Compaction: held pages at and above their number go to the free ones below, in
// order.  One workgroup.
__global__ __launch_bounds__(1024) void k_pages_squeeze(PageShape s, Plan p, int32_t *status)
{
    __shared__ int lds[3][16];
    const int tid = threadIdx.x;
    if (p.head[BAD]) {
        if (tid == 0) *status = p.head[STATUS] = -1;
        return;
    }
    int mine = 0, n;
    for (int i = tid; i < s.pages; i += 1024) mine += p.mark[i] != FREE;
    before(mine, &n, lds[2]);
    int high = 0, low = 0, b = 0;
    for (int i0 = 0; i0 < s.pages; i0 += 1024) {
        const int i = i0 + tid;
        const bool used = i < s.pages && p.mark[i] != FREE;
        int all;
        if (i0 < n) {
            const bool hole = i < n && !used;
            const int at = low + before(hole, &all, lds[b ^= 1]);
            if (hole) p.to[at] = i;
            low += all;
        }
        if (i0 + 1024 > n) {
            const bool moves = i >= n && used;
            const int at = high + before(moves, &all, lds[b ^= 1]);
            if (moves) p.from[at] = i;
            high += all;
        }
    }
    __syncthreads();
    for (int i = tid; i < s.pages; i += 1024) p.mark[i] = i;
    __syncthreads();
    for (int c = tid; c < high; c += 1024) {
        p.mark[p.from[c]] = p.to[c];
        p.count[c] = s.blocks;
    }
    if (tid == 0) {
        p.head[COPIES] = high;
        *status = n;
        p.head[STATUS] = 0;
    }
}

// The whole plan, and the table, of a small pool: one workgroup, marks in LDS.
constexpr int SMALL_PAGES = 8192, SMALL_SLOTS = 1024, SMALL_TABLE = 1 << 17, SPARE = 512;

// Calls f(slot, i) for i < n, slot < slots, over the workgroup.
template <class F>
__device__ __forceinline__ void over_rows(int slots, int n, F &&f)
{
    if (n <= 0) return;
    const int total = slots * n;                       // at most SMALL_TABLE
#pragma unroll 4
    for (int k = threadIdx.x; k < total; k += 1024) f((unsigned)k / (unsigned)n, (unsigned)k % (unsigned)n);
}

__global__ __launch_bounds__(1024) void k_pages_small(PageShape s, Plan p, int32_t *__restrict__ table,
                                                      int32_t *__restrict__ held, const int32_t *__restrict__ src,
                                                      const int32_t *__restrict__ keep, const int32_t *__restrict__ hold,
                                                      int32_t *status)
{
    extern __shared__ int mark[];                      // [pages]
    __shared__ int from[SMALL_SLOTS], first[SMALL_SLOTS], taken[SMALL_SLOTS], total[SMALL_SLOTS], tail[SMALL_SLOTS],
        fresh0[SMALL_SLOTS], has[SMALL_SLOTS], spare[SPARE], lds[2][16], most[2][16], bad;
    const int tid = threadIdx.x, r = tid;
    const bool slot = r < s.slots;
    // one thread to a slot
    int f = -1, n = 0, m = 0, take = 0;
    if (slot) {
        f = src[r];
        n = keep[r];
        m = hold == nullptr ? n : hold[r];
        has[r] = held[r];
        tail[r] = -1;
    }
    if (tid == 0) bad = 0;
    for (int i = tid; i < s.pages; i += 1024) mark[i] = FREE;
    __syncthreads();
    bool wrong = f < -1 || f >= s.slots;
    if (wrong || f < 0) n = m = 0;
    else {
        const int h = has[f];
        wrong = h < 0 || h > s.width || n < 0 || n > (long long)h * s.page_size || m < n ||
                m > (long long)s.width * s.page_size;
        if (wrong) n = m = 0;
    }
    if (slot) {
        from[r] = f;
        first[r] = n / s.page_size;
        taken[r] = take = first[r] + (n > first[r] * s.page_size);
        total[r] = (int)(((long long)m + s.page_size - 1) / s.page_size);
    }
    if (wrong) bad = 1;
    note_most(take, most[0]);
    __syncthreads();
    const int span = most_of(most[0]);
    // entries that are taken: page i of slot r.  Few of them stay in registers.
    const bool few = s.slots * span <= 4096;
    int kept[4];
    const auto mark_page = [&](int r, int i, int page) {
        if ((unsigned)page >= (unsigned)s.pages) bad = 1;
        else if (i < first[r]) atomicMin(&mark[page], WHOLE);
        else {
            atomicMin(&mark[page], r);
            tail[r] = page;
        }
    };
    if (few) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int e = tid + 1024 * k, r = span > 0 ? (unsigned)e / (unsigned)span : s.slots, i = e - r * span;
            kept[k] = -1;
            if (r < s.slots && i < taken[r]) kept[k] = table[(size_t)from[r] * s.width + i];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int e = tid + 1024 * k, r = span > 0 ? (unsigned)e / (unsigned)span : s.slots, i = e - r * span;
            if (r < s.slots && i < taken[r]) mark_page(r, i, kept[k]);
        }
    } else {
        over_rows(s.slots, span, [&](int r, int i) {
            if (i >= taken[r]) return;
            const int page = table[(size_t)from[r] * s.width + i];
            mark_page(r, i, page);
            p.rows[(size_t)r * s.width + i] = page;
        });
    }
    __syncthreads();
    if (bad) {
        if (tid == 0) *status = p.head[STATUS] = -1;
        return;
    }
    int fresh = 0, copy = 0, have = 0, t = -1, need, copies;
    if (slot) {
        t = tail[r];
        const bool stays = t >= 0 && mark[t] == r;
        copy = t >= 0 && !stays;
        have = first[r] + stays;
        fresh = total[r] - have;                       // the table's entries bound the sum
    }
    note_most(fresh, most[1]);
    static_assert(SMALL_TABLE < 1 << 18 && SMALL_SLOTS < 1 << 13, "both counts in one word");
    const int both = before(fresh | copy << 18, &need, lds[0]), at = both & 0x3ffff, c = both >> 18;
    copies = need >> 18;
    need &= 0x3ffff;
    if (slot) {
        first[r] = have;
        fresh0[r] = at;
    }
    int found = 0;
    for (int i0 = 0, b = 1; i0 < s.pages && found < need; i0 += 4096, b ^= 1) {
        const int i = i0 + 4 * tid;
        bool free[4];
        int mine = 0, all;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            free[e] = i + e < s.pages && mark[i + e] == FREE;
            mine += free[e];
        }
        int k = found + before(mine, &all, lds[b]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (free[e]) {
                if (k < SPARE) spare[k] = i + e;
                else p.list[k] = i + e;
                ++k;
            }
        found += all;
    }
    __syncthreads();
    const int left = need > found ? need - found : 0, more = most_of(most[1]);
    if (left == 0) {
        const auto dealt = [&](int k) { return k < SPARE ? spare[k] : p.list[k]; };
        if (slot) held[r] = total[r];
        if (copy) {
            p.from[c] = t;
            p.to[c] = dealt(at);
            p.count[c] = (n % s.page_size + s.block - 1) / s.block;
        }
        if (few) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int e = tid + 1024 * k, r = span > 0 ? (unsigned)e / (unsigned)span : s.slots, i = e - r * span;
                if (r < s.slots && i < taken[r] && i < first[r]) table[(size_t)r * s.width + i] = kept[k];
            }
        } else {
            over_rows(s.slots, span, [&](int r, int i) {
                if (i < taken[r] && i < first[r]) table[(size_t)r * s.width + i] = p.rows[(size_t)r * s.width + i];
            });
        }
        over_rows(s.slots, more, [&](int r, int i) {
            if (first[r] + i < total[r]) table[(size_t)r * s.width + first[r] + i] = dealt(fresh0[r] + i);
        });
    }
    if (tid == 0) {
        *status = p.head[STATUS] = left;
        p.head[COPIES] = copies;
    }
}

__global__ __launch_bounds__(1024) void k_pages_small_squeeze(PageShape s, Plan p, int32_t *__restrict__ table,
                                                              const int32_t *__restrict__ held, int32_t *status)
{
    extern __shared__ int mark[];                      // [pages], then their new numbers
    __shared__ int has[SMALL_SLOTS], lds[3][16], most[16], bad;
    const int tid = threadIdx.x;
    int h = tid < s.slots ? held[tid] : 0;
    const bool wrong = h < 0 || h > s.width;
    if (wrong) h = 0;
    if (tid < s.slots) has[tid] = h;
    for (int i = tid; i < s.pages; i += 1024) mark[i] = FREE;
    note_most(wrong ? s.width + 1 : h, most);
    if (tid == 0) bad = 0;
    __syncthreads();
    const int span = most_of(most);
    if (span > s.width) {                              // a count outside the table, the same for all threads
        if (tid == 0) *status = p.head[STATUS] = -1;
        return;
    }
    over_rows(s.slots, span, [&](int r, int i) {
        if (i >= has[r]) return;
        const int page = table[(size_t)r * s.width + i];
        if ((unsigned)page >= (unsigned)s.pages) bad = 1;
        else mark[page] = WHOLE;
    });
    __syncthreads();
    if (bad) {
        if (tid == 0) *status = p.head[STATUS] = -1;
        return;
    }
    int mine = 0, n;
    for (int i = tid; i < s.pages; i += 1024) mine += mark[i] != FREE;
    before(mine, &n, lds[2]);
    int high = 0, low = 0;
    for (int i0 = 0, b = 0; i0 < s.pages; i0 += 1024, b ^= 1) {
        const int i = i0 + tid;
        const bool used = i < s.pages && mark[i] != FREE;
        const int hole = i < n && !used, moves = i >= n && used;
        int all;
        const int at = before(hole | moves << 16, &all, lds[b]);   // at most 1024 of each
        if (hole) p.to[low + (at & 0xffff)] = i;
        if (moves) p.from[high + (at >> 16)] = i;
        low += all & 0xffff;
        high += all >> 16;
    }
    __syncthreads();
    for (int i = tid; i < s.pages; i += 1024) mark[i] = i;
    __syncthreads();
    for (int c = tid; c < high; c += 1024) {
        mark[p.from[c]] = p.to[c];
        p.count[c] = s.blocks;
    }
    __syncthreads();
    over_rows(s.slots, span, [&](int r, int i) {
        if (i >= has[r]) return;
        const size_t at = (size_t)r * s.width + i;
        table[at] = mark[table[at]];
    });
    if (tid == 0) {
        p.head[COPIES] = high;
        *status = n;
        p.head[STATUS] = 0;
    }
}

// Carries out the plan: the table's rows (ROWS 1: an assignment's, 2: a
// compaction's, 0: none), and the copies of layers' pages: layer and k or v are the
// workgroup's y, pieces of 16 KB of the copied pages its x.
constexpr int PIECE = 1024;                            // 16-byte units
template <int ROWS>
__global__ __launch_bounds__(256) void k_pages_carry(PageShape s, Plan p, PageLayers layers, int32_t *__restrict__ table,
                                                     int32_t *__restrict__ held)
{
    if (p.head[STATUS] != 0) return;
    const int tid = threadIdx.x, l = blockIdx.y >> 1, which = blockIdx.y & 1;
    if (ROWS == 1 && blockIdx.y == 0)
        for (int r = blockIdx.x; r < s.slots; r += gridDim.x) {
            const int total = p.total[r], have = p.first[r], at = p.fresh0[r];
            for (int i = tid; i < total; i += 256)
                table[(size_t)r * s.width + i] = i < have ? p.rows[(size_t)r * s.width + i] : p.list[at + i - have];
            if (tid == 0) held[r] = total;
        }
    if (ROWS == 2 && blockIdx.y == 0)
        for (int r = blockIdx.x; r < s.slots; r += gridDim.x)
            for (int i = tid; i < held[r]; i += 256) {
                const int page = table[(size_t)r * s.width + i];
                table[(size_t)r * s.width + i] = p.mark[page];
            }
    uint8_t *base = (uint8_t *)(which ? layers.v[l] : layers.k[l]);
    uint8_t *sc = s.scales ? (which ? layers.vs[l] : layers.ks[l]) : nullptr;
    const size_t page = (size_t)s.nkv * s.blocks;      // blocks of a page
    const uint32_t block_units = (uint32_t)(s.row / 16);
    const uint32_t pieces = (uint32_t)((page * block_units + PIECE - 1) / PIECE);
    const unsigned long long items = (unsigned long long)p.head[COPIES] * pieces;
    for (unsigned long long it = blockIdx.x; it < items; it += gridDim.x) {
        const uint32_t c = (uint32_t)(it / pieces), piece = (uint32_t)(it - (unsigned long long)c * pieces);
        const uint32_t n = p.count[c], head_units = n * block_units, units = s.nkv * head_units;
        const size_t a = (size_t)p.from[c] * page, b = (size_t)p.to[c] * page;
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        const u32x4 *from = (const u32x4 *)(base + a * s.row);
        u32x4 *to = (u32x4 *)(base + b * s.row);
        u32x4 w[PIECE / 256];
        uint32_t at[PIECE / 256];
#pragma unroll
        for (int k = 0; k < PIECE / 256; ++k) {        // all of a thread's loads, then its stores
            const uint32_t i = min(piece * PIECE + 256 * k + tid, units - 1), h = i / head_units;
            at[k] = h * s.blocks * block_units + (i - h * head_units);
            w[k] = from[at[k]];
        }
#pragma unroll
        for (int k = 0; k < PIECE / 256; ++k)
            if (piece * PIECE + 256 * k + tid < units) to[at[k]] = w[k];
        if (sc != nullptr && piece == 0)
            for (uint32_t i = tid; i < s.nkv * n; i += 256) {
                const uint32_t o = i / n * s.blocks + i % n;
                sc[b + o] = sc[a + o];
            }
    }
}

}  // namespace

size_t pages_ws(int slots, int width, int pages)
{
    const size_t moves = (size_t)std::max(slots, pages);
    return 4 * (16 + 2 * up4(pages) + 4 * up4(slots) + 3 * up4(moves) + up4((size_t)slots * width));
}

hipError_t launch_pages(const PageShape &s, int32_t *table, int32_t *held, const int32_t *src, const int32_t *keep,
                        const int32_t *hold, int32_t *status, int n_layers, LayersOf layers, const void *of, void *ws,
                        hipStream_t st)
{
    const Plan p = plan_of(ws, s.slots, s.width, s.pages);
    const unsigned by4 = (unsigned)((s.slots + 3) / 4);
    const bool assign = src != nullptr;
    const bool small = s.pages <= SMALL_PAGES && s.slots <= SMALL_SLOTS && (long long)s.slots * s.width <= SMALL_TABLE;
    const size_t marks = sizeof(int) * (size_t)s.pages;
    if (small && assign) {
        KLAUNCH(k_pages_small, dim3(1), dim3(1024), marks, st, s, p, table, held, src, keep, hold, status);
    } else if (small) {
        KLAUNCH(k_pages_small_squeeze, dim3(1), dim3(1024), marks, st, s, p, table, held, status);
    } else {
        KLAUNCH(k_pages_clear, dim3(std::min((s.pages + 255) / 256, 1024)), dim3(256), 0, st, p, s.pages);
        if (assign) {
            KLAUNCH(k_pages_mark, dim3(by4), dim3(256), 0, st, s, p, table, held, src, keep, hold);
            KLAUNCH(k_pages_plan, dim3(1), dim3(1024), 0, st, s, p, keep, status);
        } else {
            KLAUNCH(k_pages_held, dim3(by4), dim3(256), 0, st, s, p, table, held);
            KLAUNCH(k_pages_squeeze, dim3(1), dim3(1024), 0, st, s, p, status);
        }
    }
    for (int l = 0; l < n_layers; l += COPY_LAYERS) {
        PageLayers pl;
        layers(of, l, &pl);
        // workgroups of a layer's k or v: as many as it could have copies, up to a
        // sixteenth of what the chip takes in a few rounds
        const long long pieces = ((long long)s.nkv * s.blocks * (s.row / 16) + PIECE - 1) / PIECE;
        const long long most = (assign ? s.slots : (s.pages + 1) / 2) * pieces;
        const dim3 grid((unsigned)std::max<long long>(1, std::min<long long>(most, 16384 / (2 * pl.n))), 2 * pl.n);
        if (small || l > 0) KLAUNCH((k_pages_carry<0>), grid, dim3(256), 0, st, s, p, pl, table, held);
        else if (assign) KLAUNCH((k_pages_carry<1>), grid, dim3(256), 0, st, s, p, pl, table, held);
        else KLAUNCH((k_pages_carry<2>), grid, dim3(256), 0, st, s, p, pl, table, held);
    }
    return hipGetLastError();
}

}  // namespace corun
