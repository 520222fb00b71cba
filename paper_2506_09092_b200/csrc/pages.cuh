// The pages of a cache: copies of whole pages, and the book of which sequence holds which pages.
//
// Bound: the copies by HBM (each byte read and written once); the bookkeeping by latency (a few thousand
// words), so it is done in as few dependent steps and launches as its order allows.  A page is free if nobody holds it,
// there is no list of free pages that could disagree: the lowest free pages are found by one pass over refs.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/cudallm_cache.h"
#include "ptx.cuh"

namespace cudallm {

struct Book {
    int *refs, *lens, *table, *turn;
    long long stride;
    int pages, rows, slots, cols, cap;         // cap: states that a row of the table holds
};
__device__ __forceinline__ int book_len(const Book &b, int slot) { return min(max(b.lens[slot], 0), b.cap); }
__device__ __forceinline__ int pages_of(const Book &b, int len) { return (int)(((unsigned)len + b.rows - 1) / (unsigned)b.rows); }
__device__ __forceinline__ bool is_page(const Book &b, int page) { return (unsigned)page < (unsigned)b.pages; }
// (words that atomics of other CTAs change are read from L2)
__device__ __forceinline__ int refs_now(const Book &b, int page) { return __ldcg(b.refs + page); }

// ------------------------------------------------------------------- copies --
constexpr int kPoolsPerLaunch = 120;           // their descriptions travel in the kernel's parameters
struct PoolList { cudallm_page_pool at[kPoolsPerLaunch]; };
constexpr int kCopyThreads = 256;
constexpr int kCopyUnroll = 4;
constexpr int kCopyChunk = kCopyThreads * 16 * kCopyUnroll;    // bytes of a page that a CTA copies at a time

struct CopyParams {
    const int *src, *dst;
    const int *count;                          // how many pairs there are, or null: n
    long long n;
    int pages, pools, chunks;                  // chunks of the largest pool's page
    // compaction: numbers of moved pages are replaced in the table, from page *first_moved on
    Book book;
    const int *remap, *first_moved;
};

// Units of (pair, pool, chunk) in order.  A thread has four 16-byte loads in flight.
__global__ void __launch_bounds__(kCopyThreads)
pages_copy_kernel(const CopyParams p, const __grid_constant__ PoolList pools)
{
    grid_launch_dependents();
    grid_dependency_wait();
    if (p.remap) {
        const int first = *p.first_moved;
        for (int s = blockIdx.x; s < p.book.slots; s += gridDim.x) {
            const int held = pages_of(p.book, book_len(p.book, s));
            int *row = p.book.table + s * p.book.stride;
            for (int c = threadIdx.x; c < held; c += kCopyThreads) {
                const int page = row[c];
                if (page >= first && page < p.pages) row[c] = p.remap[page];
            }
        }
    }
    const long long pairs = p.count ? min((long long)*p.count, p.n) : p.n;
    const unsigned per_pair = (unsigned)(p.pools * p.chunks);
    const long long units = pairs * per_pair;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const long long pair = u / per_pair;
        const unsigned rest = (unsigned)(u - pair * per_pair), pool = rest / p.chunks, chunk = rest - pool * p.chunks;
        const int src = p.src[pair], dst = p.dst[pair];
        if ((unsigned)src >= (unsigned)p.pages || (unsigned)dst >= (unsigned)p.pages || src == dst) continue;
        const cudallm_page_pool &pl = pools.at[pool];
        const long long first = (long long)chunk * kCopyChunk + threadIdx.x * 16;
        const uint8_t *from = static_cast<const uint8_t *>(pl.data) + src * pl.stride;
        uint8_t *to = static_cast<uint8_t *>(pl.data) + dst * pl.stride;
        uint4 v[kCopyUnroll];
#pragma unroll
        for (int i = 0; i < kCopyUnroll; ++i) {
            const long long at = first + i * kCopyThreads * 16;
            if (at < pl.bytes) v[i] = __ldcs(reinterpret_cast<const uint4 *>(from + at));
        }
#pragma unroll
        for (int i = 0; i < kCopyUnroll; ++i) {
            const long long at = first + i * kCopyThreads * 16;
            if (at < pl.bytes) __stcs(reinterpret_cast<uint4 *>(to + at), v[i]);
        }
    }
}

// --------------------------------------------------------------------- fork --
// Two launches, since a slot may be read by one entry and overwritten by another: the sources' rows go to scratch and
// their pages get one holder more; then the old rows are given up and the new ones put in.  One CTA an entry.
struct ForkParams {
    Book book;
    const int *src, *dst;
    int n;
    int *staged_len;                           // n: the length that dst[i] gets, -1: entry i changes nothing
    int *staged;                               // n rows of cols page numbers
};
__global__ void __launch_bounds__(256)
fork_stage_kernel(const ForkParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const Book &bk = p.book;
    for (int i = blockIdx.x; i < p.n; i += gridDim.x) {
        const int src = p.src[i], dst = p.dst[i];
        bool live = (unsigned)src < (unsigned)bk.slots && (unsigned)dst < (unsigned)bk.slots;
        if (live) {                                                // (the same for all threads)
            bool first = true;
            for (int j = threadIdx.x; j < i; j += 256) first &= !(p.dst[j] == dst && (unsigned)p.src[j] < (unsigned)bk.slots);
            live = __syncthreads_and(first) && src != dst;
        }
        const int len = live ? book_len(bk, src) : -1;
        if (threadIdx.x == 0) p.staged_len[i] = len;
        if (!live) continue;
        const int held = pages_of(bk, len);
        const int *row = bk.table + src * bk.stride;
        int *to = p.staged + (long long)i * bk.cols;
        for (int c = threadIdx.x; c < held; c += 256) {
            const int page = row[c];
            to[c] = page;
            if (is_page(bk, page)) atomicAdd(bk.refs + page, 1);
        }
    }
}
__global__ void __launch_bounds__(256)
fork_put_kernel(const ForkParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const Book &bk = p.book;
    for (int i = blockIdx.x; i < p.n; i += gridDim.x) {
        const int len = p.staged_len[i];
        if (len < 0) continue;
        const int dst = p.dst[i], had = pages_of(bk, book_len(bk, dst)), held = pages_of(bk, len);
        int *row = bk.table + dst * bk.stride;
        const int *from = p.staged + (long long)i * bk.cols;
        for (int c = threadIdx.x; c < max(had, held); c += 256) {
            if (c < had) {
                const int page = row[c];
                if (is_page(bk, page)) atomicSub(bk.refs + page, 1);
            }
            if (c < held) row[c] = from[c];
        }
        __syncthreads();                                           // every thread has read the old length
        if (threadIdx.x == 0) bk.lens[dst] = len;
    }
}

// -------------------------------------------------- counting within a block --
constexpr int kBookThreads = 1024;
// Sum of v over the threads below this one; total: over all.  All of the block's 1024 threads call it.
__device__ __forceinline__ long long block_before(long long v, long long &total)
{
    __shared__ long long warps[33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long upto = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const long long x = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += x;
    }
    if (lane == 31) warps[warp] = upto;
    __syncthreads();
    if (warp == 0) {
        long long w = warps[lane];
        const long long mine = w;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const long long x = __shfl_up_sync(0xffffffffu, w, d);
            if (lane >= d) w += x;
        }
        warps[lane] = w - mine;
        if (lane == 31) warps[32] = w;
    }
    __syncthreads();
    const long long before = warps[warp] + upto - v;
    total = warps[32];
    __syncthreads();                                               // (it may be called again at once)
    return before;
}
// Two counts in one word: at most 2^16 entries that need at most 2^20 + 1 pages each, and at most 2^20 of the other.
constexpr int kLowBits = 42;
__device__ __forceinline__ long long pack2(int lo, int hi) { return (long long)hi << kLowBits | lo; }
__device__ __forceinline__ long long low_of(long long v) { return v & ((1LL << kLowBits) - 1); }
__device__ __forceinline__ int high_of(long long v) { return (int)(v >> kLowBits); }

// Which of pages first .. first + 15 are held, a bit each; pages that do not exist count as held.
__device__ __forceinline__ uint32_t held16(const Book &b, int first)
{
    uint32_t bits = 0;
    if (first + 16 <= b.pages) {
        int4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __ldcg(reinterpret_cast<const int4 *>(b.refs + first) + k);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            bits |= ((v[k].x != 0) | (v[k].y != 0) << 1 | (v[k].z != 0) << 2 | (v[k].w != 0) << 3) << 4 * k;
    } else {
        bits = 0xffff;
        for (int i = 0; i < 16 && first + i < b.pages; ++i)
            if (refs_now(b, first + i) == 0) bits &= ~(1u << i);
    }
    return bits;
}

// ------------------------------------------------------------------- resize --
struct ResizeParams {
    Book book;
    const int *slot_of, *want;
    int n;
    int *result;
    // scratch
    int *count;                                // pairs to copy
    int *src, *dst;                            // n
    int *state;                                // n: the length before, -1: passed over, -2: too long
    int *start;                                // n: first of its new pages among all, bit 31: it takes a copy
    int *fresh;                                // pages: the lowest free ones
    int *claims, *claimer;                     // pages: growing sequences that share a tail, the first of them
};
constexpr int kEntryLanes = 8;                 // lanes that work on an entry together

__device__ __forceinline__ int slot_at(const ResizeParams &p, int i) { return p.slot_of ? p.slot_of[i] : i; }

// First all CTAs give back the pages of sequences that become shorter; the last of them to be done does the rest, which
// has an order: shared tails, how many pages are needed, which are free, who gets which.  If they do not suffice, it
// takes what was given back again.
__global__ void __launch_bounds__(kBookThreads)
pages_resize_kernel(const ResizeParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const Book &bk = p.book;
    const int tid = threadIdx.x, sub = tid % kEntryLanes;
    const int groups = kBookThreads / kEntryLanes;
    const unsigned quad = 0xffu << (tid & 31 & ~(kEntryLanes - 1));        // the lanes of this thread's entry
    for (int i = blockIdx.x * groups + tid / kEntryLanes; i < p.n; i += gridDim.x * groups) {
        const int slot = slot_at(p, i), want = p.want[i];
        int state = -1;
        if ((unsigned)slot < (unsigned)bk.slots && want >= 0) {
            bool first = true;
            if (p.slot_of)
                for (int j = sub; j < i; j += kEntryLanes) first &= !(p.slot_of[j] == slot && p.want[j] >= 0);
            if (__all_sync(quad, first)) {
                const int len = book_len(bk, slot);
                state = want > bk.cap ? -2 : len;
                if (want < len) {
                    const int *row = bk.table + slot * bk.stride;
                    const int had = pages_of(bk, len);
                    for (int c = pages_of(bk, want) + sub; c < had; c += kEntryLanes)
                        if (is_page(bk, row[c])) atomicSub(bk.refs + row[c], 1);
                }
            }
        }
        if (sub == 0) p.state[i] = state;
    }
    if (gridDim.x > 1) {
        __shared__ bool last;
        __threadfence();
        __syncthreads();
        if (tid == 0) {
            last = atomicAdd(bk.turn, 1) == (int)gridDim.x - 1;
            if (last) *bk.turn = 0;
            __threadfence();
        }
        __syncthreads();
        if (!last) return;
    } else {
        __threadfence();
        __syncthreads();
    }

    // the tail that an entry's new tokens go into, if others hold it too; -1: none
    auto shared_tail = [&](int i, int state) {
        if (state <= 0 || p.want[i] <= state || state % bk.rows == 0) return -1;
        const int page = bk.table[slot_at(p, i) * bk.stride + pages_of(bk, state) - 1];
        return is_page(bk, page) && refs_now(bk, page) > 1 ? page : -1;
    };
    bool tails = false, too_long = false;
    for (int i = tid; i < p.n; i += kBookThreads) {
        const int state = __ldcg(p.state + i), page = shared_tail(i, state);
        too_long |= state == -2;
        if (page >= 0) {
            tails = true;
            __stcg(p.claims + page, 0);
            __stcg(p.claimer + page, 0x7fffffff);
        }
    }
    tails = __syncthreads_or(tails);
    if (tails) {
        __threadfence();
        __syncthreads();
        for (int i = tid; i < p.n; i += kBookThreads) {
            const int page = shared_tail(i, __ldcg(p.state + i));
            if (page < 0) continue;
            atomicAdd(p.claims + page, 1);
            atomicMin(p.claimer + page, i);
        }
        __threadfence();
        __syncthreads();
    }
    // new pages and copies of the entries before each
    long long need = 0;
    for (int base = 0; base < p.n; base += kBookThreads) {
        const int i = base + tid;
        int pages = 0, copy = 0, page = -1;
        if (i < p.n) {
            const int state = __ldcg(p.state + i);
            page = tails ? shared_tail(i, state) : -1;
            copy = page >= 0 && !(__ldcg(p.claims + page) == refs_now(bk, page) && __ldcg(p.claimer + page) == i);
            if (state >= 0) pages = min(copy + max(pages_of(bk, p.want[i]) - pages_of(bk, state), 0), bk.pages + 1);
        }
        long long total;
        const long long before = need + block_before(pack2(pages, copy), total);
        if (i < p.n) {
            p.start[i] = (int)(low_of(before) & 0x7fffffff) | (copy ? (int)0x80000000 : 0);
            if (copy) {                                            // (where the copy goes is filled in below)
                p.src[high_of(before)] = page;
                p.dst[high_of(before)] = i;
            }
        }
        need += total;
    }
    const long long pages = low_of(need);
    const int copies = high_of(need);
    int found = 0;
    const bool refused = __syncthreads_or(too_long);
    if (!refused)                                                  // (more than there are need not be found to be refused)
        for (int base = 0; base < bk.pages && found < pages; base += kBookThreads * 16) {
            const int first = base + tid * 16;
            uint32_t free = first < bk.pages ? ~held16(bk, first) & 0xffff : 0;
            long long total;
            int at = found + (int)block_before(__popc(free), total);
            for (; free; free &= free - 1) p.fresh[at++] = first + __ffs(free) - 1;
            found += (int)total;
        }
    __threadfence();
    __syncthreads();
    const bool done = !refused && found >= pages;
    if (tid == 0) {
        if (p.result) *p.result = refused ? -1 : done ? 0 : (int)min(pages - found, 0x7fffffffLL);
        *p.count = done ? copies : 0;
    }
    for (int i = tid / kEntryLanes; i < p.n; i += groups) {
        const int state = __ldcg(p.state + i);
        if (state == -1) continue;
        const int slot = slot_at(p, i), want = p.want[i];
        int *row = bk.table + slot * bk.stride;
        if (!done) {
            if (state >= 0)
                for (int c = pages_of(bk, want) + sub; c < pages_of(bk, state); c += kEntryLanes)
                    if (is_page(bk, row[c])) atomicAdd(bk.refs + row[c], 1);
            continue;
        }
        const int mark = p.start[i], had = pages_of(bk, state), held = pages_of(bk, want);
        const int copy = mark < 0, start = mark & 0x7fffffff;
        if (sub == 0) {
            if (copy) {
                const int page = p.fresh[start];
                atomicSub(bk.refs + row[had - 1], 1);
                bk.refs[page] = 1;
                row[had - 1] = page;
            }
            bk.lens[slot] = want;
        }
        for (int c = had + sub; c < held; c += kEntryLanes) {
            const int page = p.fresh[start + copy + c - had];
            row[c] = page;
            bk.refs[page] = 1;
        }
    }
    if (done)
        for (int k = tid; k < copies; k += kBookThreads) p.dst[k] = p.fresh[p.start[p.dst[k]] & 0x7fffffff];
}

// ------------------------------------------------------------------ compact --
struct CompactParams {
    Book book;
    int *used;
    // scratch
    int *count, *first_moved;                  // pages to move; pages in use
    int *src, *dst;                            // pages each
    int *remap;                                // pages: where a page from first_moved on goes
};
// One CTA.  Which pages are held goes to shared memory as bits in one pass over refs; the k-th held one above the
// number of pages in use and the k-th free one below it become pair k.
__global__ void __launch_bounds__(kBookThreads)
pages_compact_kernel(const CompactParams p)
{
    extern __shared__ uint16_t held[];
    grid_launch_dependents();
    grid_dependency_wait();
    const Book &bk = p.book;
    const int tid = threadIdx.x, words = (bk.pages + 15) / 16;
    int mine = 0;
    for (int w = tid; w < words; w += kBookThreads) {
        uint32_t bits = held16(bk, w * 16);
        if (w * 16 + 16 > bk.pages) bits &= (1u << (bk.pages - w * 16)) - 1;
        held[w] = (uint16_t)bits;
        mine += __popc(bits);
    }
    long long total;
    block_before(mine, total);                                     // (and the bits are there for all)
    const int used = (int)total;
    long long at = 0;
    for (int base = 0; base < words; base += kBookThreads) {
        const int w = base + tid, first = w * 16;
        uint32_t holes = 0, movers = 0;
        if (w < words) {
            const uint32_t exist = first + 16 > bk.pages ? (1u << (bk.pages - first)) - 1 : 0xffffu;
            const uint32_t below = used <= first ? 0u : used >= first + 16 ? 0xffffu : (1u << (used - first)) - 1;
            holes = ~held[w] & exist & below;
            movers = held[w] & ~below;
            for (uint32_t rest = exist & ~below & ~movers; rest; rest &= rest - 1)
                p.remap[first + __ffs(rest) - 1] = first + __ffs(rest) - 1;
        }
        long long sum;
        const long long before = at + block_before(pack2(__popc(holes), __popc(movers)), sum);
        at += sum;
        for (int k = (int)low_of(before); holes; holes &= holes - 1) p.dst[k++] = first + __ffs(holes) - 1;
        for (int k = high_of(before); movers; movers &= movers - 1) p.src[k++] = first + __ffs(movers) - 1;
    }
    const int moves = high_of(at);
    __threadfence_block();
    __syncthreads();
    for (int k = tid; k < moves; k += kBookThreads) {
        const int src = p.src[k], dst = p.dst[k];
        p.remap[src] = dst;
        bk.refs[dst] = bk.refs[src];
        bk.refs[src] = 0;
    }
    if (tid == 0) {
        *p.count = moves;
        *p.first_moved = used;
        if (p.used) *p.used = used;
    }
}

}  // namespace cudallm
