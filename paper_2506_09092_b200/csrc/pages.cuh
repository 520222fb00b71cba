// The pages of a cache: copies of whole pages, and the book of which sequence holds which pages.
//
// Bound: the copies by HBM (each byte read and written once); the bookkeeping by latency (a few thousand
// words), so it is done in as few dependent steps and launches as its order allows.  A page is free if nobody holds it,
// there is no list of free pages that could disagree: the lowest free pages are found by one pass over refs.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/cudallm_cache.h"
#include "mma_sync.cuh"
#include "ptx.cuh"

namespace cudallm {

struct Book {
    int *refs, *lens, *table;
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
constexpr int kCopyUnroll = 8;
constexpr int kCopyChunk = 32 * 16 * kCopyUnroll;              // bytes of a page that a warp copies at a time

struct CopyParams {
    const int *src, *dst;
    const int *count;                          // how many pairs there are, or null: n
    long long n;
    int pages, pools, chunks;                  // chunks of the largest pool's page
    // compaction: numbers of moved pages are replaced in the table, from page *first_moved on
    Book book;
    const int *remap, *first_moved;
};

// Units of (pair, pool, chunk) in order, a warp each, so that short pages leave no threads idle; a thread has eight 16-byte
// loads in flight.  1024 pages of 32 KiB in 16 pools (1.07 GB moved): 170 us, 6.30 TB/s (4000 of them: 6.40); with four loads
// 179 us, with sixteen 174, with a CTA's worth of each page at a time and four loads 190, on half of the CTAs 176.
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
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (long long u = blockIdx.x * (kCopyThreads / 32) + warp; u < units; u += gridDim.x * (kCopyThreads / 32)) {
        const long long pair = u / per_pair;
        const unsigned rest = (unsigned)(u - pair * per_pair), pool = rest / p.chunks, chunk = rest - pool * p.chunks;
        const int src = p.src[pair], dst = p.dst[pair];
        if ((unsigned)src >= (unsigned)p.pages || (unsigned)dst >= (unsigned)p.pages || src == dst) continue;
        const cudallm_page_pool &pl = pools.at[pool];
        const long long first = (long long)chunk * kCopyChunk + lane * 16;
        const uint8_t *from = static_cast<const uint8_t *>(pl.data) + src * pl.stride;
        uint8_t *to = static_cast<uint8_t *>(pl.data) + dst * pl.stride;
        uint4 v[kCopyUnroll];
#pragma unroll
        for (int i = 0; i < kCopyUnroll; ++i) {
            const long long at = first + i * 512;
            if (at < pl.bytes) v[i] = __ldcs(reinterpret_cast<const uint4 *>(from + at));
        }
#pragma unroll
        for (int i = 0; i < kCopyUnroll; ++i) {
            const long long at = first + i * 512;
            if (at < pl.bytes) __stcs(reinterpret_cast<uint4 *>(to + at), v[i]);
        }
    }
}

// --------------------------------------------------------------------- fork --
constexpr int kBookThreads = 1024;
constexpr int kBookCluster = 8;                // CTAs of a launch that changes a book, at most: one cluster

struct ForkParams {
    Book book;
    const int *src, *dst;
    int n;
    int *staged_len;                           // n: the length that dst[i] gets, -1: entry i changes nothing
    int *staged;                               // n rows of cols page numbers
    int chunks;                                // pieces of kForkCols columns in a row of the table
};
constexpr int kForkCols = 256;

// A slot may be read by one entry and overwritten by another, so the sources' rows first go to scratch, their pages
// getting one holder more; then, behind a barrier of the whole cluster, the old rows are given up and the
// new ones put in.  A warp works on 256 columns of an entry at a time.  Bound: the latency of four dependent reads and two cluster
// barriers; 256 sequences of 11 pages: 7.8 us under a profiler on eight CTAs (8 sequences on one: 5.5).
__global__ void __launch_bounds__(kBookThreads, 1)
pages_fork_kernel(const ForkParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const Book &bk = p.book;
    const int lane = threadIdx.x & 31, warp = (blockIdx.x * kBookThreads + threadIdx.x) >> 5, warps = gridDim.x * kBookThreads / 32;
    const long long tasks = (long long)p.n * p.chunks;
    for (long long k = warp; k < tasks; k += warps) {
        const int i = (int)(k / p.chunks), c0 = (int)(k - (long long)i * p.chunks) * kForkCols;
        const int src = p.src[i], dst = p.dst[i];
        bool live = (unsigned)src < (unsigned)bk.slots && (unsigned)dst < (unsigned)bk.slots && src != dst;
        const int len = live ? book_len(bk, src) : -1, held = live ? pages_of(bk, len) : 0;
        if (c0 > 0 && c0 >= held) continue;
        bool taken = false;                                        // (no early end: the loads of several rounds run side by side)
#pragma unroll 4
        for (int j = lane; j < i; j += 32) taken |= p.dst[j] == dst & (unsigned)p.src[j] < (unsigned)bk.slots;
        live &= !taken;
        live = __all_sync(0xffffffffu, live);
        if (c0 == 0 && lane == 0) p.staged_len[i] = live ? len : -1;
        if (!live) continue;
        const int *row = bk.table + src * bk.stride;
        int *to = p.staged + (long long)i * bk.cols;
#pragma unroll
        for (int m = 0; m < kForkCols / 32; ++m) {
            const int c = c0 + m * 32 + lane;
            if (c >= held) break;
            const int page = row[c];
            to[c] = page;
            if (is_page(bk, page)) atomicAdd(bk.refs + page, 1);
        }
    }
    cluster_sync_all();
    for (long long k = warp; k < tasks; k += warps) {
        const int i = (int)(k / p.chunks), c0 = (int)(k - (long long)i * p.chunks) * kForkCols;
        const int len = __ldcg(p.staged_len + i);
        if (len < 0) continue;
        const int dst = p.dst[i], had = pages_of(bk, book_len(bk, dst)), held = pages_of(bk, len);
        int *row = bk.table + dst * bk.stride;
        const int *from = p.staged + (long long)i * bk.cols;
#pragma unroll
        for (int m = 0; m < kForkCols / 32; ++m) {
            const int c = c0 + m * 32 + lane;
            if (c >= max(had, held)) break;
            if (c < had) {
                const int page = row[c];
                if (is_page(bk, page)) atomicSub(bk.refs + page, 1);
            }
            if (c < held) row[c] = __ldcg(from + c);
        }
    }
    cluster_sync_all();                                            // every warp has read the old lengths
    for (int i = blockIdx.x * kBookThreads + threadIdx.x; i < p.n; i += gridDim.x * kBookThreads) {
        const int len = __ldcg(p.staged_len + i);
        if (len >= 0) bk.lens[p.dst[i]] = len;
    }
}

// -------------------------------------------------- counting within a block --
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
// Two counts in one word: at most 2^14 entries that need fewer than 2^31 pages each, and at most 2^14 copies (or, in a compaction,
// at most 2^20 of either).
constexpr int kLowBits = 45;
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
constexpr int kFreshShared = 2048;             // up to so many new pages pass through shared memory

struct ResizeEntry {
    int slot, want, state;                     // (as in the scratch)
    int tail;                                  // the page that its new tokens go into, if others hold it too; -1: none
};

// Which of several entries with one key (a slot, a page) comes first, and how many there are: a table in shared memory for
// the at most 1024 entries of a list that one thread each works on.
struct KeyTable {
    static constexpr int kSize = 2048;
    int key[kSize], first[kSize], count[kSize];
    __device__ __forceinline__ void clear()
    {
        for (int i = threadIdx.x; i < kSize; i += kBookThreads) {
            key[i] = -1;
            first[i] = 0x7fffffff;
            count[i] = 0;
        }
    }
    __device__ __forceinline__ int add(int k, int entry)
    {
        int at = (unsigned)k * 2654435761u >> 21;
        for (;; at = (at + 1) % kSize) {                           // (half of the places stay free)
            const int old = atomicCAS(key + at, -1, k);
            if (old == -1 || old == k) break;
        }
        atomicMin(first + at, entry);
        atomicAdd(count + at, 1);
        return at;
    }
};

// First all CTAs of the cluster give back the pages of sequences that become shorter; then the first does the rest, which
// has an order: shared tails, how many pages are needed, which are free, who gets which.  If they do not suffice, it
// takes what was given back again.  ONE: up to 1024 entries, a thread each, in registers and shared
// memory; longer lists go through the scratch.  Bound: latency (list -> length -> last page -> its holders, then the counting
// within a block, twice): 256 sequences, 256 new pages: 11.0 us under a profiler, 8 sequences 10.2, of which the launch is four.
template <bool ONE>
__global__ void __launch_bounds__(kBookThreads, 1)
pages_resize_kernel(const ResizeParams p)
{
    __shared__ KeyTable table;
    __shared__ int s_fresh[kFreshShared];
    __shared__ int s_slot[ONE ? kBookThreads : 1], s_want[ONE ? kBookThreads : 1], s_state[ONE ? kBookThreads : 1];
    const Book &bk = p.book;
    const int tid = threadIdx.x, sub = tid % kEntryLanes, groups = kBookThreads / kEntryLanes;
    if constexpr (ONE) {
        table.clear();
        __syncthreads();
    }
    grid_launch_dependents();
    grid_dependency_wait();
    // gives back (sign -1), or takes again, the pages behind an entry's new end
    auto give = [&](int slot, int want, int state, int sign) {
        const int *row = bk.table + slot * bk.stride;
        const int had = pages_of(bk, state);
        for (int c = pages_of(bk, want) + sub; c < had; c += kEntryLanes)
            if (is_page(bk, row[c])) atomicAdd(bk.refs + row[c], sign);
    };
    auto slot_at = [&](int i) { return p.slot_of ? p.slot_of[i] : i; };
    ResizeEntry mine{-1, 0, -1, -1};
    bool gives = false;
    uint32_t early = 0xffff;                                       // the first pages: asked for beside the list
    if constexpr (ONE) {
        int place = -1;
        if (tid < p.n) {
            mine.slot = slot_at(tid);
            mine.want = p.want[tid];
        }
        if (tid * 16 < bk.pages) early = held16(bk, tid * 16);
        if (tid < p.n) {
            if ((unsigned)mine.slot < (unsigned)bk.slots && mine.want >= 0) {
                mine.state = mine.want > bk.cap ? -2 : book_len(bk, mine.slot);
                if (p.slot_of) place = table.add(mine.slot, tid);
            }
        }
        __syncthreads();
        if (place >= 0 && table.first[place] != tid) mine.state = -1;
        s_slot[tid] = mine.slot;
        s_want[tid] = mine.want;
        s_state[tid] = mine.state;
        gives = __syncthreads_or(mine.state > mine.want && pages_of(bk, mine.state) > pages_of(bk, mine.want));
        table.clear();
        if (gives)
            for (int i = blockIdx.x * groups + tid / kEntryLanes; i < p.n; i += gridDim.x * groups)
                if (s_state[i] > s_want[i]) give(s_slot[i], s_want[i], s_state[i], -1);
    } else {
        const unsigned quad = 0xffu << (tid & 31 & ~(kEntryLanes - 1));    // the lanes of this thread's entry
        for (int i = blockIdx.x * groups + tid / kEntryLanes; i < p.n; i += gridDim.x * groups) {
            const int slot = slot_at(i), want = p.want[i];
            int state = -1;
            if ((unsigned)slot < (unsigned)bk.slots && want >= 0) {
                bool first = true;
                if (p.slot_of)
                    for (int j = sub; j < i; j += kEntryLanes) first &= !(p.slot_of[j] == slot && p.want[j] >= 0);
                if (__all_sync(quad, first)) {
                    state = want > bk.cap ? -2 : book_len(bk, slot);
                    if (state > want) give(slot, want, state, -1);
                }
            }
            if (sub == 0) p.state[i] = state;
        }
        gives = true;
    }
    if (gridDim.x > 1) {
        __threadfence();
        cluster_sync_all();
        if (blockIdx.x != 0) return;
    } else if (gives) {
        __threadfence();
    }
    __syncthreads();

    auto find_tail = [&](const ResizeEntry &e) {
        if (e.state <= 0 || e.want <= e.state || e.state % bk.rows == 0) return -1;
        const int page = bk.table[e.slot * bk.stride + pages_of(bk, e.state) - 1];
        return is_page(bk, page) && refs_now(bk, page) > 1 ? page : -1;
    };
    auto each = [&](auto f) {
        if constexpr (ONE) {
            if (tid < p.n) f(tid, mine);
        } else {
            for (int i = tid; i < p.n; i += kBookThreads) {
                ResizeEntry e{slot_at(i), p.want[i], __ldcg(p.state + i), -1};
                e.tail = find_tail(e);
                f(i, e);
            }
        }
    };
    // growing sequences that share a tail: how many, and the first of them
    bool too_long = false, tails = false;
    int claim = -1;                                                // (ONE: this entry's place in the table)
    if constexpr (ONE) {
        mine.tail = find_tail(mine);
        too_long = mine.state == -2;
        if (mine.tail >= 0) claim = table.add(mine.tail, tid);
        __syncthreads();
    } else {
        each([&](int, ResizeEntry &e) {
            too_long |= e.state == -2;
            if (e.tail < 0) return;
            tails = true;
            __stcg(p.claims + e.tail, 0);
            __stcg(p.claimer + e.tail, 0x7fffffff);
        });
        tails = __syncthreads_or(tails);
        if (tails) {
            __threadfence();
            __syncthreads();
            each([&](int i, ResizeEntry &e) {
                if (e.tail < 0) return;
                atomicAdd(p.claims + e.tail, 1);
                atomicMin(p.claimer + e.tail, i);
            });
            __threadfence();
            __syncthreads();
        }
    }
    // new pages and copies of the entries before each
    long long need = 0;
    int start = 0, copy = 0;                                       // (ONE: of this entry)
    for (int base = 0; base < p.n; base += kBookThreads) {
        const int i = base + tid;
        ResizeEntry e{-1, 0, -1, -1};
        if constexpr (ONE) {
            e = mine;
        } else if (i < p.n) {
            e = ResizeEntry{slot_at(i), p.want[i], __ldcg(p.state + i), -1};
            if (tails) e.tail = find_tail(e);
        }
        int pages = 0;
        copy = 0;
        if (e.tail >= 0) {
            const int sharers = ONE ? table.count[claim] : __ldcg(p.claims + e.tail);
            const int first = ONE ? table.first[claim] : __ldcg(p.claimer + e.tail);
            copy = !(sharers == refs_now(bk, e.tail) && first == i);
        }
        if (e.state >= 0) pages = copy + max(pages_of(bk, e.want) - pages_of(bk, e.state), 0);
        long long total;
        const long long before = need + block_before(pack2(pages, copy), total);
        start = (int)(low_of(before) & 0x7fffffff);
        if (!ONE && i < p.n) p.start[i] = start | (copy ? (int)0x80000000 : 0);
        if (copy) {                                                // (where the copy goes is filled in below)
            p.src[high_of(before)] = e.tail;
            p.dst[high_of(before)] = start;
        }
        need += total;
    }
    const long long pages = low_of(need);
    const int copies = high_of(need);
    int found = 0;
    int *const fresh = pages <= kFreshShared ? s_fresh : p.fresh;
    const bool refused = __syncthreads_or(too_long);
    if (!refused)                                                  // (more than there are need not be found to be refused)
        for (int base = 0; base < bk.pages && found < pages; base += kBookThreads * 16) {
            const int first = base + tid * 16;
            uint32_t free = first < bk.pages ? ~(ONE && !gives && base == 0 ? early : held16(bk, first)) & 0xffff : 0;
            long long total;
            int at = found + (int)block_before(__popc(free), total);
            for (; free && at < pages; free &= free - 1) fresh[at++] = first + __ffs(free) - 1;
            found += (int)total;
        }
    __syncthreads();                                               // (this CTA reads what it has written)
    const bool done = !refused && found >= pages;
    if (tid == 0) {
        if (p.result) *p.result = refused ? -1 : done ? 0 : (int)min(pages - found, 0x7fffffffLL);
        *p.count = done ? copies : 0;
    }
    if (!done) {
        for (int i = tid / kEntryLanes; i < p.n && gives; i += groups) {
            const int state = ONE ? s_state[i] : __ldcg(p.state + i), want = ONE ? s_want[i] : p.want[i];
            if (state >= 0) give(ONE ? s_slot[i] : slot_at(i), want, state, 1);
        }
        return;
    }
    // Every entry's lanes put in its new pages.  (ONE: what its thread knows goes round by shuffle.)
    auto put = [&](int slot, int want, int state, int first, int takes) {
        int *row = bk.table + slot * bk.stride;
        const int had = pages_of(bk, state), held = pages_of(bk, want);
        if (sub == 0) {
            if (takes) {
                const int page = fresh[first];
                atomicSub(bk.refs + row[had - 1], 1);
                bk.refs[page] = 1;
                row[had - 1] = page;
            }
            bk.lens[slot] = want;
        }
        for (int c = had + sub; c < held; c += kEntryLanes) {
            const int page = fresh[first + takes + c - had];
            row[c] = page;
            bk.refs[page] = 1;
        }
    };
    if constexpr (ONE) {
        for (int k = 0; k < kEntryLanes; ++k) {                    // entry k of this thread's group of lanes
            const int from = (tid & 31 & ~(kEntryLanes - 1)) + k;
            const int slot = __shfl_sync(0xffffffffu, mine.slot, from), want = __shfl_sync(0xffffffffu, mine.want, from);
            const int state = __shfl_sync(0xffffffffu, mine.state, from), first = __shfl_sync(0xffffffffu, start, from);
            const int takes = __shfl_sync(0xffffffffu, copy, from);
            if (state >= 0) put(slot, want, state, first, takes);
        }
    } else {
        for (int i = tid / kEntryLanes; i < p.n; i += groups) {
            const int state = __ldcg(p.state + i), mark = p.start[i];
            if (state >= 0) put(slot_at(i), p.want[i], state, mark & 0x7fffffff, mark < 0);
        }
    }
    for (int k = tid; k < copies; k += kBookThreads) p.dst[k] = fresh[p.dst[k]];
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
// One CTA (3000 pages: 7.7 us under a profiler, 4 of them the launch).  Which pages are held goes to shared memory as bits in one pass over refs; the k-th held one above the
// number of pages in use and the k-th free one below it become pair k.
__global__ void __launch_bounds__(kBookThreads, 1)
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
