// Page and book entry points of include/cudallm_cache.h: validation, scratch, launches.
#include "../../include/cudallm_cache.h"

#include <algorithm>
#include <atomic>

#include "runtime.h"
#include "pages.cuh"

using namespace cudallm;

namespace {

constexpr int64_t kMaxDim = (int64_t(1) << 31) - 1024;
constexpr int64_t kMaxBytes = int64_t(1) << 46;
constexpr int64_t kMaxPage = int64_t(1) << 35;           // bytes: the chunks of a launch's pools are counted in 31 bits
static_assert(kMaxPage / kCopyChunk * kPoolsPerLaunch < kMaxDim, "chunks");
constexpr int64_t kMaxBook = int64_t(1) << 20;           // pages of a book
constexpr int64_t kMaxList = int64_t(1) << 14;           // entries of a list
constexpr int64_t kMaxPools = 65536;
constexpr int64_t kPlanSms = 148;

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool off(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

int check_pools(const cudallm_page_pool *pools, int64_t count, int64_t pages)
{
    if (count < 0 || count > kMaxPools || pages < 0 || pages > kMaxDim) return CUDALLM_ERR_INVALID_DIM;
    if (count == 0) return CUDALLM_OK;
    if (!pools) return CUDALLM_ERR_INVALID_POINTER;
    for (int64_t i = 0; i < count; ++i) {
        const cudallm_page_pool &p = pools[i];
        if (p.bytes < 0 || p.bytes > kMaxPage) return CUDALLM_ERR_INVALID_DIM;
        if (p.bytes == 0 || pages == 0) continue;
        if (!p.data) return CUDALLM_ERR_INVALID_POINTER;
        if (pages > 1 && p.stride < p.bytes) return CUDALLM_ERR_INVALID_LD;
        if (pages > 1 && (long double)p.stride * pages > (long double)kMaxBytes) return CUDALLM_ERR_INVALID_DIM;
        if (off(p.data, 16) || p.bytes % 16 || (pages > 1 && p.stride % 16)) return CUDALLM_ERR_UNSUPPORTED_SHAPE;
    }
    return CUDALLM_OK;
}

int check_book(const cudallm_page_book *bp)
{
    if (!bp) return CUDALLM_ERR_INVALID_POINTER;
    const cudallm_page_book &b = *bp;
    if (b.pages < 0 || b.pages > kMaxBook || b.page_rows < 1 || b.page_rows > kMaxDim || b.slots < 0 || b.slots > kMaxDim
        || b.table_cols < 0 || b.table_cols > kMaxDim / b.page_rows)
        return CUDALLM_ERR_INVALID_DIM;
    if (b.slots > 1 && b.table_stride < b.table_cols) return CUDALLM_ERR_INVALID_LD;
    if (b.slots > 1 && (long double)b.table_stride * b.slots > (long double)kMaxBytes) return CUDALLM_ERR_INVALID_DIM;
    if ((b.pages > 0 && !b.refs) || (b.slots > 0 && (!b.lens || (b.table_cols > 0 && !b.table))))
        return CUDALLM_ERR_INVALID_POINTER;
    if (off(b.refs, 16) || off(b.lens, 4) || off(b.table, 4)) return CUDALLM_ERR_MISALIGNED;
    return CUDALLM_OK;
}

Book device_book(const cudallm_page_book &b)
{
    Book d{};
    d.refs = b.refs; d.lens = b.lens; d.table = b.table;
    d.stride = b.table_stride;
    d.pages = (int)b.pages; d.rows = (int)b.page_rows; d.slots = (int)b.slots; d.cols = (int)b.table_cols;
    d.cap = (int)(b.table_cols * b.page_rows);
    return d;
}

// Words of scratch from `at` on, each array beginning on 16 bytes.
struct Words {
    size_t used = 0;
    size_t take(int64_t n)
    {
        const size_t at = used;
        used += (size_t)cdiv(n, 4) * 4;
        return at;
    }
    size_t bytes() const { return used * sizeof(int); }
};
struct ResizeScratch {
    size_t count, src, dst, state, start, fresh, claims, claimer, bytes;
    ResizeScratch(const cudallm_page_book &b, int64_t n)
    {
        Words w;
        count = w.take(4);
        src = w.take(n); dst = w.take(n); state = w.take(n); start = w.take(n);
        fresh = w.take(b.pages); claims = w.take(b.pages); claimer = w.take(b.pages);
        bytes = w.bytes();
    }
};
struct CompactScratch {
    size_t count, first_moved, src, dst, remap, bytes;
    explicit CompactScratch(const cudallm_page_book &b)
    {
        Words w;
        count = w.take(4); first_moved = w.take(4);
        src = w.take(b.pages); dst = w.take(b.pages); remap = w.take(b.pages);
        bytes = w.bytes();
    }
};
size_t fork_bytes(const cudallm_page_book &b, int64_t n) { return (size_t)(cdiv(n, 4) * 4 + n * b.table_cols) * sizeof(int); }

bool list_size(int64_t n) { return n >= 0 && n <= kMaxList; }
bool scratch_short(const void *scratch, size_t have, size_t need) { return !scratch || off(scratch, 16) || have < need; }

// CTAs of a cluster for so many CTAs' worth of work: one, two, four or eight.
int64_t cluster_for(int64_t ctas) { return ctas <= 1 ? 1 : ctas <= 2 ? 2 : ctas <= 4 ? 4 : kBookCluster; }

// The copies (and, for compaction, the table) of up to kPoolsPerLaunch pools a launch.
int copy_pools(CopyParams p, const cudallm_page_pool *pools, int64_t count, cudaStream_t stream)
{
    int64_t i = 0;
    do {
        PoolList list{};
        int64_t largest = 0;
        p.pools = 0;
        for (; i < count && p.pools < kPoolsPerLaunch; ++i)
            if (pools[i].bytes > 0) {
                list.at[p.pools++] = pools[i];
                largest = std::max(largest, pools[i].bytes);
            }
        if (p.pools == 0 && !p.remap) return CUDALLM_OK;
        const int64_t chunks = std::max<int64_t>(1, cdiv(largest, kCopyChunk));
        p.chunks = (int)chunks;
        int64_t want = p.pools > 0 ? (p.n > kMaxDim / (chunks * p.pools) ? kMaxDim : cdiv(p.n * chunks * p.pools, kCopyThreads / 32)) : 0;
        if (p.remap) want = std::max<int64_t>(want, p.book.slots);
        const int st = rt_launch(pages_copy_kernel, dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(want, 16 * kPlanSms))),
                                 kCopyThreads, 0, stream, p, list);
        if (st != CUDALLM_OK) return st;
        p.remap = nullptr;
    } while (i < count);
    return CUDALLM_OK;
}

}  // namespace

extern "C" {

int cudallm_pages_copy(const cudallm_page_pool *pools, int64_t count, int64_t pages, const int32_t *src, const int32_t *dst,
                       int64_t n, void *stream)
{
    int st = check_pools(pools, count, pages);
    if (st != CUDALLM_OK) return st;
    if (n < 0 || n > kMaxDim) return CUDALLM_ERR_INVALID_DIM;
    if (n == 0 || count == 0 || pages == 0) return CUDALLM_OK;
    if (!src || !dst) return CUDALLM_ERR_INVALID_POINTER;
    if (off(src, 4) || off(dst, 4)) return CUDALLM_ERR_MISALIGNED;
    int dev = 0, sms = 0;
    if ((st = rt_current_device(&dev, &sms)) != CUDALLM_OK) return st;
    CopyParams p{};
    p.src = src; p.dst = dst; p.n = n; p.pages = (int)pages;
    return copy_pools(p, pools, count, static_cast<cudaStream_t>(stream));
}

size_t cudallm_pages_fork_scratch_bytes(const cudallm_page_book *book, int64_t n)
{
    return check_book(book) == CUDALLM_OK && list_size(n) ? fork_bytes(*book, n) : 0;
}

int cudallm_pages_fork(const cudallm_page_book *book, const int32_t *src, const int32_t *dst, int64_t n,
                       void *scratch, size_t scratch_bytes, void *stream_v)
{
    int st = check_book(book);
    if (st != CUDALLM_OK) return st;
    if (!list_size(n)) return CUDALLM_ERR_INVALID_DIM;
    if (n == 0 || book->slots == 0) return CUDALLM_OK;
    if (!src || !dst) return CUDALLM_ERR_INVALID_POINTER;
    if (off(src, 4) || off(dst, 4)) return CUDALLM_ERR_MISALIGNED;
    if (scratch_short(scratch, scratch_bytes, fork_bytes(*book, n))) return CUDALLM_ERR_WORKSPACE;
    int dev = 0, sms = 0;
    if ((st = rt_current_device(&dev, &sms)) != CUDALLM_OK) return st;
    ForkParams p{};
    p.book = device_book(*book);
    p.src = src; p.dst = dst; p.n = (int)n;
    p.staged_len = static_cast<int *>(scratch);
    p.staged = p.staged_len + cdiv(n, 4) * 4;
    p.chunks = (int)std::max<int64_t>(1, cdiv(book->table_cols, kForkCols));
    const int64_t ctas = cluster_for(cdiv(n * p.chunks, kBookThreads / 32));
    return rt_launch_cluster(pages_fork_kernel, dim3((unsigned)ctas), (unsigned)ctas, kBookThreads, 0, static_cast<cudaStream_t>(stream_v), p);
}

size_t cudallm_pages_resize_scratch_bytes(const cudallm_page_book *book, int64_t n)
{
    return check_book(book) == CUDALLM_OK && list_size(n) ? ResizeScratch(*book, n).bytes : 0;
}

int cudallm_pages_resize(const cudallm_page_book *book, const cudallm_page_pool *pools, int64_t count, const int32_t *slot_of,
                         const int32_t *new_lens, int64_t n, int32_t *result, void *scratch, size_t scratch_bytes,
                         void *stream_v)
{
    int st = check_book(book);
    if (st == CUDALLM_OK) st = check_pools(pools, count, book->pages);
    if (st != CUDALLM_OK) return st;
    if (!list_size(n) || (!slot_of && n > book->slots)) return CUDALLM_ERR_INVALID_DIM;
    if (n > 0 && !new_lens) return CUDALLM_ERR_INVALID_POINTER;
    if (off(slot_of, 4) || off(new_lens, 4) || off(result, 4)) return CUDALLM_ERR_MISALIGNED;
    const ResizeScratch at(*book, n);
    if (scratch_short(scratch, scratch_bytes, at.bytes)) return CUDALLM_ERR_WORKSPACE;
    int dev = 0, sms = 0;
    if ((st = rt_current_device(&dev, &sms)) != CUDALLM_OK) return st;
    int *w = static_cast<int *>(scratch);
    ResizeParams p{};
    p.book = device_book(*book);
    p.slot_of = slot_of; p.want = new_lens; p.n = (int)n; p.result = result;
    p.count = w + at.count; p.src = w + at.src; p.dst = w + at.dst; p.state = w + at.state; p.start = w + at.start;
    p.fresh = w + at.fresh; p.claims = w + at.claims; p.claimer = w + at.claimer;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    const int64_t ctas = cluster_for(cdiv(n, kBookThreads / kEntryLanes));
    st = rt_launch_cluster(n <= kBookThreads ? pages_resize_kernel<true> : pages_resize_kernel<false>, dim3((unsigned)ctas),
                           (unsigned)ctas, kBookThreads, 0, stream, p);
    if (st != CUDALLM_OK || count == 0 || n == 0 || book->pages == 0) return st;
    CopyParams c{};
    c.src = p.src; c.dst = p.dst; c.count = p.count; c.n = n; c.pages = p.book.pages;
    return copy_pools(c, pools, count, stream);
}

size_t cudallm_pages_compact_scratch_bytes(const cudallm_page_book *book)
{
    return check_book(book) == CUDALLM_OK ? CompactScratch(*book).bytes : 0;
}

int cudallm_pages_compact(const cudallm_page_book *book, const cudallm_page_pool *pools, int64_t count, int32_t *used,
                          void *scratch, size_t scratch_bytes, void *stream_v)
{
    int st = check_book(book);
    if (st == CUDALLM_OK) st = check_pools(pools, count, book->pages);
    if (st != CUDALLM_OK) return st;
    if (off(used, 4)) return CUDALLM_ERR_MISALIGNED;
    const CompactScratch at(*book);
    if (scratch_short(scratch, scratch_bytes, at.bytes)) return CUDALLM_ERR_WORKSPACE;
    int dev = 0, sms = 0;
    if ((st = rt_current_device(&dev, &sms)) != CUDALLM_OK) return st;
    int *w = static_cast<int *>(scratch);
    CompactParams p{};
    p.book = device_book(*book);
    p.used = used;
    p.count = w + at.count; p.first_moved = w + at.first_moved;
    p.src = w + at.src; p.dst = w + at.dst; p.remap = w + at.remap;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    const int smem = (int)(cdiv(book->pages, 16) * 2);             // 128 KiB for 2^20 pages
    // (the kernel's own shared memory counts in the 48 KiB that a launch may have unasked, so it is asked for whatever the size)
    static std::atomic<bool> done[kRtMaxDevices] = {};
    if (!done[dev].load(std::memory_order_relaxed)) {
        RT_CUDA_TRY(cudaFuncSetAttribute(pages_compact_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kMaxBook / 8)));
        done[dev].store(true, std::memory_order_relaxed);
    }
    st = rt_launch(pages_compact_kernel, dim3(1), kBookThreads, (size_t)smem, stream, p);
    if (st != CUDALLM_OK) return st;
    CopyParams c{};
    c.src = p.src; c.dst = p.dst; c.count = p.count; c.n = book->pages / 2 + 1; c.pages = p.book.pages;
    c.book = p.book; c.remap = p.remap; c.first_moved = p.first_moved;
    return copy_pools(c, pools, count, stream);
}

}  // extern "C"
