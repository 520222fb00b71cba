// Paged cache entry points of include/cudallm_cache.h: appending keys and values, attention of the newest
// tokens.  Validation, the choice of the split, launches.
#include "../../include/cudallm_cache.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <limits>

#include "runtime.h"
#include "paged_attn.cuh"
#include "paged_narrow.cuh"
#include "paged_tile.cuh"

using namespace cudallm;

namespace {

constexpr int64_t kMaxDim = (int64_t(1) << 31) - 1024;
constexpr int64_t kMaxElems = int64_t(1) << 46;          // of an operand, strides included
constexpr int64_t kMaxTmaStride = int64_t(1) << 39;      // elements
constexpr float kMaxScale = 2.0e38f;                     // (times log2 e it is still a number)
constexpr int64_t kPlanSms = 148;                        // the split is planned for this many SMs
constexpr int64_t kClusterBlocks = 16;                   // blocks of keys that a CTA of a cluster may get at most,
constexpr int64_t kClusterMore = 4;                      // and how many more than an equal share would have

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool off(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

// Strides of a three-level operand: multiples of 8, no two elements in one place.
int check_strides(const int64_t (&st)[3], int64_t e0, int64_t e1, int64_t e2, int64_t dim)
{
    const int64_t ext[3] = {e0, e1, e2};
    int order[3], n = 0;
    for (int i = 0; i < 3; ++i)
        if (ext[i] > 1) order[n++] = i;
    for (int i = 0; i < n; ++i)
        if (st[order[i]] <= 0) return CUDALLM_ERR_INVALID_LD;
    std::sort(order, order + n, [&](int a, int b) { return st[a] < st[b]; });
    long double cover = (long double)dim;
    for (int i = 0; i < n; ++i) {
        const int64_t s = st[order[i]];
        if ((long double)s < cover) return CUDALLM_ERR_INVALID_LD;
        cover += (long double)s * (long double)(ext[order[i]] - 1);
        if (cover > (long double)kMaxElems) return CUDALLM_ERR_INVALID_DIM;
    }
    for (int i = 0; i < n; ++i)
        if (st[order[i]] % 8) return CUDALLM_ERR_UNSUPPORTED_SHAPE;
    return CUDALLM_OK;
}

bool no_states(const cudallm_paged_shape &s) { return s.pages == 0 || s.table_cols == 0; }
// Nothing to write: no items, tokens or values, or no item that is there.
bool append_empty(const cudallm_paged_shape &s)
{
    return s.batch == 0 || s.q_rows == 0 || s.kv_heads == 0 || s.head_dim == 0 || s.slots == 0 || no_states(s);
}
bool attn_empty(const cudallm_paged_shape &s)
{
    return s.batch == 0 || s.q_rows == 0 || s.q_heads == 0 || s.head_dim == 0 || s.slots == 0;
}

int check_shape(const cudallm_paged_shape *sp)
{
    if (!sp) return CUDALLM_ERR_INVALID_POINTER;
    const cudallm_paged_shape &s = *sp;
    if (s.dtype != CUDALLM_BF16 && s.dtype != CUDALLM_F16) return CUDALLM_ERR_INVALID_DTYPE;
    for (int64_t v : {s.batch, s.q_rows, s.q_heads, s.kv_heads, s.head_dim, s.pages, s.slots, s.table_cols})
        if (v < 0 || v > kMaxDim) return CUDALLM_ERR_INVALID_DIM;
    if (s.page_rows < 1 || s.page_rows > kMaxDim) return CUDALLM_ERR_INVALID_DIM;
    if (!(s.scale >= 0.f) || !(s.scale <= kMaxScale)) return CUDALLM_ERR_INVALID_DIM;
    if (s.q_heads > 0 && (s.kv_heads == 0 || s.q_heads % s.kv_heads)) return CUDALLM_ERR_INVALID_DIM;
    if (s.table_cols > kMaxDim / s.page_rows) return CUDALLM_ERR_INVALID_DIM;
    if (s.slots > 1 && s.table_stride < s.table_cols) return CUDALLM_ERR_INVALID_LD;
    if (s.slots > 1 && (long double)s.table_stride * s.slots > (long double)kMaxElems) return CUDALLM_ERR_INVALID_DIM;
    if (s.head_dim % 8 || s.head_dim > 128) return CUDALLM_ERR_UNSUPPORTED_SHAPE;
    // items x heads x tokens x 16-byte pieces (16 of a head at most) are counted in 31 bits
    if ((long double)s.batch * std::max(s.q_heads, s.kv_heads) * s.q_rows > (long double)(kMaxDim / 16)) return CUDALLM_ERR_INVALID_DIM;
    if (no_states(s) || s.kv_heads == 0 || s.head_dim == 0) return CUDALLM_OK;
    int st = check_strides(s.k_stride, s.pages, s.page_rows, s.kv_heads, s.head_dim);
    if (st == CUDALLM_OK) st = check_strides(s.v_stride, s.pages, s.page_rows, s.kv_heads, s.head_dim);
    return st;
}

// Whether TMA can bring the pools' pages into tiles (its strides are below 2^40 bytes).
bool tile_pages(const cudallm_paged_shape &s)
{
    for (const auto *st : {&s.k_stride, &s.v_stride})
        if ((s.pages > 1 && (*st)[0] >= kMaxTmaStride) || (s.page_rows > 1 && (*st)[1] >= kMaxTmaStride)
            || (s.kv_heads > 1 && (*st)[2] >= kMaxTmaStride))
            return false;
    return !no_states(s) && paged_tile_pages(s.page_rows);
}

// How an attention call runs.
struct Plan {
    bool wide;                  // head dims above 64
    int mt, row_tiles;          // row tiles of 16 mt rows; 0: of 128, by paged_tile_kernel
    int cluster;                // CTAs a cluster; 0: equal shares
    int shares, ctas;           // equal shares of a key head; CTAs in all
    size_t part_bytes, scratch;
};
Plan plan_attn(const cudallm_paged_shape &s)
{
    Plan f{};
    const int64_t rows = (s.q_heads / s.kv_heads) * s.q_rows, cap = no_states(s) ? 0 : s.table_cols * s.page_rows;
    f.wide = s.head_dim > 64;
    // More than 16 rows on a key head: by tiles of 128 on tcgen05 where TMA can bring the pages.  Up to 32 rows and 1024
    // states by mma.sync, in clusters or equal shares: a tile costs the same however few its rows and keys are.  (mma.sync against
    // tiles, us.  Clusters, 32 rows x 8 key heads of 128: 9.6 / 10.2 at 120 states, 10.8 / 11.8 at 500, 12.4 / 12.4 at 1000, 20.6 /
    // 17.0 at 4000; 64 rows: 14.3 / 10.9 at 120.  16 sequences of 8 key heads at 250 and 500 states: 20 rows 12.4 / 12.3, 15.9 / 14.9, 32
    // rows 13.7 / 12.0, 17.0 / 14.5, of a quarter to all of 500 16.2 / 18.2; heads of 64, 32 rows 9.6 / 11.2, 11.6 / 13.6.  Equal
    // shares, 64 sequences at 100, 250, 500: 20 rows 21.1 / 24.1, 29.7 / 32.9, 44.4 / 50.3, 32 rows 23.4 / 24.4, 32.9 / 32.4,
    // 48.5 / 47.9, of a quarter to all of 500 34.4 / 43.1; heads of 64, 20 rows 14.5 / 21.6, 19.7 / 29.9, 27.6 / 40.6.)
    const bool tile = rows > 16 && tile_pages(s) && !(rows <= 32 && cap <= 1024);
    f.mt = tile ? 0 : (int)std::min<int64_t>(4, cdiv(rows, 16));
    const int64_t tile_rows = tile ? kXaRows : 16 * f.mt, block = tile ? kXaRows : f.wide ? 64 : 128;
    f.row_tiles = (int)cdiv(rows, tile_rows);
    const int64_t items = s.batch * s.kv_heads * f.row_tiles, blocks = std::max<int64_t>(1, cdiv(cap, block));
    const int64_t fits = std::min<int64_t>({int64_t(kPaCluster), 2 * kPlanSms / std::max<int64_t>(items, 1), blocks});
    // A cluster per item needs no second launch, but takes as long as the longest item and may leave SMs idle: blocks / fits against
    // blocks x items / (two CTAs an SM) blocks, one of them about a microsecond, and the launch that joins costs about four.
    // (Heads of 128, 4 rows, clusters against equal shares, us: one item of 1000, 2000, 4000 states 8.3 / 9.6, 10.0 / 9.9, 14.0 / 10.0;
    // 8 items of 2000, 4000: 10.4 / 11.2, 14.5 / 11.6; 32 items of 4000, 8000: 16.4 / 18.4, 27.9 / 30.2; 64 items of 4000: 27.1 /
    // 29.6, of 1000 to 4000: 23.5 / 20.1.)
    if (!tile && items <= kPlanSms && blocks <= kClusterBlocks * fits
        && blocks * (2 * kPlanSms - fits * items) <= kClusterMore * 2 * kPlanSms * fits) {
        f.cluster = (int)std::max<int64_t>(1, fits);
        f.ctas = (int)(items * f.cluster);
        return f;
    }
    // As many shares of every key head as fit at once, but no more than there are blocks.  A whole number for each: neighbouring CTAs
    // take the same share for the different heads (see paged_attn.cuh), at the cost of the rest of the SMs where their number
    // is no multiple of kv_heads (40 key heads on tiles: 120 of 148).
    f.shares = (int)std::max<int64_t>(1, std::min<int64_t>((tile ? 1 : 2) * kPlanSms / s.kv_heads, s.batch * f.row_tiles * blocks));
    f.ctas = (int)(f.shares * s.kv_heads);
    f.part_bytes = f.shares == 1 ? 0 : 2 * (size_t)f.ctas * (size_t)tile_rows * ((f.wide ? 128 : 64) + 1) * sizeof(float);
    f.scratch = f.part_bytes + (size_t)f.ctas * kPaDesc * sizeof(int);
    return f;
}

// Factor of the exponentials' arguments.  Masked scores are -inf, and -inf x 0 is no number, so a scale that leaves nothing enters as
// the smallest number, 2^-149: finite scores differ by less than 2^129, so their exponents by less than 2^-20, and their
// exponentials are 1 to within that.  Other scales are taken as they are, however small.
inline float scale_log2(float scale)
{
    return std::max(scale * 1.4426950408889634f, std::numeric_limits<float>::denorm_min());
}

inline XaStrides strides(const int64_t (&s)[3]) { return XaStrides{(long long)s[0], (long long)s[1], (long long)s[2]}; }
inline PagedStrides page_strides(const int64_t (&s)[3]) { return PagedStrides{(long long)s[0], (long long)s[1], (long long)s[2]}; }
inline XaStrides pieces(const int64_t (&s)[3]) { return XaStrides{s[0] / 8, s[1] / 8, s[2] / 8}; }
inline PagedStrides page_pieces(const int64_t (&s)[3]) { return PagedStrides{s[0] / 8, s[1] / 8, s[2] / 8}; }

// Raises a kernel's limit of dynamic shared memory, once per device.
template <typename Kernel>
int allow_smem(Kernel kernel, int bytes, std::atomic<bool> (&done)[kRtMaxDevices], int dev)
{
    if (!done[dev].load(std::memory_order_relaxed)) {
        RT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
        done[dev].store(true, std::memory_order_relaxed);
    }
    return CUDALLM_OK;
}

constexpr int64_t kJoinCtas = 16 * kPlanSms;             // of 128 threads: a full machine
// Equal shares leave parts of items behind, to be joined.
template <int DP, int ROWS, typename T>
int join(const cudallm_paged_shape &s, const Plan &f, const PagedParams &p, cudaStream_t stream)
{
    if (f.shares == 1) return CUDALLM_OK;
    constexpr int64_t kMaxGroups = kPaJoinThreads / (DP / 8);
    const int64_t rows = std::min<int64_t>(ROWS, (int64_t)p.group * s.q_rows);
    // threads for every eight or so of the parts that an item has on average; all CTAs that may have one to join run at once
    const int64_t parts = cdiv(f.shares, s.batch * f.row_tiles) + 1;
    int shift = 0;
    while (1 << shift < kMaxGroups && parts > 8 << shift) ++shift;
    const int64_t y = cdiv(rows, kMaxGroups >> shift);
    return rt_launch(paged_join_kernel<DP, ROWS, T>, dim3((unsigned)f.ctas, (unsigned)std::min<int64_t>(y, std::max<int64_t>(1, kJoinCtas / f.ctas))),
                     kPaJoinThreads, 0, stream, p, shift);
}
// The mma.sync kernels: ROWS rows of a key head a CTA.
template <int DP, int ROWS, typename T, typename Kernel>
int run_mma(Kernel kernel, int bytes, const cudallm_paged_shape &s, const Plan &f, const PagedParams &p, int dev, cudaStream_t stream)
{
    static std::atomic<bool> done[kRtMaxDevices] = {};
    int st = allow_smem(kernel, bytes, done, dev);
    if (st != CUDALLM_OK) return st;
    st = rt_launch_cluster(kernel, dim3((unsigned)f.ctas), f.cluster ? (unsigned)f.cluster : 1u, kPaThreads, (size_t)bytes, stream, p);
    return st != CUDALLM_OK || f.cluster ? st : join<DP, ROWS, T>(s, f, p, stream);
}
// Tensor map of a pool: 64 columns of one key head of up to 128 rows of a page.
int encode(CUtensorMap *tm, const void *base, bool f16, const cudallm_paged_shape &s, const int64_t (&st)[3])
{
    const uint64_t dims[4] = {(uint64_t)s.head_dim, (uint64_t)s.kv_heads, (uint64_t)s.page_rows, (uint64_t)s.pages};
    const uint64_t bytes[3] = {(uint64_t)(s.kv_heads > 1 ? st[2] : 8) * 2, (uint64_t)(s.page_rows > 1 ? st[1] : 8) * 2,
                               (uint64_t)(s.pages > 1 ? st[0] : 8) * 2};
    return rt_encode_rows(tm, base, f16, dims, bytes, (int)std::min<int64_t>(s.page_rows, kXaRows));
}
template <int DP, typename T>
int run_tile(const cudallm_paged_shape &s, const Plan &f, PagedParams &p, int dev, cudaStream_t stream)
{
    using L = PagedTileSmem<DP>;
    static std::atomic<bool> done[kRtMaxDevices] = {};
    int st = allow_smem(paged_tile_kernel<DP, T>, L::kBytes, done, dev);
    if (st != CUDALLM_OK) return st;
    const bool f16 = s.dtype == CUDALLM_F16;
    CUtensorMap tk, tv;
    if ((st = encode(&tk, p.k, f16, s, s.k_stride)) != CUDALLM_OK || (st = encode(&tv, p.v, f16, s, s.v_stride)) != CUDALLM_OK) return st;
    PagedTileParams t{};
    t.a = p;
    if ((st = rt_attention_status_word(dev, &t.status)) != CUDALLM_OK) return st;
    t.skip_loads = rt_take_skip_loads();
    t.wait_limit_ns = rt_wait_limit_ns();
    st = rt_launch(paged_tile_kernel<DP, T>, dim3((unsigned)f.ctas), kPtThreads, (size_t)L::kBytes, stream, tk, tv, t);
    return st != CUDALLM_OK ? st : join<DP, L::kRows, T>(s, f, p, stream);
}
template <int DP, typename T>
int run(const cudallm_paged_shape &s, const Plan &f, PagedParams &p, int dev, cudaStream_t stream)
{
    switch (f.mt) {
    case 0: return run_tile<DP, T>(s, f, p, dev, stream);
    case 1: return run_mma<DP, 16, T>(paged_narrow_kernel<DP, T>, PagedNarrowSmem<DP>::kBytes, s, f, p, dev, stream);
    case 2: return run_mma<DP, 32, T>(paged_wide_kernel<DP, 2, T>, PagedSmem<DP, 2>::kBytes, s, f, p, dev, stream);
    case 3: return run_mma<DP, 48, T>(paged_wide_kernel<DP, 3, T>, PagedSmem<DP, 3>::kBytes, s, f, p, dev, stream);
    default: return run_mma<DP, 64, T>(paged_wide_kernel<DP, 4, T>, PagedSmem<DP, 4>::kBytes, s, f, p, dev, stream);
    }
}
template <typename T>
int run(const cudallm_paged_shape &s, const Plan &f, PagedParams &p, int dev, cudaStream_t stream)
{
    return f.wide ? run<128, T>(s, f, p, dev, stream) : run<64, T>(s, f, p, dev, stream);
}

}  // namespace

extern "C" {

size_t cudallm_paged_attn_scratch_bytes(const cudallm_paged_shape *shape)
{
    if (check_shape(shape) != CUDALLM_OK || attn_empty(*shape)) return 0;
    return plan_attn(*shape).scratch;
}

int cudallm_paged_attn(const cudallm_paged_shape *shape, const void *q, const void *k, const void *v, const int32_t *table,
                       const int32_t *lens, const int32_t *slot_of, const int32_t *new_lens, void *o, float *lse,
                       void *scratch, size_t scratch_bytes, void *stream)
{
    int st = check_shape(shape);
    if (st != CUDALLM_OK) return st;
    const cudallm_paged_shape &s = *shape;
    if (attn_empty(s)) return CUDALLM_OK;
    st = check_strides(s.q_stride, s.batch, s.q_rows, s.q_heads, s.head_dim);
    if (st == CUDALLM_OK) st = check_strides(s.o_stride, s.batch, s.q_rows, s.q_heads, s.head_dim);
    if (st != CUDALLM_OK) return st;
    const bool states = !no_states(s);
    if (!q || !o || !lens || (states && (!k || !v || !table))) return CUDALLM_ERR_INVALID_POINTER;
    if (off(table, 4) || off(lens, 4) || off(slot_of, 4) || off(new_lens, 4) || off(lse, 4)) return CUDALLM_ERR_MISALIGNED;
    if (off(q, 16) || off(o, 16) || (states && (off(k, 16) || off(v, 16)))) return CUDALLM_ERR_UNSUPPORTED_SHAPE;
    const Plan f = plan_attn(s);
    if (f.scratch && (!scratch || off(scratch, 16) || scratch_bytes < f.scratch)) return CUDALLM_ERR_WORKSPACE;
    int dev = 0, sms = 0;
    if ((st = rt_current_device(&dev, &sms)) != CUDALLM_OK) return st;
    PagedParams p{};
    p.q = q; p.k = k; p.v = v; p.o = o; p.lse = lse;
    if (f.scratch) {
        p.part = static_cast<float *>(scratch);
        p.desc = reinterpret_cast<int *>(static_cast<char *>(scratch) + f.part_bytes);
    }
    p.table = table; p.lens = lens; p.slot_of = slot_of; p.new_lens = new_lens;
    p.sq = strides(s.q_stride); p.so = strides(s.o_stride);
    p.sk = page_strides(s.k_stride); p.sv = page_strides(s.v_stride);
    p.table_stride = s.table_stride;
    p.batch = (int)s.batch; p.q_rows = (int)s.q_rows; p.q_heads = (int)s.q_heads; p.kv_heads = (int)s.kv_heads;
    p.group = (int)(s.q_heads / s.kv_heads); p.head_dim = (int)s.head_dim;
    p.pages = (int)s.pages; p.page_rows = (int)s.page_rows; p.slots = (int)s.slots;
    p.cap = states ? (int)(s.table_cols * s.page_rows) : 0;
    p.by_page_rows = make_fast_div((uint32_t)s.page_rows);
    p.by_group = make_fast_div((uint32_t)p.group);
    p.row_tiles = f.row_tiles;
    p.cluster = f.cluster;
    p.shares = f.shares;
    // 128 threads count the units of all row tiles: some items each, or (more row tiles than one, few items) some each of an item's
    p.count_items = (int)cdiv(s.batch, kPaThreads);
    if (f.row_tiles > 1)
        while (s.batch << (p.count_shift + 1) <= kPaThreads) ++p.count_shift;
    p.count_tiles = (int)cdiv(f.row_tiles, int64_t(1) << p.count_shift);
    p.scale = s.scale; p.scale_log2 = scale_log2(s.scale);
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    return s.dtype == CUDALLM_BF16 ? run<__nv_bfloat16>(s, f, p, dev, cs) : run<__half>(s, f, p, dev, cs);
}

int cudallm_cache_append(const cudallm_paged_shape *shape, const void *k_new, const void *v_new, void *k, void *v,
                         const int32_t *table, const int32_t *lens, const int32_t *slot_of, const int32_t *new_lens,
                         void *stream)
{
    int st = check_shape(shape);
    if (st != CUDALLM_OK) return st;
    const cudallm_paged_shape &s = *shape;
    if (append_empty(s)) return CUDALLM_OK;
    st = check_strides(s.kn_stride, s.batch, s.q_rows, s.kv_heads, s.head_dim);
    if (st == CUDALLM_OK) st = check_strides(s.vn_stride, s.batch, s.q_rows, s.kv_heads, s.head_dim);
    if (st != CUDALLM_OK) return st;
    if (!k_new || !v_new || !k || !v || !table || !lens) return CUDALLM_ERR_INVALID_POINTER;
    if (off(table, 4) || off(lens, 4) || off(slot_of, 4) || off(new_lens, 4)) return CUDALLM_ERR_MISALIGNED;
    if (off(k_new, 16) || off(v_new, 16) || off(k, 16) || off(v, 16)) return CUDALLM_ERR_UNSUPPORTED_SHAPE;
    int dev = 0, sms = 0;
    if ((st = rt_current_device(&dev, &sms)) != CUDALLM_OK) return st;
    AppendParams p{};
    p.k_new = static_cast<const uint4 *>(k_new); p.v_new = static_cast<const uint4 *>(v_new);
    p.k = static_cast<uint4 *>(k); p.v = static_cast<uint4 *>(v);
    p.table = table; p.lens = lens; p.slot_of = slot_of; p.new_lens = new_lens;
    p.skn = pieces(s.kn_stride); p.svn = pieces(s.vn_stride);
    p.sk = page_pieces(s.k_stride); p.sv = page_pieces(s.v_stride);
    p.table_stride = s.table_stride;
    p.chunks = (int)(s.head_dim / 8); p.q_rows = (int)s.q_rows; p.page_rows = (int)s.page_rows;
    p.tokens = (int)(s.batch * s.q_rows); p.pieces = (int)(s.kv_heads * p.chunks);           // (their product is below 2^31: see check_shape)
    p.by_chunks = make_fast_div((uint32_t)p.chunks); p.by_rows = make_fast_div((uint32_t)p.q_rows);
    p.by_page_rows = make_fast_div((uint32_t)p.page_rows);
    p.pages = (int)s.pages; p.slots = (int)s.slots; p.cap = (int)(s.table_cols * s.page_rows);
    // a warp a token, or a part of one where the token's pieces do not fill it
    for (p.lanes = 1; p.lanes < 32 && p.lanes < p.pieces; p.lanes *= 2) {}
    const int64_t threads = (int64_t)p.tokens * p.lanes;
    return rt_launch(cache_append_kernel, dim3((unsigned)cdiv(threads, kAppendThreads)), kAppendThreads, 0,
                     static_cast<cudaStream_t>(stream), p);
}

}  // extern "C"
