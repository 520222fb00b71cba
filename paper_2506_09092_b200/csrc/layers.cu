// Entry points of include/cudallm_layers.h that are bound by memory bandwidth: LayerNorm over
// rows (forward, backward), and the norm and clipping of a list of gradients.
#include "../../include/cudallm_layers.h"

#include <algorithm>
#include <atomic>
#include <cmath>

#include "runtime.h"
#include "layernorm_rows.cuh"
#include "grad_norm.cuh"

using namespace cudallm;

namespace {

constexpr int64_t kMaxDim = (int64_t(1) << 31) - 1024;
constexpr int64_t kMaxElems = int64_t(1) << 46;

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int elem_size(int dtype) { return dtype == CUDALLM_F32 ? 4 : 2; }
inline bool valid_dtype(int d) { return d == CUDALLM_F32 || d == CUDALLM_BF16 || d == CUDALLM_F16; }
inline bool off(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

// --------------------------------------------------------------- LayerNorm --
// What both directions check; dtype-sized operands first.
int check_ln(int64_t rows, int64_t n, int dtype, int param_dtype)
{
    if (!valid_dtype(dtype) || (param_dtype != dtype && param_dtype != CUDALLM_F32)) return CUDALLM_ERR_INVALID_DTYPE;
    if (rows < 0 || n < 0 || rows > kMaxDim || n > kMaxDim) return CUDALLM_ERR_INVALID_DIM;
    return CUDALLM_OK;
}
int check_ld(int64_t rows, int64_t n, int64_t ld)
{
    if (ld < n) return CUDALLM_ERR_INVALID_LD;
    if (ld > kMaxElems || (long double)rows * ld > (long double)kMaxElems) return CUDALLM_ERR_INVALID_DIM;
    return CUDALLM_OK;
}

// CTAs of `kernel` that one SM holds, asked once per kernel and device, for the most shared memory that
// the kernel is ever launched with: grids, and with them the order of the sums, do not depend on earlier calls.
struct Residency {
    std::atomic<int> ctas[kRtMaxDevices];
};
template <typename Kernel>
int resident(Kernel kernel, int threads, int max_smem, int dev, Residency &cache, int *out)
{
    int v = cache.ctas[dev].load(std::memory_order_relaxed);
    if (v == 0) {
        if (max_smem > 48 * 1024)
            RT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, max_smem));
        RT_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&v, kernel, threads, max_smem));
        if (v < 1) v = 1;
        cache.ctas[dev].store(v, std::memory_order_relaxed);
    }
    *out = v;
    return CUDALLM_OK;
}

struct LnLaunch {
    int dev, sms;
    cudaStream_t stream;
};

template <typename T, int VEC, int TPR, int E, int R>
int launch_warp(const LnRowsParams &p, const LnLaunch &at)
{
    static Residency occ = {};
    auto kernel = layernorm_warp_kernel<T, VEC, TPR, E / kUnit<VEC>, R>;
    const int smem = 2 * p.n * (int)sizeof(float);                 // (n <= TPR * E)
    int per_sm = 0;
    const int st = resident(kernel, kLnWarpThreads, 2 * TPR * E * (int)sizeof(float), at.dev, occ, &per_sm);
    if (st != CUDALLM_OK) return st;
    const int64_t grid = std::min<int64_t>(cdiv(p.rows, R * (kLnWarpThreads / TPR)), (int64_t)at.sms * per_sm);
    return rt_launch(kernel, dim3((unsigned)grid), kLnWarpThreads, (size_t)smem, at.stream, p);
}
template <typename T, int VEC, int TPR, int E, int R>
int launch_block(const LnRowsParams &p, const LnLaunch &at)
{
    static Residency occ = {};
    auto kernel = layernorm_block_kernel<T, VEC, TPR, E / kUnit<VEC>, R>;
    constexpr int smem = ln_slot_bytes(VEC, TPR, E / kUnit<VEC>, R, 1);
    static_assert(smem <= 200 * 1024, "slots of the rows read and of those on their way");
    int per_sm = 0;
    const int st = resident(kernel, TPR, smem, at.dev, occ, &per_sm);
    if (st != CUDALLM_OK) return st;
    const int64_t grid = std::min<int64_t>(p.rows, (int64_t)at.sms * per_sm);
    return rt_launch(kernel, dim3((unsigned)grid), TPR, (size_t)smem, at.stream, p);
}

// Lanes or threads per row, values per thread and rows at a time by the row's length.  Where there are rows
// for every SM's warps, 32 values a thread: the shuffles and addresses of a row are then shared by
// enough of them (16384 x 4096 bf16: 48.3 us; with 16 values 56, with 8 60; 262144 x 256 on 8 lanes 48.3 us,
// on 32 lanes 61).  With few rows a row's latency counts and it is spread over more threads.  The numbers of rows
// at which that turns, bf16, the form for few rows | for many: 256 columns 4700 rows 2.9 | 3.3 us, 9472 rows 4.1 | 3.5;
// 4096 columns 580 rows 5.8 | 6.8 us, 2368 rows 12.7 | 12.1; 8192 columns 580 rows 8.5 | 8.4, 1184 rows 14.0 | 12.3 (rows of 512
// and 1024 turn earlier: 512 columns 4700 rows 6.4 | 4.4).  Rows that are not whole 16-byte pieces carry the next row in
// registers and take 16 values.
template <typename T, int VEC>
int launch_ln_by_length(const LnRowsParams &p, const LnLaunch &at)
{
    if (p.n <= 32) return launch_warp<T, VEC, 4, 8, 2>(p, at);
    if (p.n <= 64) return launch_warp<T, VEC, 4, 16, 2>(p, at);
    if (p.rows >= 32 * at.sms) {
        if (p.n <= 128) return launch_warp<T, VEC, 4, 32, 2>(p, at);
        if (p.n <= 256) return launch_warp<T, VEC, 8, 32, 2>(p, at);
        if (p.n <= 512) return launch_warp<T, VEC, 16, 32, 2>(p, at);
        if (p.n <= 1024) return launch_warp<T, VEC, 32, 32, 1>(p, at);
    }
    if (p.n <= 256) return launch_warp<T, VEC, 32, 8, 2>(p, at);
    if constexpr (VEC > 1)
        if (p.rows >= 4 * at.sms) {
            if (p.n <= 2048) return launch_block<T, VEC, 64, 32, 1>(p, at);
            if (p.n <= 4096) return launch_block<T, VEC, 128, 32, 1>(p, at);
            if (p.n <= 8192) return launch_block<T, VEC, 256, 32, 1>(p, at);
        }
    if (p.n <= 1024) return launch_block<T, VEC, 128, 8, 1>(p, at);
    if constexpr (VEC == 1) {
        if (p.n <= 2048) return launch_block<T, VEC, 128, 16, 1>(p, at);
        if (p.n <= 4096) return launch_block<T, VEC, 256, 16, 1>(p, at);
    } else {
        if (p.n <= 4096) return launch_block<T, VEC, 512, 8, 1>(p, at);
    }
    if (p.n <= 16384) return launch_block<T, VEC, 512, 32, 1>(p, at);
    const int64_t grid = std::min<int64_t>(p.rows, (int64_t)at.sms * 2);
    return rt_launch(layernorm_long_kernel<T>, dim3((unsigned)grid), kLnLongThreads, 0, at.stream, p);
}

// Partial rows of dgamma and dbeta at most: enough CTAs for eight per SM where rows are short,
// one per SM where a CTA's partial rows are long (they are written once and read once).
int64_t ln_max_parts(int64_t n)
{
    return std::min<int64_t>(1184, std::max<int64_t>(148, int64_t(148) * 8192 / std::max<int64_t>(n, 1)));
}

template <typename T, int VEC, int TPR, int E, int R>
int launch_warp_bwd(const LnRowsParams &p, const LnLaunch &at, int *parts)
{
    static Residency occ = {};
    auto kernel = layernorm_warp_bwd_kernel<T, VEC, TPR, E / kUnit<VEC>, R>;
    constexpr int kRows = kLnWarpThreads / TPR;
    const int smem = kRows * p.n * (int)sizeof(float);
    int per_sm = 0;
    const int st = resident(kernel, kLnWarpThreads, kRows * TPR * E * (int)sizeof(float), at.dev, occ, &per_sm);
    if (st != CUDALLM_OK) return st;
    const int64_t grid = std::min<int64_t>({cdiv(p.rows, R * kRows), (int64_t)at.sms * per_sm, ln_max_parts(p.n)});
    *parts = (int)grid;
    return rt_launch(kernel, dim3((unsigned)grid), kLnWarpThreads, (size_t)smem, at.stream, p);
}
template <typename T, int VEC, int TPR, int E, int R>
int launch_block_bwd(const LnRowsParams &p, const LnLaunch &at, int *parts)
{
    static Residency occ = {};
    auto kernel = layernorm_block_bwd_kernel<T, VEC, TPR, E / kUnit<VEC>, R>;
    constexpr int smem = ln_slot_bytes(VEC, TPR, E / kUnit<VEC>, R, 2);
    static_assert(smem <= 200 * 1024, "slots of the rows read and of those on their way");
    int per_sm = 0;
    const int st = resident(kernel, TPR, smem, at.dev, occ, &per_sm);
    if (st != CUDALLM_OK) return st;
    const int64_t grid = std::min<int64_t>({(int64_t)p.rows, (int64_t)at.sms * per_sm, ln_max_parts(p.n)});
    *parts = (int)grid;
    return rt_launch(kernel, dim3((unsigned)grid), TPR, (size_t)smem, at.stream, p);
}

// The same for the gradient, whose column sums take registers too: 8 values a thread and two or four rows at
// a time (16384 x 4096 bf16: 82.5 us; 16 values 85.8, one row at a time 97 to 112).  Few | many: 256 columns 4700 rows 7.1 | 8.0 us,
// 18944 rows 13.9 | 12.5; 512 columns 4700 rows 11.7 | 9.2; 1024 columns 580 rows 12.0 | 12.5, 1184 rows 13.4 | 12.8; 4096 columns
// 580 rows 14.8 | 14.4, 2368 rows 24.8 | 22.6.
template <typename T, int VEC>
int launch_ln_bwd_by_length(const LnRowsParams &p, const LnLaunch &at, int *parts)
{
    if (p.n <= 32) return launch_warp_bwd<T, VEC, 4, 8, 2>(p, at, parts);
    if (p.rows >= 32 * at.sms) {
        if (p.n <= 64) return launch_warp_bwd<T, VEC, 4, 16, 2>(p, at, parts);
        if (p.n <= 128) return launch_warp_bwd<T, VEC, 8, 16, 2>(p, at, parts);
        if (p.n <= 256) return launch_warp_bwd<T, VEC, 16, 16, 2>(p, at, parts);
        if (p.n <= 512) return launch_warp_bwd<T, VEC, 32, 16, 2>(p, at, parts);
    }
    if (p.n <= 256) return launch_warp_bwd<T, VEC, 32, 8, 1>(p, at, parts);
    if constexpr (VEC > 1)
        if (p.rows >= 4 * at.sms) {
            if (p.n <= 1024) return launch_block_bwd<T, VEC, 128, 8, 4>(p, at, parts);
            if (p.n <= 2048) return launch_block_bwd<T, VEC, 256, 8, 2>(p, at, parts);
            if (p.n <= 4096) return launch_block_bwd<T, VEC, 512, 8, 2>(p, at, parts);
        }
    if (p.n <= 1024) return launch_block_bwd<T, VEC, 128, 8, 1>(p, at, parts);
    if (p.n <= 2048) return launch_block_bwd<T, VEC, 256, 8, 1>(p, at, parts);
    if (p.n <= 4096) return launch_block_bwd<T, VEC, 512, 8, 1>(p, at, parts);
    if (p.n <= 8192) return launch_block_bwd<T, VEC, 512, 16, 1>(p, at, parts);
    // (two rows of 16384 fp32 values and the next two take more than an SM's shared memory)
    if constexpr (sizeof(T) == 2)
        if (p.n <= 16384) return launch_block_bwd<T, VEC, 1024, 16, 1>(p, at, parts);
    // Long rows: the column sums first (dx may lie over x or dy), then dx.  Parts for eight CTAs per SM, and at least as many as
    // leave 1024 rows to each.
    if (p.partials) {
        const int64_t want = std::max<int64_t>({int64_t(1), 148 * 8 / cdiv(p.n, 256), cdiv(p.rows, 1024)});
        const int64_t g = std::min<int64_t>({int64_t(148), int64_t(p.rows), want});
        *parts = (int)g;
        const int st = rt_launch(layernorm_long_columns_kernel<T>, dim3((unsigned)cdiv(p.n, 256), (unsigned)g), 256, 0,
                                 at.stream, p);
        if (st != CUDALLM_OK) return st;
    }
    if (!p.y) return CUDALLM_OK;
    const int64_t grid = std::min<int64_t>(p.rows, (int64_t)at.sms * 2);
    return rt_launch(layernorm_long_dx_kernel<T>, dim3((unsigned)grid), kLnLongThreads, 0, at.stream, p);
}

// 16-byte accesses need bases and pitches on 16-byte boundaries and whole pieces per row.
template <typename T, typename... Ptrs>
bool pieces_ok(int64_t n, std::initializer_list<int64_t> lds, Ptrs... ptrs)
{
    uintptr_t all = 0;
    for (const void *q : {static_cast<const void *>(ptrs)...}) all |= reinterpret_cast<uintptr_t>(q);
    int64_t m = n;
    for (int64_t ld : lds) m |= ld;
    return (all & 15) == 0 && m % ElemVec<T>::kN == 0;
}

template <typename T>
int run_ln(const LnRowsParams &p, const LnLaunch &at)
{
    if (pieces_ok<T>(p.n, {p.ldx, p.ldy}, p.x, p.y))
        return launch_ln_by_length<T, ElemVec<T>::kN>(p, at);
    return launch_ln_by_length<T, 1>(p, at);
}
template <typename T>
int run_ln_bwd(const LnRowsParams &p, const LnLaunch &at, int *parts)
{
    if (pieces_ok<T>(p.n, {p.ldx, p.lddy, p.y ? p.ldy : p.ldx}, p.x, p.dy, p.y))
        return launch_ln_bwd_by_length<T, ElemVec<T>::kN>(p, at, parts);
    return launch_ln_bwd_by_length<T, 1>(p, at, parts);
}

// -------------------------------------------------------------- gradients --
constexpr int64_t kGradMaxTensors = int64_t(1) << 24;
constexpr int64_t kGradMaxElems = int64_t(1) << 44;
constexpr int kGradSmallCap = 64;          // entries of the two parameter blocks: 2 KB and 30 KB (a
constexpr int kGradLargeCap = 1024;        // kernel's parameters end at 32,764 bytes)
static_assert(sizeof(GradList<kGradLargeCap>) + 64 <= 32764, "kernel parameters");

int check_grads(const cudallm_tensor *t, int64_t count, bool scaled, int64_t *total, int64_t *live)
{
    if (count < 0 || count > kGradMaxTensors) return CUDALLM_ERR_INVALID_DIM;
    if (count > 0 && !t) return CUDALLM_ERR_INVALID_POINTER;
    *total = *live = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (t[i].n < 0 || t[i].n > (int64_t(1) << 40)) return CUDALLM_ERR_INVALID_DIM;
        if (!valid_dtype(t[i].dtype)) return CUDALLM_ERR_INVALID_DTYPE;
        if (t[i].n == 0) continue;
        if (!t[i].data || (scaled && !t[i].out)) return CUDALLM_ERR_INVALID_POINTER;
        if (off(t[i].data, elem_size(t[i].dtype)) || (scaled && off(t[i].out, elem_size(t[i].dtype))))
            return CUDALLM_ERR_MISALIGNED;
        *total += t[i].n;
        ++*live;
        if (*total > kGradMaxElems) return CUDALLM_ERR_INVALID_DIM;
    }
    return CUDALLM_OK;
}

// Elements per chunk: about eight chunks per SM, within 2048 (eight elements a thread) and
// 16384 (enough 16-byte loads in a row to pay for finding the chunk).
constexpr int64_t kGradMaxChunk = 16384;
unsigned grad_chunk_elems(int64_t total, int sms)
{
    const int64_t c = cdiv(cdiv(total, (int64_t)sms * 8), 2048) * 2048;
    return (unsigned)std::min<int64_t>(kGradMaxChunk, std::max<int64_t>(2048, c));
}

// Fills `l` with entries from t[*next] on; returns the CTAs that its chunks occupy (0: no entry left).
template <int CAP>
unsigned fill_list(GradList<CAP> &l, const cudallm_tensor *t, int64_t count, int64_t *next, unsigned chunk, int sms)
{
    l.count = 0;
    l.chunk = chunk;
    uint64_t chunks = 0;                                  // <= 2^44 / 16384 + 2^24: fits 32 bits
    int64_t i = *next;
    for (; i < count && l.count < CAP; ++i) {
        if (t[i].n == 0) continue;
        const uint64_t c = (uint64_t)cdiv(t[i].n, chunk);
        l.data[l.count] = t[i].data;
        l.out[l.count] = t[i].out;
        l.n[l.count] = t[i].n;
        l.dtype[l.count] = (unsigned char)t[i].dtype;
        l.first[l.count] = (unsigned)chunks;
        ++l.count;
        chunks += c;
    }
    l.first[l.count] = (unsigned)chunks;
    *next = i;
    return (unsigned)std::min<uint64_t>(chunks, (uint64_t)std::min(kGradMaxBlocks, 8 * sms));
}

// Launches that write at most CAP entries' partial sums each, then either the join (norm only)
// or the scaling launches.
template <int CAP>
int run_grads(const cudallm_tensor *t, int64_t count, int64_t total, int sms, bool want_norm, bool want_scale,
              float max_norm, float eps, float *norm, double *partials, size_t max_partials, cudaStream_t stream)
{
    GradList<CAP> l;
    const unsigned chunk = grad_chunk_elems(total, sms);
    int64_t next = 0;
    int nparts = 0, st = CUDALLM_OK;
    bool one = false;
    unsigned grid = 0;
    if (want_norm) {
        while (next < count && (grid = fill_list(l, t, count, &next, chunk, sms)) != 0) {
            if ((size_t)nparts + grid > max_partials) return CUDALLM_ERR_WORKSPACE;
            st = rt_launch(grad_norm_kernel<CAP>, dim3(grid), kGradThreads, 0, stream, l, partials + nparts);
            if (st != CUDALLM_OK) return st;
            one = nparts == 0;
            nparts += (int)grid;
        }
        // one list: the scaling launch joins the partial sums itself
        one = one && want_scale;
        if (!one) {
            st = rt_launch(grad_norm_join_kernel, dim3(1), kGradThreads, 0, stream, (const double *)partials, nparts, norm);
            if (st != CUDALLM_OK) return st;
        }
    }
    if (!want_scale) return CUDALLM_OK;
    // Chunks of full length fill a loop of eight pieces a thread (norm and scaling of 403 M bf16 values: 396 us, with four 413); below that
    // the registers of eight leave fewer CTAs on an SM and nothing to fill them (6.8 M: 11.0 us, with four 10.0).
    const auto scale = chunk == kGradMaxChunk ? grad_scale_kernel<CAP, 8> : grad_scale_kernel<CAP, 4>;
    next = 0;
    while (next < count && (grid = fill_list(l, t, count, &next, chunk, sms)) != 0) {
        st = rt_launch(scale, dim3(grid), kGradThreads, 0, stream, l,
                       one ? (const double *)partials : (const double *)nullptr, nparts, norm, max_norm, eps);
        if (st != CUDALLM_OK) return st;
    }
    return CUDALLM_OK;
}

int grads(const cudallm_tensor *t, int64_t count, bool want_norm, bool want_scale, float max_norm, float eps,
          float *norm, void *scratch, size_t scratch_bytes, void *stream_v)
{
    int64_t total = 0, live = 0;
    int st = check_grads(t, count, want_scale, &total, &live);
    if (st != CUDALLM_OK) return st;
    if (want_scale && (!(max_norm >= 0.f) || !(eps >= 0.f))) return CUDALLM_ERR_INVALID_DIM;
    if (!norm) return CUDALLM_ERR_INVALID_POINTER;
    if (off(norm, 4)) return CUDALLM_ERR_MISALIGNED;
    if (want_norm && (!scratch || off(scratch, 16) || scratch_bytes < cudallm_grad_norm_scratch_bytes(live)))
        return CUDALLM_ERR_WORKSPACE;
    if (live == 0 && !want_norm) return CUDALLM_OK;
    int dev = 0, sms = 0;
    st = rt_current_device(&dev, &sms);
    if (st != CUDALLM_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    double *partials = static_cast<double *>(scratch);
    const size_t cap = scratch_bytes / sizeof(double);
    if (live <= kGradSmallCap)
        return run_grads<kGradSmallCap>(t, count, total, sms, want_norm, want_scale, max_norm, eps, norm, partials, cap, stream);
    return run_grads<kGradLargeCap>(t, count, total, sms, want_norm, want_scale, max_norm, eps, norm, partials, cap, stream);
}

}  // namespace

extern "C" {

int cudallm_layernorm_rows(const void *x, const void *gamma, const void *beta, void *y, float *mean, float *rstd,
                           int64_t rows, int64_t n, int64_t ldx, int64_t ldy, int dtype, int param_dtype, float eps,
                           void *stream_v)
{
    int st = check_ln(rows, n, dtype, param_dtype);
    if (st != CUDALLM_OK) return st;
    if (!(eps >= 0.f) || !(eps <= 3.0e38f)) return CUDALLM_ERR_INVALID_DIM;
    if (rows == 0 || n == 0) return CUDALLM_OK;
    if ((st = check_ld(rows, n, ldx)) != CUDALLM_OK || (st = check_ld(rows, n, ldy)) != CUDALLM_OK) return st;
    if (!x || !y) return CUDALLM_ERR_INVALID_POINTER;
    if (y == x && ldy != ldx && rows > 1) return CUDALLM_ERR_INVALID_LD;      // rows would be read after others lie over them
    const int es = elem_size(dtype), ps = elem_size(param_dtype);
    if (off(x, es) || off(y, es) || off(gamma, ps) || off(beta, ps) || off(mean, 4) || off(rstd, 4))
        return CUDALLM_ERR_MISALIGNED;
    int dev = 0, sms = 0;
    if ((st = rt_current_device(&dev, &sms)) != CUDALLM_OK) return st;
    LnRowsParams p{};
    p.x = x; p.gamma = gamma; p.beta = beta; p.y = y; p.mean = mean; p.rstd = rstd;
    p.ldx = ldx; p.ldy = ldy;
    p.rows = (int)rows; p.n = (int)n; p.param_dtype = param_dtype;
    p.eps = eps;
    p.inv_n = 1.f / (float)n;
    const LnLaunch at{dev, sms, static_cast<cudaStream_t>(stream_v)};
    if (dtype == CUDALLM_F32) return run_ln<float>(p, at);
    if (dtype == CUDALLM_BF16) return run_ln<__nv_bfloat16>(p, at);
    return run_ln<__half>(p, at);
}

size_t cudallm_layernorm_rows_bwd_scratch_bytes(int64_t rows, int64_t n)
{
    if (rows < 0 || n < 0 || rows > kMaxDim || n > kMaxDim) return 0;
    return (size_t)(std::min<int64_t>(std::max<int64_t>(rows, 1), ln_max_parts(n)) * n * 8);
}

int cudallm_layernorm_rows_bwd(const void *dy, const void *x, const void *gamma, const float *mean, const float *rstd,
                               void *dx, void *dgamma, void *dbeta, int64_t rows, int64_t n, int64_t lddy, int64_t ldx,
                               int64_t lddx, int dtype, int param_dtype, void *scratch, size_t scratch_bytes,
                               void *stream_v)
{
    int st = check_ln(rows, n, dtype, param_dtype);
    if (st != CUDALLM_OK) return st;
    if (n == 0 || (!dx && !dgamma && !dbeta)) return CUDALLM_OK;
    const int es = elem_size(dtype), ps = elem_size(param_dtype);
    if (rows > 0) {
        if ((st = check_ld(rows, n, lddy)) != CUDALLM_OK || (st = check_ld(rows, n, ldx)) != CUDALLM_OK) return st;
        if (dx && (st = check_ld(rows, n, lddx)) != CUDALLM_OK) return st;
        if (!dy || !x || !mean || !rstd) return CUDALLM_ERR_INVALID_POINTER;
        if (rows > 1 && ((dx == x && lddx != ldx) || (dx == dy && lddx != lddy))) return CUDALLM_ERR_INVALID_LD;
    }
    if (off(dy, es) || off(x, es) || off(dx, es) || off(gamma, ps) || off(dgamma, ps) || off(dbeta, ps) || off(mean, 4)
        || off(rstd, 4))
        return CUDALLM_ERR_MISALIGNED;
    const bool sums = dgamma || dbeta;
    if (sums && (!scratch || off(scratch, 16) || scratch_bytes < cudallm_layernorm_rows_bwd_scratch_bytes(rows, n)))
        return CUDALLM_ERR_WORKSPACE;
    if (rows == 0 && !sums) return CUDALLM_OK;
    int dev = 0, sms = 0;
    if ((st = rt_current_device(&dev, &sms)) != CUDALLM_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    int parts = 0;
    if (rows > 0) {
        LnRowsParams p{};
        p.x = x; p.dy = dy; p.gamma = gamma; p.y = dx;
        p.mean = const_cast<float *>(mean); p.rstd = const_cast<float *>(rstd);
        p.partials = sums ? static_cast<float *>(scratch) : nullptr;
        p.ldx = ldx; p.lddy = lddy; p.ldy = lddx;
        p.rows = (int)rows; p.n = (int)n; p.param_dtype = param_dtype;
        p.inv_n = 1.f / (float)n;
        const LnLaunch at{dev, sms, stream};
        if (dtype == CUDALLM_F32) st = run_ln_bwd<float>(p, at, &parts);
        else if (dtype == CUDALLM_BF16) st = run_ln_bwd<__nv_bfloat16>(p, at, &parts);
        else st = run_ln_bwd<__half>(p, at, &parts);
        if (st != CUDALLM_OK) return st;
    }
    if (!sums) return CUDALLM_OK;
    LnJoinParams j{};
    j.partials = static_cast<const float *>(scratch);
    j.dgamma = dgamma; j.dbeta = dbeta;
    j.n = (int)n; j.parts = parts; j.param_dtype = param_dtype;
    return rt_launch(layernorm_join_kernel, dim3((unsigned)cdiv(n, 32), 2), 1024, 0, stream, j);
}

size_t cudallm_grad_norm_scratch_bytes(int64_t count)
{
    if (count < 0 || count > kGradMaxTensors) return 0;
    const int64_t launches = std::max<int64_t>(1, cdiv(count, kGradLargeCap));     // of up to kGradLargeCap tensors
    return (size_t)(launches * kGradMaxBlocks) * sizeof(double);
}

int cudallm_grad_norm(const cudallm_tensor *tensors, int64_t count, float *norm, void *scratch, size_t scratch_bytes,
                      void *stream)
{
    return grads(tensors, count, true, false, 0.f, 0.f, norm, scratch, scratch_bytes, stream);
}

int cudallm_grad_clip(const cudallm_tensor *tensors, int64_t count, const float *norm, float max_norm, float eps,
                      void *stream)
{
    return grads(tensors, count, false, true, max_norm, eps, const_cast<float *>(norm), nullptr, 0, stream);
}

int cudallm_grad_clip_norm(const cudallm_tensor *tensors, int64_t count, float max_norm, float eps, float *norm,
                           void *scratch, size_t scratch_bytes, void *stream)
{
    return grads(tensors, count, true, true, max_norm, eps, norm, scratch, scratch_bytes, stream);
}

}  // extern "C"
