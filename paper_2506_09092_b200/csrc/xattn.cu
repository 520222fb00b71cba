// Cross attention entry points of include/cudallm_layers.h: validation, the choice of kernel and of
// the split over the keys, tensor maps and launches.
#include "../../include/cudallm_layers.h"

#include <algorithm>
#include <atomic>
#include <cmath>

#include "runtime.h"
#include "xattn_fwd.cuh"
#include "xattn_token.cuh"
#include "xattn_bwd.cuh"

using namespace cudallm;

namespace {

__device__ int g_xattn_status[2];

constexpr int64_t kMaxDim = (int64_t(1) << 31) - 1024;
constexpr int64_t kMaxElems = int64_t(1) << 38;          // per operand: byte strides of tensor maps stay below 2^40
constexpr int64_t kPlanSms = 148;                        // the split over the keys is planned for this many SMs

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return cdiv(a, b) * b; }
inline bool off(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

// Nothing to read or write at all; no queries.
bool is_void(const cudallm_xattn_shape &s) { return s.batch == 0 || s.q_heads == 0 || s.head_dim == 0; }
bool is_empty(const cudallm_xattn_shape &s) { return is_void(s) || s.q_rows == 0; }

// Strides of a (batch, rows, heads, head_dim) operand: multiples of 8, no two elements in one place.
int check_strides(const int64_t (&st)[3], int64_t batch, int64_t rows, int64_t heads, int64_t dim)
{
    const int64_t ext[3] = {batch, rows, heads};
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

int check_shape(const cudallm_xattn_shape *sp)
{
    if (!sp) return CUDALLM_ERR_INVALID_POINTER;
    const cudallm_xattn_shape &s = *sp;
    if (s.dtype != CUDALLM_BF16 && s.dtype != CUDALLM_F16) return CUDALLM_ERR_INVALID_DTYPE;
    for (int64_t v : {s.batch, s.q_rows, s.kv_rows, s.q_heads, s.kv_heads, s.head_dim})
        if (v < 0 || v > kMaxDim) return CUDALLM_ERR_INVALID_DIM;
    if (!(s.scale >= 0.f) || !(s.scale <= 3.0e38f)) return CUDALLM_ERR_INVALID_DIM;
    if (is_void(s)) return CUDALLM_OK;
    if (s.kv_heads == 0 || s.q_heads % s.kv_heads) return CUDALLM_ERR_INVALID_DIM;
    if (s.head_dim % 8 || s.head_dim > 128) return CUDALLM_ERR_UNSUPPORTED_SHAPE;
    if ((long double)s.batch * s.q_heads * cdiv(s.q_rows, kXaRows) > (long double)kMaxDim
        || (long double)s.batch * s.kv_heads * cdiv(s.kv_rows, kXaRows) > (long double)kMaxDim)
        return CUDALLM_ERR_INVALID_DIM;
    if ((long double)s.batch * s.q_heads * s.q_rows * s.head_dim > (long double)kMaxElems) return CUDALLM_ERR_INVALID_DIM;
    int st = CUDALLM_OK;
    if (s.q_rows > 0) {
        st = check_strides(s.q_stride, s.batch, s.q_rows, s.q_heads, s.head_dim);
        if (st == CUDALLM_OK) st = check_strides(s.o_stride, s.batch, s.q_rows, s.q_heads, s.head_dim);
    }
    if (s.kv_rows > 0) {
        if (st == CUDALLM_OK) st = check_strides(s.k_stride, s.batch, s.kv_rows, s.kv_heads, s.head_dim);
        if (st == CUDALLM_OK) st = check_strides(s.v_stride, s.batch, s.kv_rows, s.kv_heads, s.head_dim);
    }
    return st;
}

// How the forward call runs: which kernel, and into how many parts the keys are cut.
struct FwdPlan {
    bool token;
    int splits;
    int64_t per_split;          // keys (token), blocks of 128 keys (else)
    int64_t rows_all;           // batch * q_heads * q_rows
    size_t scratch;
};
FwdPlan plan_fwd(const cudallm_xattn_shape &s)
{
    FwdPlan f{};
    f.rows_all = s.batch * s.q_heads * s.q_rows;
    f.token = (s.q_heads / s.kv_heads) * s.q_rows <= kXaTokRows;
    const int64_t kv = std::max<int64_t>(s.kv_rows, 1);
    int64_t want;
    if (f.token) {
        // one wave of two CTAs per SM (two waves: 19.4 instead of 14.9 us on 16 x 16 heads of 64 x 1500 states);
        // at least 256 keys each
        want = std::min<int64_t>({int64_t(32), 2 * kPlanSms / (s.batch * s.kv_heads), kv / 256});
        f.per_split = round_up(cdiv(kv, std::max<int64_t>(want, 1)), 32);
        f.splits = (int)cdiv(kv, f.per_split);
    } else {
        // one CTA per SM; at least two blocks each
        const int64_t blocks = cdiv(kv, kXaRows), ctas = s.batch * s.q_heads * cdiv(s.q_rows, 2 * kXaRows);
        want = std::min<int64_t>({int64_t(32), kPlanSms / ctas, blocks / 2});
        f.per_split = cdiv(blocks, std::max<int64_t>(want, 1));
        f.splits = (int)cdiv(blocks, f.per_split);
    }
    f.scratch = f.splits > (f.token ? kXaTokCluster : 1) ? (size_t)f.splits * (size_t)f.rows_all * (size_t)(s.head_dim + 1) * sizeof(float) : 0;
    return f;
}

// Factor of the exponentials' arguments.  Masked scores are -inf, and -inf x 0 is no number, so a
// scale of 0 enters as 1e-30: every finite score then gives exp2(0) = 1 all the same.
inline float scale_log2(const cudallm_xattn_shape &s) { return std::max(s.scale, 1e-30f) * 1.4426950408889634f; }

// The backward call's parts (see xattn_bwd.cuh), planned for kPlanSms SMs, and where they lie in the scratch.
struct BwdPlan {
    int dq_parts, dkv_parts, dq_blocks, dkv_blocks;
    int64_t q_elems, kv_elems;                  // of one part of dQ; of dK and of dV
    size_t off_dq, off_dk, off_dv, scratch;     // in floats; bytes
};
int parts_for(int64_t ctas, int64_t blocks, int *per_part)
{
    // at least two blocks a part: one costs about as much as starting a CTA
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>({int64_t(32), kPlanSms / std::max<int64_t>(ctas, 1), blocks / 2}));
    *per_part = (int)cdiv(std::max<int64_t>(blocks, 1), want);
    return (int)std::max<int64_t>(1, cdiv(blocks, *per_part));
}
BwdPlan plan_bwd(const cudallm_xattn_shape &s)
{
    BwdPlan f{};
    const int64_t q_tiles = cdiv(s.q_rows, kXaRows), kv_tiles = cdiv(s.kv_rows, kXaRows), group = s.q_heads / s.kv_heads;
    f.dq_parts = parts_for(s.batch * s.q_heads * q_tiles, kv_tiles, &f.dq_blocks);
    f.dkv_parts = parts_for(s.batch * s.kv_heads * kv_tiles, group * q_tiles, &f.dkv_blocks);
    f.q_elems = s.batch * s.q_heads * s.q_rows * s.head_dim;
    f.kv_elems = s.batch * s.kv_heads * s.kv_rows * s.head_dim;
    f.off_dq = (size_t)round_up(s.batch * s.q_heads * s.q_rows, 4);             // behind delta
    f.off_dk = f.off_dq + (f.dq_parts > 1 ? (size_t)f.dq_parts * f.q_elems : 0);
    f.off_dv = f.off_dk + (f.dkv_parts > 1 ? (size_t)f.dkv_parts * f.kv_elems : 0);
    f.scratch = (f.off_dv + (f.dkv_parts > 1 ? (size_t)f.dkv_parts * f.kv_elems : 0)) * sizeof(float);
    return f;
}

inline XaStrides strides(const int64_t (&s)[3]) { return XaStrides{(long long)s[0], (long long)s[1], (long long)s[2]}; }

// Tensor map of an operand; an absent one (no rows; its strides are not checked then) gets a map of one row
// of `other` that no kernel uses.
int encode(CUtensorMap *tm, const void *base, const void *other, bool f16, const int64_t (&st)[3], int64_t batch, int64_t rows,
           int64_t heads, int64_t dim)
{
    if (rows == 0) {
        base = other;
        batch = rows = heads = 1;
    }
    const uint64_t dims[4] = {(uint64_t)dim, (uint64_t)heads, (uint64_t)rows, (uint64_t)batch};
    const int64_t used[3] = {heads > 1 ? st[2] : 8, rows > 1 ? st[1] : 8, batch > 1 ? st[0] : 8};
    const uint64_t bytes[3] = {(uint64_t)used[0] * 2, (uint64_t)used[1] * 2, (uint64_t)used[2] * 2};
    return rt_encode_rows(tm, base, f16, dims, bytes, kXaRows);
}

std::atomic<int *> g_status_at[kRtMaxDevices] = {};      // g_xattn_status of each device that has launched a kernel which writes it

int status_word(int dev, int **out)
{
    int *p = g_status_at[dev].load(std::memory_order_relaxed);
    if (!p) {
        RT_CUDA_TRY(cudaGetSymbolAddress(reinterpret_cast<void **>(&p), g_xattn_status));
        g_status_at[dev].store(p, std::memory_order_relaxed);
    }
    *out = p;
    return CUDALLM_OK;
}

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

template <typename T>
int join(const cudallm_xattn_shape &s, const FwdPlan &f, const float *o_part, const float *lse_part, void *o, float *lse,
         cudaStream_t stream)
{
    XaJoinParams j{};
    j.o_part = o_part; j.lse_part = lse_part;
    j.o = o; j.lse = lse;
    j.so = strides(s.o_stride);
    j.q_rows = (int)s.q_rows; j.q_heads = (int)s.q_heads; j.head_dim = (int)s.head_dim; j.splits = f.splits;
    j.rows_all = f.rows_all;
    return rt_launch(xattn_join_kernel<T>, dim3((unsigned)cdiv(f.rows_all, 8)), 256, 0, stream, j);
}

template <int DP, typename T>
int run_fwd(const cudallm_xattn_shape &s, const FwdPlan &f, const void *q, const void *k, const void *v, const int32_t *lens,
            void *o, float *lse, float *scratch, int dev, cudaStream_t stream)
{
    float *o_part = scratch, *lse_part = scratch ? scratch + (size_t)f.splits * f.rows_all * s.head_dim : nullptr;
    int st;
    if (f.token) {
        using L = XaTokSmem<DP>;
        static std::atomic<bool> done[kRtMaxDevices] = {};
        if ((st = allow_smem(xattn_token_kernel<DP, T>, L::kBytes, done, dev)) != CUDALLM_OK) return st;
        XaTokParams p{};
        p.q = q; p.k = k; p.v = v; p.o = o; p.lse = lse; p.o_part = o_part; p.lse_part = lse_part; p.lens = lens;
        p.sq = strides(s.q_stride); p.sk = strides(s.k_stride); p.sv = strides(s.v_stride); p.so = strides(s.o_stride);
        p.q_rows = (int)s.q_rows; p.kv_rows = (int)s.kv_rows; p.q_heads = (int)s.q_heads; p.kv_heads = (int)s.kv_heads;
        p.group = (int)(s.q_heads / s.kv_heads); p.batch = (int)s.batch; p.head_dim = (int)s.head_dim;
        p.splits = f.splits; p.keys_per_split = (int)f.per_split;
        p.scale = s.scale; p.scale_log2 = scale_log2(s);
        p.cluster = f.splits > 1 && f.splits <= kXaTokCluster;
        st = rt_launch_cluster(xattn_token_kernel<DP, T>, dim3((unsigned)(s.batch * s.kv_heads * f.splits)),
                               p.cluster ? (unsigned)f.splits : 1u, kXaTokThreads, (size_t)L::kBytes, stream, p);
        if (p.cluster) return st;
    } else {
        using L = XaFwdSmem<DP>;
        static std::atomic<bool> done[kRtMaxDevices] = {};
        if ((st = allow_smem(xattn_fwd_kernel<DP, T>, L::kBytes, done, dev)) != CUDALLM_OK) return st;
        const bool f16 = s.dtype == CUDALLM_F16;
        CUtensorMap tq, tk, tv;
        if ((st = encode(&tq, q, q, f16, s.q_stride, s.batch, s.q_rows, s.q_heads, s.head_dim)) != CUDALLM_OK
            || (st = encode(&tk, k, q, f16, s.k_stride, s.batch, s.kv_rows, s.kv_heads, s.head_dim)) != CUDALLM_OK
            || (st = encode(&tv, v, q, f16, s.v_stride, s.batch, s.kv_rows, s.kv_heads, s.head_dim)) != CUDALLM_OK)
            return st;
        XaFwdParams p{};
        p.o = o; p.lse = lse; p.o_part = o_part; p.lse_part = lse_part; p.lens = lens;
        p.so = strides(s.o_stride);
        p.q_rows = (int)s.q_rows; p.kv_rows = (int)s.kv_rows; p.q_heads = (int)s.q_heads;
        p.group = (int)(s.q_heads / s.kv_heads); p.batch = (int)s.batch; p.head_dim = (int)s.head_dim;
        p.q_tiles = (int)cdiv(s.q_rows, 2 * kXaRows);
        p.splits = f.splits; p.tiles_per_split = (int)f.per_split;
        p.scale = s.scale; p.scale_log2 = scale_log2(s);
        if ((st = status_word(dev, &p.status)) != CUDALLM_OK) return st;
        p.skip_loads = rt_take_skip_loads();
        p.wait_limit_ns = rt_wait_limit_ns();
        st = rt_launch(xattn_fwd_kernel<DP, T>, dim3((unsigned)((int64_t)p.q_tiles * s.q_heads * s.batch), (unsigned)f.splits),
                       kXaFwdThreads, (size_t)L::kBytes, stream, tq, tk, tv, p);
    }
    if (st != CUDALLM_OK || f.splits == 1) return st;
    return join<T>(s, f, o_part, lse_part, o, lse, stream);
}

template <int DP, typename T>
int run_bwd(const cudallm_xattn_shape &s, const void *q, const void *k, const void *v, const int32_t *lens, const void *o,
            const float *lse, const void *d_o, void *dq, void *dk, void *dv, float *scratch, int dev, cudaStream_t stream)
{
    const BwdPlan f = plan_bwd(s);
    using L = XaBwdSmem<DP>;
    static std::atomic<bool> done_dq[kRtMaxDevices] = {}, done_dkv[kRtMaxDevices] = {};
    int st;
    if ((st = allow_smem(xattn_dq_kernel<DP, T>, L::kBytes, done_dq, dev)) != CUDALLM_OK
        || (st = allow_smem(xattn_dkv_kernel<DP, T>, L::kBytes, done_dkv, dev)) != CUDALLM_OK)
        return st;
    const bool f16 = s.dtype == CUDALLM_F16;
    CUtensorMap tq, tk, tv, tdo;
    if ((st = encode(&tq, q, k, f16, s.q_stride, s.batch, s.q_rows, s.q_heads, s.head_dim)) != CUDALLM_OK
        || (st = encode(&tk, k, q, f16, s.k_stride, s.batch, s.kv_rows, s.kv_heads, s.head_dim)) != CUDALLM_OK
        || (st = encode(&tv, v, q, f16, s.v_stride, s.batch, s.kv_rows, s.kv_heads, s.head_dim)) != CUDALLM_OK
        || (st = encode(&tdo, d_o, k, f16, s.o_stride, s.batch, s.q_rows, s.q_heads, s.head_dim)) != CUDALLM_OK)
        return st;
    XaBwdParams p{};
    p.o = o; p.d_o = d_o; p.dq = dq; p.dk = dk; p.dv = dv; p.lse = lse; p.delta = scratch; p.lens = lens;
    if (scratch && f.dq_parts > 1) p.dq_part = scratch + f.off_dq;
    if (scratch && f.dkv_parts > 1) { p.dk_part = scratch + f.off_dk; p.dv_part = scratch + f.off_dv; }
    p.dq_blocks = f.dq_blocks; p.dkv_blocks = f.dkv_blocks;
    p.sq = strides(s.q_stride); p.sk = strides(s.k_stride); p.sv = strides(s.v_stride); p.so = strides(s.o_stride);
    p.q_rows = (int)s.q_rows; p.kv_rows = (int)s.kv_rows; p.q_heads = (int)s.q_heads; p.kv_heads = (int)s.kv_heads;
    p.group = (int)(s.q_heads / s.kv_heads); p.batch = (int)s.batch; p.head_dim = (int)s.head_dim;
    p.q_tiles = (int)cdiv(s.q_rows, kXaRows); p.kv_tiles = (int)cdiv(s.kv_rows, kXaRows);
    p.scale = s.scale; p.scale_log2 = scale_log2(s);
    if ((st = status_word(dev, &p.status)) != CUDALLM_OK) return st;
    p.wait_limit_ns = rt_wait_limit_ns();
    p.skip_loads = rt_take_skip_loads();
    if (s.q_rows > 0) {
        st = rt_launch(xattn_dq_kernel<DP, T>, dim3((unsigned)((int64_t)p.q_tiles * s.q_heads * s.batch), (unsigned)f.dq_parts),
                       kXaBwdThreads, (size_t)L::kBytes, stream, tq, tk, tv, tdo, p);
        p.skip_loads = 0;
    }
    if (st == CUDALLM_OK && dk && s.kv_rows > 0)
        st = rt_launch(xattn_dkv_kernel<DP, T>, dim3((unsigned)((int64_t)p.kv_tiles * s.kv_heads * s.batch), (unsigned)f.dkv_parts),
                       kXaBwdThreads, (size_t)L::kBytes, stream, tq, tk, tv, tdo, p);
    // the parts' sums
    if (st == CUDALLM_OK && s.q_rows > 0 && f.dq_parts > 1) {
        XaGradJoinParams j{};
        j.part[0] = p.dq_part; j.out[0] = dq; j.st[0] = p.sq; j.f[0] = s.scale;
        j.parts = f.dq_parts; j.rows = p.q_rows; j.heads = p.q_heads; j.head_dim = p.head_dim;
        j.rows_all = s.batch * s.q_heads * s.q_rows;
        st = rt_launch(xattn_grad_join_kernel<T>, dim3((unsigned)cdiv(f.q_elems / 4, 256)), 256, 0, stream, j);
    }
    if (st == CUDALLM_OK && dk && s.kv_rows > 0 && f.dkv_parts > 1) {
        XaGradJoinParams j{};
        j.part[0] = p.dk_part; j.out[0] = dk; j.st[0] = p.sk; j.f[0] = s.scale;
        j.part[1] = p.dv_part; j.out[1] = dv; j.st[1] = p.sv; j.f[1] = 1.f;
        j.parts = f.dkv_parts; j.rows = p.kv_rows; j.heads = p.kv_heads; j.head_dim = p.head_dim;
        j.rows_all = s.batch * s.kv_heads * s.kv_rows;
        st = rt_launch(xattn_grad_join_kernel<T>, dim3((unsigned)cdiv(f.kv_elems / 4, 256), 2), 256, 0, stream, j);
    }
    return st;
}

}  // namespace

namespace cudallm {

int rt_xattn_status(int dev, int (&host)[2])
{
    int *p = g_status_at[dev].load(std::memory_order_relaxed);
    if (!p) return CUDALLM_OK;
    RT_CUDA_TRY(cudaMemcpy(host, p, sizeof host, cudaMemcpyDeviceToHost));
    if (host[0] != 0) RT_CUDA_TRY(cudaMemset(p, 0, sizeof host));
    return CUDALLM_OK;
}

}  // namespace cudallm

extern "C" {

size_t cudallm_xattn_fwd_scratch_bytes(const cudallm_xattn_shape *shape)
{
    if (check_shape(shape) != CUDALLM_OK || is_empty(*shape)) return 0;
    return plan_fwd(*shape).scratch;
}

int cudallm_xattn_fwd(const cudallm_xattn_shape *shape, const void *q, const void *k, const void *v, const int32_t *kv_lens,
                      void *o, float *lse, void *scratch, size_t scratch_bytes, void *stream_v)
{
    int st = check_shape(shape);
    if (st != CUDALLM_OK) return st;
    const cudallm_xattn_shape &s = *shape;
    if (is_empty(s)) return CUDALLM_OK;
    if (!q || !o || (s.kv_rows > 0 && (!k || !v))) return CUDALLM_ERR_INVALID_POINTER;
    if (off(kv_lens, 4) || off(lse, 4)) return CUDALLM_ERR_MISALIGNED;
    if (off(q, 16) || off(o, 16) || (s.kv_rows > 0 && (off(k, 16) || off(v, 16)))) return CUDALLM_ERR_UNSUPPORTED_SHAPE;
    const FwdPlan f = plan_fwd(s);
    if (f.scratch && (!scratch || off(scratch, 16) || scratch_bytes < f.scratch)) return CUDALLM_ERR_WORKSPACE;
    if (f.rows_all * (int64_t)f.splits > kMaxElems || s.batch * s.kv_heads * (int64_t)f.splits > kMaxDim)
        return CUDALLM_ERR_INVALID_DIM;
    int dev = 0, sms = 0;
    if ((st = rt_current_device(&dev, &sms)) != CUDALLM_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    float *scr = f.scratch ? static_cast<float *>(scratch) : nullptr;
    const bool wide = s.head_dim > 64;
    if (s.dtype == CUDALLM_BF16)
        return wide ? run_fwd<128, __nv_bfloat16>(s, f, q, k, v, kv_lens, o, lse, scr, dev, stream)
                    : run_fwd<64, __nv_bfloat16>(s, f, q, k, v, kv_lens, o, lse, scr, dev, stream);
    return wide ? run_fwd<128, __half>(s, f, q, k, v, kv_lens, o, lse, scr, dev, stream)
                : run_fwd<64, __half>(s, f, q, k, v, kv_lens, o, lse, scr, dev, stream);
}

size_t cudallm_xattn_bwd_scratch_bytes(const cudallm_xattn_shape *shape)
{
    if (check_shape(shape) != CUDALLM_OK || is_empty(*shape)) return 0;
    return plan_bwd(*shape).scratch;
}

int cudallm_xattn_bwd(const cudallm_xattn_shape *shape, const void *q, const void *k, const void *v, const int32_t *kv_lens,
                      const void *o, const float *lse, const void *d_o, void *dq, void *dk, void *dv, void *scratch,
                      size_t scratch_bytes, void *stream_v)
{
    int st = check_shape(shape);
    if (st != CUDALLM_OK) return st;
    const cudallm_xattn_shape &s = *shape;
    const bool queries = s.q_rows > 0, kv = s.kv_rows > 0;
    if (is_void(s) || (!queries && !kv)) return CUDALLM_OK;
    if ((queries && (!q || !o || !lse || !d_o || !dq)) || (kv && (!k || !v || !dk != !dv))) return CUDALLM_ERR_INVALID_POINTER;
    if (off(kv_lens, 4) || off(lse, 4)) return CUDALLM_ERR_MISALIGNED;
    if ((queries && (off(q, 16) || off(o, 16) || off(d_o, 16) || off(dq, 16)))
        || (kv && (off(k, 16) || off(v, 16) || off(dk, 16) || off(dv, 16))))
        return CUDALLM_ERR_UNSUPPORTED_SHAPE;
    if (queries && (!scratch || off(scratch, 16) || scratch_bytes < cudallm_xattn_bwd_scratch_bytes(shape)))
        return CUDALLM_ERR_WORKSPACE;
    if (!queries && !dk) return CUDALLM_OK;
    int dev = 0, sms = 0;
    if ((st = rt_current_device(&dev, &sms)) != CUDALLM_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    float *scr = queries ? static_cast<float *>(scratch) : nullptr;
    const bool wide = s.head_dim > 64;
    if (s.dtype == CUDALLM_BF16)
        return wide ? run_bwd<128, __nv_bfloat16>(s, q, k, v, kv_lens, o, lse, d_o, dq, dk, dv, scr, dev, stream)
                    : run_bwd<64, __nv_bfloat16>(s, q, k, v, kv_lens, o, lse, d_o, dq, dk, dv, scr, dev, stream);
    return wide ? run_bwd<128, __half>(s, q, k, v, kv_lens, o, lse, d_o, dq, dk, dv, scr, dev, stream)
                : run_bwd<64, __half>(s, q, k, v, kv_lens, o, lse, d_o, dq, dk, dv, scr, dev, stream);
}

}  // extern "C"
