// The norm of many tensors together, and scaling them by min(1, max_norm / (norm + eps)).
//
// The list of tensors travels in the kernels' parameters (constant memory): no copy, no
// table on the device to keep alive, and a captured graph holds its own.  Every tensor is
// cut into chunks of p.chunk elements; a CTA visits chunks b, b + grid, ... and finds a
// chunk's tensor by bisection.  Bound: HBM; the second kernel visits the chunks in reverse, so
// that it starts with what the first one left in L2.
// Measured (one B200): 403 M bf16 values in 291 tensors, scaled into other buffers: 396 us; the norm alone 130-134
// us = 6.0-6.2 TB/s, the scaling alone 278 us = 5.8 TB/s; 6.8 M in 27 tensors: 10 us.  Eviction priorities for the chunks
// that the second pass meets first: 407 to 410 instead of then 414 us whatever was kept, so none are given.
// In place: 408 and 10.9 us.  A group of zeros goes the way of doubles: the norm of 403 M zeros takes 143 us.
#pragma once
#include "elem.cuh"

namespace cudallm {

constexpr int kGradThreads = 256;
constexpr int kGradMaxBlocks = 1184;      // CTAs, and partial sums, of one launch

template <int CAP> struct GradList {
    void *data[CAP];
    void *out[CAP];
    long long n[CAP];
    unsigned first[CAP + 1];              // chunks before tensor i
    unsigned char dtype[CAP];
    int count;
    unsigned chunk;                       // elements: a multiple of 2048
};

struct GradChunk {
    int tensor;
    long long begin;                      // element range inside the tensor
    int len;
};
template <int CAP>
__device__ __forceinline__ GradChunk grad_chunk(const GradList<CAP> &l, unsigned c)
{
    int lo = 0, hi = l.count;             // first[lo] <= c < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.first[mid] <= c) lo = mid; else hi = mid;
    }
    GradChunk g;
    g.tensor = lo;
    g.begin = (long long)(c - l.first[lo]) * l.chunk;
    const long long left = l.n[lo] - g.begin;
    g.len = left < (long long)l.chunk ? (int)left : (int)l.chunk;
    return g;
}

// Sum of the squares of NV values.  In fp32 where that is safe: a square is rounded to 2^-24 of
// itself, and only a sum between 2^-90 and 2^120 can neither have lost an underflowing square
// that matters (each is below 2^-126 then) nor have overflowed; otherwise in double.
template <int NV>
__device__ __forceinline__ double group_squares(const float (&f)[NV])
{
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) s = fmaf(f[i], f[i], s);
    if (s > 0x1p-90f && s < 0x1p120f) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < NV; ++i) d = fma((double)f[i], (double)f[i], d);
    return d;
}

__device__ __forceinline__ double block_sum_double(double v, double *warp_part)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) warp_part[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kGradThreads / 32; ++w) s += warp_part[w];
    return s;
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const T *p, int len)
{
    constexpr int kV = ElemVec<T>::kN;
    double acc = 0.0;
    int head = (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T);
    if (head > len) head = len;
    const int nvec = (len - head) / kV;
    const T *body = p + head;
    int i = threadIdx.x;
    for (; i + 3 * kGradThreads < nvec; i += 4 * kGradThreads) {
        Piece<T, kV> v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u].load(body + (i + u * kGradThreads) * kV);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float f[kV];
            v[u].unpack(f);
            acc += group_squares<kV>(f);
        }
    }
    for (; i < nvec; i += kGradThreads) {
        Piece<T, kV> v;
        v.load(body + i * kV);
        float f[kV];
        v.unpack(f);
        acc += group_squares<kV>(f);
    }
    // elements outside the 16-byte body
    const int rest = len - nvec * kV;
    if ((int)threadIdx.x < rest) {
        const int j = (int)threadIdx.x < head ? threadIdx.x : threadIdx.x + nvec * kV;
        const double d = (double)elem_to_float(p[j]);
        acc = fma(d, d, acc);
    }
    return acc;
}

template <int CAP>
__global__ void __launch_bounds__(kGradThreads)
grad_norm_kernel(const __grid_constant__ GradList<CAP> l, double *partials)
{
    __shared__ double warp_part[kGradThreads / 32];
    grid_launch_dependents();
    grid_dependency_wait();
    double acc = 0.0;
    const unsigned total = l.first[l.count];
    for (unsigned c = blockIdx.x; c < total; c += gridDim.x) {
        const GradChunk g = grad_chunk(l, c);
        const void *base = l.data[g.tensor];
        if (l.dtype[g.tensor] == 0) acc += chunk_squares(static_cast<const float *>(base) + g.begin, g.len);
        else if (l.dtype[g.tensor] == 1) acc += chunk_squares(static_cast<const __nv_bfloat16 *>(base) + g.begin, g.len);
        else acc += chunk_squares(static_cast<const __half *>(base) + g.begin, g.len);
    }
    acc = block_sum_double(acc, warp_part);
    if (threadIdx.x == 0) partials[blockIdx.x] = acc;
}

// norm = sqrt of the sum of `count` partial sums, the same bits in every CTA that asks.
__device__ __forceinline__ float join_norm(const double *partials, int count, double *warp_part)
{
    double acc = 0.0;
    for (int i = threadIdx.x; i < count; i += kGradThreads) acc += partials[i];
    return (float)sqrt(block_sum_double(acc, warp_part));
}
__global__ void __launch_bounds__(kGradThreads)
grad_norm_join_kernel(const double *partials, int count, float *norm)
{
    __shared__ double warp_part[kGradThreads / 32];
    grid_launch_dependents();
    grid_dependency_wait();
    const float v = join_norm(partials, count, warp_part);
    if (threadIdx.x == 0) *norm = v;
}

// U pieces in flight per thread.
template <int U, typename T>
__device__ __forceinline__ void chunk_scale(const T *src, T *dst, int len, float coef)
{
    constexpr int kV = ElemVec<T>::kN;
    int head = (int)((16 - (reinterpret_cast<uintptr_t>(src) & 15)) & 15) / (int)sizeof(T);
    if (head > len) head = len;
    // source and destination off a 16-byte boundary by different amounts: element by element
    const bool same = ((reinterpret_cast<uintptr_t>(src) ^ reinterpret_cast<uintptr_t>(dst)) & 15) == 0;
    const int nvec = same ? (len - head) / kV : 0;
    if (!same) head = 0;
    int i = threadIdx.x;
    const T *sb = src + head;
    T *db = dst + head;
    for (; i + (U - 1) * kGradThreads < nvec; i += U * kGradThreads) {
        Piece<T, kV> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u].load(sb + (i + u * kGradThreads) * kV);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[kV];
            v[u].unpack(f);
#pragma unroll
            for (int e = 0; e < kV; ++e) f[e] *= coef;
            v[u].pack(f);
            v[u].store_stream(db + (i + u * kGradThreads) * kV);
        }
    }
    for (; i < nvec; i += kGradThreads) {
        Piece<T, kV> v;
        v.load(sb + i * kV);
        float f[kV];
        v.unpack(f);
#pragma unroll
        for (int e = 0; e < kV; ++e) f[e] *= coef;
        v.pack(f);
        v.store_stream(db + i * kV);
    }
    const int rest = len - nvec * kV;
    for (int k = threadIdx.x; k < rest; k += kGradThreads) {
        const int j = k < head ? k : k + nvec * kV;
        dst[j] = elem_from_float<T>(elem_to_float(src[j]) * coef);
    }
}

// partials != NULL: the norm is joined here, by every CTA for itself (and written by the first
// one); else it is read from `norm`.
template <int CAP, int U>
__global__ void __launch_bounds__(kGradThreads)
grad_scale_kernel(const __grid_constant__ GradList<CAP> l, const double *partials, int nparts, float *norm,
                  float max_norm, float eps)
{
    __shared__ double warp_part[kGradThreads / 32];
    grid_launch_dependents();
    grid_dependency_wait();
    float v;
    if (partials) {
        v = join_norm(partials, nparts, warp_part);
        if (blockIdx.x == 0 && threadIdx.x == 0) *norm = v;
    } else {
        v = *norm;
    }
    // (not min(1, quotient): 0 / 0 of zero gradients and inf / inf without a limit are 1; a NaN norm stays one)
    const float coef = max_norm >= v + eps ? 1.f : max_norm / (v + eps);
    const unsigned total = l.first[l.count];
    for (unsigned b = blockIdx.x; b < total; b += gridDim.x) {
        const unsigned c = total - 1 - b;
        const GradChunk g = grad_chunk(l, c);
        void *src = l.data[g.tensor], *dst = l.out[g.tensor];
        if (coef == 1.f && src == dst) continue;
        if (l.dtype[g.tensor] == 0)
            chunk_scale<U>(static_cast<const float *>(src) + g.begin, static_cast<float *>(dst) + g.begin, g.len, coef);
        else if (l.dtype[g.tensor] == 1)
            chunk_scale<U>(static_cast<const __nv_bfloat16 *>(src) + g.begin, static_cast<__nv_bfloat16 *>(dst) + g.begin, g.len, coef);
        else
            chunk_scale<U>(static_cast<const __half *>(src) + g.begin, static_cast<__half *>(dst) + g.begin, g.len, coef);
    }
}

}  // namespace cudallm
