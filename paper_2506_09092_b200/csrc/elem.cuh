// Element types of the row and list operators: 16-byte pieces of fp32, bf16 or fp16
// values, widened to fp32 and rounded back to nearest even.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "ptx.cuh"

namespace cudallm {

// Two fp32 values in one register pair: packed arithmetic issues half the instructions.
__device__ __forceinline__ uint64_t f32x2(float lo, float hi)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
    return v;
}
__device__ __forceinline__ void f32x2_split(uint64_t v, float &lo, float &hi)
{
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t f32x2_fma(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t f32x2_add(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t f32x2_mul(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t f32x2_both(float v) { return f32x2(v, v); }
__device__ __forceinline__ float f32x2_sum(uint64_t v)
{
    float lo, hi;
    f32x2_split(v, lo, hi);
    return lo + hi;
}

__device__ __forceinline__ float elem_to_float(float v) { return v; }
__device__ __forceinline__ float elem_to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float elem_to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T elem_from_float(float v);
template <> __device__ __forceinline__ float elem_from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 elem_from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half elem_from_float<__half>(float v) { return __float2half_rn(v); }

template <typename T> struct ElemVec { static constexpr int kN = 16 / sizeof(T); };   // elements of a 16-byte piece

// VEC consecutive elements as they lie in memory: one 16-byte access, or one element.
template <typename T, int VEC> struct Piece;
template <typename T> struct Piece<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T *p) { v = *p; }
    __device__ __forceinline__ void clear() { v = elem_from_float<T>(0.f); }
    __device__ __forceinline__ void unpack(float (&f)[1]) const { f[0] = elem_to_float(v); }
    __device__ __forceinline__ void pack(const float (&f)[1]) { v = elem_from_float<T>(f[0]); }
    __device__ __forceinline__ void store(T *p) const { *p = v; }
    __device__ __forceinline__ void store_stream(T *p) const { *p = v; }
};
template <typename T> struct PieceBits {
    uint4 v;
    __device__ __forceinline__ void load(const T *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void clear() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<uint4 *>(p) = v; }
    __device__ __forceinline__ void store_stream(T *p) const { __stcs(reinterpret_cast<uint4 *>(p), v); }
};
template <> struct Piece<float, 4> : PieceBits<float> {
    __device__ __forceinline__ void unpack(float (&f)[4]) const
    {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y);
        f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    __device__ __forceinline__ void pack(const float (&f)[4])
    {
        v = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};
template <> struct Piece<__nv_bfloat16, 8> : PieceBits<__nv_bfloat16> {
    __device__ __forceinline__ void unpack(float (&f)[8]) const
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    __device__ __forceinline__ void pack(const float (&f)[8])
    {
        v = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
    }
};
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <> struct Piece<__half, 8> : PieceBits<__half> {
    __device__ __forceinline__ void unpack(float (&f)[8]) const
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            f[2 * i] = p.x;
            f[2 * i + 1] = p.y;
        }
    }
    __device__ __forceinline__ void pack(const float (&f)[8])
    {
        v = make_uint4(pack_f16x2(f[0], f[1]), pack_f16x2(f[2], f[3]), pack_f16x2(f[4], f[5]), pack_f16x2(f[6], f[7]));
    }
};

// Element i of an array of fp32 (code 0), bf16 (1) or fp16 (2) values.
__device__ __forceinline__ float load_as_float(const void *p, int dtype, long long i)
{
    if (dtype == 0) return static_cast<const float *>(p)[i];
    if (dtype == 1) return elem_to_float(static_cast<const __nv_bfloat16 *>(p)[i]);
    return elem_to_float(static_cast<const __half *>(p)[i]);
}
__device__ __forceinline__ void store_from_float(void *p, int dtype, long long i, float v)
{
    if (dtype == 0) static_cast<float *>(p)[i] = v;
    else if (dtype == 1) static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
    else static_cast<__half *>(p)[i] = __float2half_rn(v);
}

}  // namespace cudallm
