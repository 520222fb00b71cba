// LayerNorm over the rows of a matrix, forward and backward.
//
//   forward   mean, rstd = 1 / sqrt(var + eps),  y = (x - mean) rstd gamma + beta
//   backward  xhat = (x - mean) rstd,  g = dy gamma,
//             dx = rstd (g - mean(g) - xhat mean(g xhat)),
//             dgamma = sum_rows dy xhat,  dbeta = sum_rows dy
//
// Bound: HBM (x read once, y written once; dy, x read and dx written once).  A row stays in
// registers, as it came from memory, between its statistics and its normalisation, so nothing is
// read twice.  The CTAs are persistent: gamma and beta are read once per CTA (per row they would
// cost more L2 traffic than the row itself), dgamma and dbeta are summed in registers.  At 16 bits
// a value the instructions per value come next to the memory's rate, hence arithmetic on pairs, and
// R rows at a time, whose sums share their shuffles and barriers.
//
// Up to 1024 columns a row belongs to a warp or a part of one: no barrier.  Longer rows, and rows too
// few to occupy the warps, are a CTA's.
//
// Measured (one B200; bytes read and written once): 16384 x 4096 bf16 forward 48.4 us = 5.5 TB/s (0.85 of the
// measured copy bandwidth), backward 82.2 us = 4.9 TB/s; the same in fp32 97 us = 5.6 and 132 us =
// 6.1 TB/s; 262144 x 256 bf16 forward 48.3 us = 5.6 TB/s; 2999 x 1537 fp32 (no 16-byte rows) 9.7 and
// 19.4 us.  What is left is issue slots (55 and 63 % of them at 4096 bf16) and the two barriers of a row.  Longer rows are
// slower: 4096 x 12288 bf16 backward 130 us = 2.3 TB/s (64 registers a thread, some spilled), with 12289 columns 262 forward and
// 416 us backward; 2048 x 32768 fp32, read again for every pass, 160 us = 3.4 and 428 us = 1.9 TB/s.
#pragma once
#include "elem.cuh"

namespace cudallm {

struct LnRowsParams {
    const void *x, *dy, *gamma, *beta;
    void *y;                       // forward: y; backward: dx (or NULL)
    float *mean, *rstd;
    float *partials;               // backward: [gridDim.x][2][n] column sums (or NULL)
    long long ldx, lddy, ldy;
    int rows, n, param_dtype;
    float eps, inv_n;
};

// First half of a sum of NV values (a power of two) over the lanes of groups of TPR: the lanes halve the
// values they carry per shuffle (9 shuffles for eight values on 32 lanes instead of 40), until
// lane i of a group holds v[0], the total of value i / (TPR / NV).
template <int TPR, int NV>
__device__ __forceinline__ void lanes_fold(float (&v)[NV])
{
    static_assert((NV & (NV - 1)) == 0 && NV <= TPR, "values");
    const int lane = threadIdx.x;
    int offset = TPR / 2;
#pragma unroll
    for (int m = NV / 2; m; m >>= 1, offset >>= 1) {
        const bool up = (lane & offset) != 0;
#pragma unroll
        for (int k = 0; k < m; ++k) {
            const float other = __shfl_xor_sync(0xffffffffu, up ? v[k] : v[k + m], offset);
            v[k] = (up ? v[k + m] : v[k]) + other;
        }
    }
#pragma unroll
    for (; offset; offset >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], offset);
}

// Sums of NV values over the TPR <= 32 neighbouring lanes that share a row, given to all of them.
template <int TPR, int NV>
__device__ __forceinline__ void lanes_sum(float (&v)[NV])
{
    if (NV == 1) {
#pragma unroll
        for (int o = TPR / 2; o; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
        return;
    }
    lanes_fold<TPR, NV>(v);
    const float s = v[0];
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] = __shfl_sync(0xffffffffu, s, k * (TPR / NV), TPR);
}

// The same over a CTA of TPR > 32 threads.  `xch` is used alternately (`flip`), so one barrier is enough.
template <int TPR, int NV>
__device__ __forceinline__ void block_sum(float (&v)[NV], float (*xch)[32][NV], int &flip)
{
    constexpr int kWarps = TPR / 32, kShare = 32 / NV;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    lanes_fold<32, NV>(v);
    const int mine = lane / kShare, at = lane % kShare;
    if (at == 0) xch[flip][warp][mine] = v[0];
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < (kWarps + kShare - 1) / kShare; ++w)
        if (at + w * kShare < kWarps) s += xch[flip][at + w * kShare][mine];
#pragma unroll
    for (int o = kShare / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] = __shfl_sync(0xffffffffu, s, k * kShare);
    flip ^= 1;
}

// gamma and beta (or gamma alone) of all columns in shared memory as fp32, in planes of four: element
// e of piece i lies at plane e / 4, so that neighbouring lanes' 16-byte reads hit distinct banks.
template <int VEC>
__device__ __forceinline__ void stage_params(float *dst, const void *src, const LnRowsParams &p, float absent)
{
    for (int c = threadIdx.x; c < p.n; c += blockDim.x) {
        const float v = src ? load_as_float(src, p.param_dtype, c) : absent;
        if (VEC == 1) dst[c] = v;
        else dst[((c % VEC) / 4 * (p.n / VEC) + c / VEC) * 4 + c % 4] = v;
    }
}
// What a thread holds of a row is a number of units: 16 bytes of VEC neighbouring values or, where rows do
// not consist of such pieces (VEC == 1), two single values TPR columns apart; their arithmetic is on
// pairs either way.  Unit v of lane t starts at column unit_column(v, t).
template <int VEC> constexpr int kUnit = VEC > 1 ? VEC : 2;
template <int VEC> constexpr int kPairs = kUnit<VEC> / 2;
template <int VEC, int TPR>
__device__ __forceinline__ int unit_column(int v, int t) { return VEC > 1 ? (v * TPR + t) * VEC : 2 * v * TPR + t; }

template <typename T, int VEC, int TPR> struct Unit {
    Piece<T, VEC> q;
    __device__ __forceinline__ void clear() { q.clear(); }
    __device__ __forceinline__ void load(const T *row, int c, int) { q.load(row + c); }
    __device__ __forceinline__ void pairs(uint64_t (&f)[kPairs<VEC>]) const
    {
        float v[VEC];
        q.unpack(v);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) f[i] = f32x2(v[2 * i], v[2 * i + 1]);
    }
    static __device__ __forceinline__ void store(T *row, int c, int, const uint64_t (&f)[kPairs<VEC>])
    {
        float v[VEC];
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) f32x2_split(f[i], v[2 * i], v[2 * i + 1]);
        Piece<T, VEC> out;
        out.pack(v);
        out.store(row + c);
    }
};
template <typename T, int TPR> struct Unit<T, 1, TPR> {
    T a, b;
    __device__ __forceinline__ void clear() { a = b = elem_from_float<T>(0.f); }
    __device__ __forceinline__ void load(const T *row, int c, int n)
    {
        a = row[c];
        if (c + TPR < n) b = row[c + TPR];
    }
    __device__ __forceinline__ void pairs(uint64_t (&f)[1]) const { f[0] = f32x2(elem_to_float(a), elem_to_float(b)); }
    static __device__ __forceinline__ void store(T *row, int c, int n, const uint64_t (&f)[1])
    {
        float lo, hi;
        f32x2_split(f[0], lo, hi);
        row[c] = elem_from_float<T>(lo);
        if (c + TPR < n) row[c + TPR] = elem_from_float<T>(hi);
    }
};

// gamma or beta of the unit at column c, as fp32: staged in shared memory, or from memory.
template <int VEC, int TPR>
__device__ __forceinline__ void read_params(const float *src, int n, int c, uint64_t (&o)[kPairs<VEC>])
{
    if constexpr (VEC == 1) {
        o[0] = f32x2(src[c], c + TPR < n ? src[c + TPR] : 0.f);
    } else {
#pragma unroll
        for (int h = 0; h < VEC / 4; ++h) {
            const float4 f = reinterpret_cast<const float4 *>(src)[h * (n / VEC) + c / VEC];
            o[2 * h] = f32x2(f.x, f.y);
            o[2 * h + 1] = f32x2(f.z, f.w);
        }
    }
}
template <int VEC, int TPR>
__device__ __forceinline__ void load_params(const void *src, const LnRowsParams &p, int c, float absent, uint64_t (&o)[kPairs<VEC>])
{
    float v[kUnit<VEC>];
#pragma unroll
    for (int e = 0; e < kUnit<VEC>; ++e) {
        const int at = VEC == 1 ? c + e * TPR : c + e;
        v[e] = (src && at < p.n) ? load_as_float(src, p.param_dtype, at) : absent;
    }
#pragma unroll
    for (int i = 0; i < kPairs<VEC>; ++i) o[i] = f32x2(v[2 * i], v[2 * i + 1]);
}

// The statistics of a row by one pass for a first mean and one for the differences to it, whose own mean
// corrects the first: a mean far above the spread is off by its fp32 rounding, the differences are not.
struct LnStats { float mean0, shift, rstd; };
__device__ __forceinline__ LnStats ln_stats(float mean0, float sum_d, float sum_dd, const LnRowsParams &p)
{
    LnStats s;
    s.mean0 = mean0;
    s.shift = sum_d * p.inv_n;
    const float var = fmaxf(fmaf(-s.shift, s.shift, sum_dd * p.inv_n), 0.f);
    // (fmaxf drops a NaN: a row that holds one keeps it in the sum, which is tested here)
    s.rstd = sum_dd == sum_dd ? 1.f / sqrtf(var + p.eps) : sum_dd;
    return s;
}

// What a unit adds to its row's sum; to the sums of its differences to mean0 and of their squares.
template <typename T, int VEC, int TPR>
__device__ __forceinline__ void add_sum(const Unit<T, VEC, TPR> &q, uint64_t &acc)
{
    uint64_t f[kPairs<VEC>];
    q.pairs(f);
#pragma unroll
    for (int i = 0; i < kPairs<VEC>; ++i) acc = f32x2_add(acc, f[i]);
}
template <typename T, int VEC, int TPR>
__device__ __forceinline__ void add_differences(const Unit<T, VEC, TPR> &q, int c, int n, float mean0, uint64_t &d, uint64_t &dd)
{
    const uint64_t minus = f32x2(-mean0, VEC > 1 || c + TPR < n ? -mean0 : 0.f);   // (a value that does not exist is 0 - 0)
    uint64_t f[kPairs<VEC>];
    q.pairs(f);
#pragma unroll
    for (int i = 0; i < kPairs<VEC>; ++i) {
        const uint64_t t = f32x2_add(f[i], minus);
        d = f32x2_add(d, t);
        dd = f32x2_fma(t, t, dd);
    }
}
template <typename T, int VEC, int TPR>
__device__ __forceinline__ void store_normalised(T *row, int c, int n, const Unit<T, VEC, TPR> &q, const LnStats &st,
                                                 const uint64_t (&g)[kPairs<VEC>], const uint64_t (&b)[kPairs<VEC>])
{
    const uint64_t minus = f32x2_both(-st.mean0), shift = f32x2_both(-st.shift), rstd = f32x2_both(st.rstd);
    uint64_t f[kPairs<VEC>];
    q.pairs(f);
#pragma unroll
    for (int i = 0; i < kPairs<VEC>; ++i)
        f[i] = f32x2_fma(f32x2_mul(f32x2_add(f32x2_add(f[i], minus), shift), rstd), g[i], b[i]);
    Unit<T, VEC, TPR>::store(row, c, n, f);
}
// Backward: a unit's part of the column sums and of the row's sums of g and g xhat (dy is zero where nothing
// is); its part of dx.
template <typename T, int VEC, int TPR>
__device__ __forceinline__ void add_gradients(const Unit<T, VEC, TPR> &qx, const Unit<T, VEC, TPR> &qy, float mean, float rstd,
                                              const uint64_t (&gamma)[kPairs<VEC>], uint64_t (&dg)[kPairs<VEC>],
                                              uint64_t (&db)[kPairs<VEC>], uint64_t &s0, uint64_t &s1)
{
    const uint64_t minus = f32x2_both(-mean), r = f32x2_both(rstd);
    uint64_t f[kPairs<VEC>], d[kPairs<VEC>];
    qx.pairs(f);
    qy.pairs(d);
#pragma unroll
    for (int i = 0; i < kPairs<VEC>; ++i) {
        const uint64_t xh = f32x2_mul(f32x2_add(f[i], minus), r), g = f32x2_mul(d[i], gamma[i]);
        dg[i] = f32x2_fma(d[i], xh, dg[i]);
        db[i] = f32x2_add(db[i], d[i]);
        s0 = f32x2_add(s0, g);
        s1 = f32x2_fma(g, xh, s1);
    }
}
template <typename T, int VEC, int TPR>
__device__ __forceinline__ void store_gradient(T *row, int c, int n, const Unit<T, VEC, TPR> &qx, const Unit<T, VEC, TPR> &qy,
                                               float mean, float rstd, float c1, float c2, const uint64_t (&gamma)[kPairs<VEC>])
{
    const uint64_t minus = f32x2_both(-mean), r = f32x2_both(rstd), m1 = f32x2_both(-c1), m2 = f32x2_both(-c2);
    uint64_t f[kPairs<VEC>], d[kPairs<VEC>];
    qx.pairs(f);
    qy.pairs(d);
#pragma unroll
    for (int i = 0; i < kPairs<VEC>; ++i) {
        const uint64_t xh = f32x2_mul(f32x2_add(f[i], minus), r);
        f[i] = f32x2_mul(f32x2_fma(d[i], gamma[i], f32x2_fma(xh, m2, m1)), r);
    }
    Unit<T, VEC, TPR>::store(row, c, n, f);
}
// Column sums of the unit at column c, to fp32 rows.
template <int VEC, int TPR>
__device__ __forceinline__ void put_sums(float *dst, int c, int n, const uint64_t (&f)[kPairs<VEC>])
{
#pragma unroll
    for (int i = 0; i < kPairs<VEC>; ++i) {
        float lo, hi;
        f32x2_split(f[i], lo, hi);
        dst[c + 2 * i] = lo;
        if (VEC > 1) dst[c + 2 * i + 1] = hi;
        else if (c + TPR < n) dst[c + TPR] = hi;
    }
}

constexpr int kLnWarpThreads = 256;

// Forward, rows of up to TPR * VPT units on TPR <= 32 lanes, R rows of the lanes at a time.  n is a multiple
// of VEC.
template <typename T, int VEC, int TPR, int VPT, int R>
__global__ void __launch_bounds__(kLnWarpThreads, 2)
layernorm_warp_kernel(const LnRowsParams p)
{
    extern __shared__ __align__(16) float ln_params[];
    constexpr int kRows = kLnWarpThreads / TPR;                    // rows of a CTA, R times
    const int t = threadIdx.x % TPR;
    float *gamma_s = ln_params, *beta_s = ln_params + p.n;
    const T *x = static_cast<const T *>(p.x);
    T *y = static_cast<T *>(p.y);
    grid_launch_dependents();
    grid_dependency_wait();
    stage_params<VEC>(gamma_s, p.gamma, p, 1.f);
    stage_params<VEC>(beta_s, p.beta, p, 0.f);
    __syncthreads();
    for (long long base = (long long)blockIdx.x * kRows * R; base < p.rows; base += (long long)gridDim.x * kRows * R) {
        const long long row = base + threadIdx.x / TPR;            // and row + kRows, ...
        Unit<T, VEC, TPR> q[R][VPT];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                q[r][v].clear();
                const int c = unit_column<VEC, TPR>(v, t);
                if (row + r * kRows < p.rows && c < p.n) q[r][v].load(x + (row + r * kRows) * p.ldx, c, p.n);
            }
        float s[R], d[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            uint64_t acc[2] = {0, 0};
#pragma unroll
            for (int v = 0; v < VPT; ++v) add_sum(q[r][v], acc[v & 1]);      // (zeros where there is nothing)
            s[r] = f32x2_sum(f32x2_add(acc[0], acc[1]));
        }
        lanes_sum<TPR, R>(s);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            s[r] *= p.inv_n;
            uint64_t d0[2] = {0, 0}, d1[2] = {0, 0};
#pragma unroll
            for (int v = 0; v < VPT; ++v)
                if (unit_column<VEC, TPR>(v, t) < p.n)
                    add_differences(q[r][v], unit_column<VEC, TPR>(v, t), p.n, s[r], d0[v & 1], d1[v & 1]);
            d[2 * r] = f32x2_sum(f32x2_add(d0[0], d0[1]));
            d[2 * r + 1] = f32x2_sum(f32x2_add(d1[0], d1[1]));
        }
        lanes_sum<TPR, 2 * R>(d);
        LnStats st[R];
#pragma unroll
        for (int r = 0; r < R; ++r) st[r] = ln_stats(s[r], d[2 * r], d[2 * r + 1], p);
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int c = unit_column<VEC, TPR>(v, t);
            if (c < p.n) {
                uint64_t g[kPairs<VEC>], b[kPairs<VEC>];
                read_params<VEC, TPR>(gamma_s, p.n, c, g);
                read_params<VEC, TPR>(beta_s, p.n, c, b);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (row + r * kRows < p.rows) store_normalised(y + (row + r * kRows) * p.ldy, c, p.n, q[r][v], st[r], g, b);
            }
        }
        if (t == 0)
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (row + r * kRows < p.rows) {
                    if (p.mean) p.mean[row + r * kRows] = st[r].mean0 + st[r].shift;
                    if (p.rstd) p.rstd[row + r * kRows] = st[r].rstd;
                }
    }
}

// Rows that a CTA of TPR threads works on, R at a time, on their way into shared memory slots that only
// one thread writes and reads each (cp.async, so no barrier for them): `arrays` of them (x; x and dy), two
// rounds of R rows.  Of rows that are not whole 16-byte pieces the next round is held in registers.
__device__ __forceinline__ void ln_copy_16(uint32_t smem_addr, const void *gptr)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr), "l"(gptr) : "memory");
}
template <typename T, int VEC, int TPR, int VPT, int R, int ARRAYS>
struct LnSlots {
    uint32_t base;
    Unit<T, VEC, TPR> held[VEC == 1 ? R : 1][VEC == 1 ? ARRAYS : 1][VEC == 1 ? VPT : 1];
    __device__ __forceinline__ uint32_t at(int parity, int r, int a, int v) const
    {
        return base + (((parity * R + r) * ARRAYS + a) * VPT + v) * (TPR * 16);
    }
    // rows row, row + grid, ... of array a
    __device__ __forceinline__ void fetch(const T *src, long long ld, long long row, int a, int parity, const LnRowsParams &p)
    {
#pragma unroll
        for (int r = 0; r < R; ++r, row += gridDim.x)
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                const int c = unit_column<VEC, TPR>(v, threadIdx.x);
                if (row < p.rows && c < p.n) {
                    if constexpr (VEC > 1) ln_copy_16(at(parity, r, a, v), src + row * ld + c);
                    else held[r][a][v].load(src + row * ld, c, p.n);
                }
            }
    }
    __device__ __forceinline__ void commit() const { if (VEC > 1) asm volatile("cp.async.commit_group;" ::: "memory"); }
    __device__ __forceinline__ void wait() const { if (VEC > 1) asm volatile("cp.async.wait_group 1;" ::: "memory"); }
    __device__ __forceinline__ void read(long long row, int r, int a, int parity, int v, const LnRowsParams &p,
                                         Unit<T, VEC, TPR> &q) const
    {
        const int c = unit_column<VEC, TPR>(v, threadIdx.x);
        q.clear();
        if (row < p.rows && c < p.n) {
            if constexpr (VEC > 1)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(q.q.v.x), "=r"(q.q.v.y), "=r"(q.q.v.z), "=r"(q.q.v.w) : "r"(at(parity, r, a, v)) : "memory");
            else {
                q.a = held[r][a][v].a;
                if (c + TPR < p.n) q.b = held[r][a][v].b;
            }
        }
    }
};
__host__ __device__ constexpr int ln_slot_bytes(int vec, int tpr, int vpt, int r, int arrays)
{
    return vec == 1 ? 0 : 2 * r * arrays * vpt * tpr * 16;
}

// Forward, a CTA of TPR threads per row.
template <typename T, int VEC, int TPR, int VPT, int R>
__global__ void __launch_bounds__(TPR, 512 / TPR)
layernorm_block_kernel(const LnRowsParams p)
{
    __shared__ float xch1[2][32][R];
    __shared__ float xch2[2][32][2 * R];
    extern __shared__ __align__(16) uint8_t ln_bytes[];
    const int t = threadIdx.x;
    LnSlots<T, VEC, TPR, VPT, R, 1> slots;
    slots.base = smem_u32(ln_bytes) + t * 16;
    const T *x = static_cast<const T *>(p.x);
    T *y = static_cast<T *>(p.y);
    grid_launch_dependents();
    grid_dependency_wait();
    slots.fetch(x, p.ldx, blockIdx.x, 0, 0, p);
    slots.commit();
    uint64_t gamma[VPT][kPairs<VEC>], beta[VPT][kPairs<VEC>];
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        load_params<VEC, TPR>(p.gamma, p, unit_column<VEC, TPR>(v, t), 1.f, gamma[v]);
        load_params<VEC, TPR>(p.beta, p, unit_column<VEC, TPR>(v, t), 0.f, beta[v]);
    }
    int flip1 = 0, flip2 = 0, parity = 0;
    for (long long row = blockIdx.x; row < p.rows; row += (long long)R * gridDim.x, parity ^= 1) {
        if (VEC > 1) slots.fetch(x, p.ldx, row + (long long)R * gridDim.x, 0, parity ^ 1, p);
        slots.commit();
        slots.wait();
        Unit<T, VEC, TPR> q[R][VPT];
        float s[R], d[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            uint64_t acc = 0;
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                slots.read(row + (long long)r * gridDim.x, r, 0, parity, v, p, q[r][v]);
                add_sum(q[r][v], acc);                             // (zeros where there is nothing)
            }
            s[r] = f32x2_sum(acc);
        }
        if (VEC == 1) slots.fetch(x, p.ldx, row + (long long)R * gridDim.x, 0, 0, p);
        block_sum<TPR, R>(s, xch1, flip1);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            s[r] *= p.inv_n;
            uint64_t d0 = 0, d1 = 0;
#pragma unroll
            for (int v = 0; v < VPT; ++v)
                if (unit_column<VEC, TPR>(v, t) < p.n)
                    add_differences(q[r][v], unit_column<VEC, TPR>(v, t), p.n, s[r], d0, d1);
            d[2 * r] = f32x2_sum(d0);
            d[2 * r + 1] = f32x2_sum(d1);
        }
        block_sum<TPR, 2 * R>(d, xch2, flip2);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long at = row + (long long)r * gridDim.x;
            if (at >= p.rows) break;
            const LnStats st = ln_stats(s[r], d[2 * r], d[2 * r + 1], p);
#pragma unroll
            for (int v = 0; v < VPT; ++v)
                if (unit_column<VEC, TPR>(v, t) < p.n)
                    store_normalised(y + at * p.ldy, unit_column<VEC, TPR>(v, t), p.n, q[r][v], st, gamma[v], beta[v]);
            if (t == 0) {
                if (p.mean) p.mean[at] = st.mean0 + st.shift;
                if (p.rstd) p.rstd[at] = st.rstd;
            }
        }
    }
}

// Backward, rows on TPR <= 32 lanes.  The column sums of a lane's columns stay in its registers over
// all rows that it visits and join over the CTA's rows in shared memory, in order, at the end.
template <typename T, int VEC, int TPR, int VPT, int R>
__global__ void __launch_bounds__(kLnWarpThreads, 2)
layernorm_warp_bwd_kernel(const LnRowsParams p)
{
    extern __shared__ __align__(16) float ln_params[];             // gamma, later the join: [kRows][n]
    constexpr int kRows = kLnWarpThreads / TPR;
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const T *x = static_cast<const T *>(p.x);
    const T *dy = static_cast<const T *>(p.dy);
    T *dx = static_cast<T *>(p.y);
    grid_launch_dependents();
    grid_dependency_wait();
    stage_params<VEC>(ln_params, p.gamma, p, 1.f);
    __syncthreads();
    uint64_t dg[VPT][kPairs<VEC>] = {}, db[VPT][kPairs<VEC>] = {};
    for (long long base = (long long)blockIdx.x * kRows * R; base < p.rows; base += (long long)gridDim.x * kRows * R) {
        const long long row = base + sub;                          // and row + kRows, ...
        Unit<T, VEC, TPR> qx[R][VPT], qy[R][VPT];
        float mean[R], rstd[R], s[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool live_row = row + r * kRows < p.rows;
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                qx[r][v].clear();
                qy[r][v].clear();
                const int c = unit_column<VEC, TPR>(v, t);
                if (live_row && c < p.n) {
                    qx[r][v].load(x + (row + r * kRows) * p.ldx, c, p.n);
                    qy[r][v].load(dy + (row + r * kRows) * p.lddy, c, p.n);
                }
            }
            mean[r] = live_row ? p.mean[row + r * kRows] : 0.f;
            rstd[r] = live_row ? p.rstd[row + r * kRows] : 0.f;
        }
        uint64_t s0[R] = {}, s1[R] = {};
#pragma unroll
        for (int v = 0; v < VPT; ++v)
            if (unit_column<VEC, TPR>(v, t) < p.n) {
                uint64_t g[kPairs<VEC>];
                read_params<VEC, TPR>(ln_params, p.n, unit_column<VEC, TPR>(v, t), g);
#pragma unroll
                for (int r = 0; r < R; ++r) add_gradients(qx[r][v], qy[r][v], mean[r], rstd[r], g, dg[v], db[v], s0[r], s1[r]);
            }
        if (!dx) continue;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            s[2 * r] = f32x2_sum(s0[r]);
            s[2 * r + 1] = f32x2_sum(s1[r]);
        }
        lanes_sum<TPR, 2 * R>(s);
#pragma unroll
        for (int v = 0; v < VPT; ++v)
            if (unit_column<VEC, TPR>(v, t) < p.n) {
                uint64_t g[kPairs<VEC>];
                read_params<VEC, TPR>(ln_params, p.n, unit_column<VEC, TPR>(v, t), g);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (row + r * kRows < p.rows)
                        store_gradient(dx + (row + r * kRows) * p.ldy, unit_column<VEC, TPR>(v, t), p.n, qx[r][v], qy[r][v],
                                       mean[r], rstd[r], s[2 * r] * p.inv_n, s[2 * r + 1] * p.inv_n, g);
            }
    }
    if (!p.partials) return;
    float *out = p.partials + (long long)blockIdx.x * 2 * p.n;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < VPT; ++v)
            if (unit_column<VEC, TPR>(v, t) < p.n)
                put_sums<VEC, TPR>(ln_params + sub * p.n, unit_column<VEC, TPR>(v, t), p.n, k ? db[v] : dg[v]);
        __syncthreads();
        for (int c = threadIdx.x; c < p.n; c += kLnWarpThreads) {
            float a = 0.f;
            for (int r = 0; r < kRows; ++r) a += ln_params[r * p.n + c];
            out[(long long)k * p.n + c] = a;
        }
    }
}

// Backward, a CTA of TPR threads per row.
template <typename T, int VEC, int TPR, int VPT, int R>
__global__ void __launch_bounds__(TPR, TPR > 512 ? 1 : 512 / TPR)
layernorm_block_bwd_kernel(const LnRowsParams p)
{
    __shared__ float xch[2][32][2 * R];
    extern __shared__ __align__(16) uint8_t ln_bytes[];
    const int t = threadIdx.x;
    LnSlots<T, VEC, TPR, VPT, R, 2> slots;
    slots.base = smem_u32(ln_bytes) + t * 16;
    const T *x = static_cast<const T *>(p.x);
    const T *dy = static_cast<const T *>(p.dy);
    T *dx = static_cast<T *>(p.y);
    grid_launch_dependents();
    grid_dependency_wait();
    slots.fetch(x, p.ldx, blockIdx.x, 0, 0, p);
    slots.fetch(dy, p.lddy, blockIdx.x, 1, 0, p);
    slots.commit();
    uint64_t gamma[VPT][kPairs<VEC>], dg[VPT][kPairs<VEC>] = {}, db[VPT][kPairs<VEC>] = {};
#pragma unroll
    for (int v = 0; v < VPT; ++v) load_params<VEC, TPR>(p.gamma, p, unit_column<VEC, TPR>(v, t), 1.f, gamma[v]);
    float next_mean[R], next_rstd[R];
    auto fetch_stats = [&](long long row) {
#pragma unroll
        for (int r = 0; r < R; ++r, row += gridDim.x) {
            next_mean[r] = row < p.rows ? p.mean[row] : 0.f;
            next_rstd[r] = row < p.rows ? p.rstd[row] : 0.f;
        }
    };
    fetch_stats(blockIdx.x);
    int flip = 0, parity = 0;
    for (long long row = blockIdx.x; row < p.rows; row += (long long)R * gridDim.x, parity ^= 1) {
        const long long next = row + (long long)R * gridDim.x;
        if (VEC > 1) {
            slots.fetch(x, p.ldx, next, 0, parity ^ 1, p);
            slots.fetch(dy, p.lddy, next, 1, parity ^ 1, p);
        }
        slots.commit();
        float mean[R], rstd[R], s[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean[r] = next_mean[r];
            rstd[r] = next_rstd[r];
        }
        fetch_stats(next);
        slots.wait();
        Unit<T, VEC, TPR> qx[R][VPT], qy[R][VPT];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long at = row + (long long)r * gridDim.x;
            uint64_t s0 = 0, s1 = 0;
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                slots.read(at, r, 0, parity, v, p, qx[r][v]);
                slots.read(at, r, 1, parity, v, p, qy[r][v]);
                if (unit_column<VEC, TPR>(v, t) < p.n)
                    add_gradients(qx[r][v], qy[r][v], mean[r], rstd[r], gamma[v], dg[v], db[v], s0, s1);
            }
            s[2 * r] = f32x2_sum(s0);
            s[2 * r + 1] = f32x2_sum(s1);
        }
        if (VEC == 1) {
            slots.fetch(x, p.ldx, next, 0, 0, p);
            slots.fetch(dy, p.lddy, next, 1, 0, p);
        }
        if (!dx) continue;
        block_sum<TPR, 2 * R>(s, xch, flip);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long at = row + (long long)r * gridDim.x;
            if (at >= p.rows) break;
#pragma unroll
            for (int v = 0; v < VPT; ++v)
                if (unit_column<VEC, TPR>(v, t) < p.n)
                    store_gradient(dx + at * p.ldy, unit_column<VEC, TPR>(v, t), p.n, qx[r][v], qy[r][v], mean[r], rstd[r],
                                   s[2 * r] * p.inv_n, s[2 * r + 1] * p.inv_n, gamma[v]);
        }
    }
    if (!p.partials) return;
    float *out = p.partials + (long long)blockIdx.x * 2 * p.n;
#pragma unroll
    for (int v = 0; v < VPT; ++v)
        if (unit_column<VEC, TPR>(v, t) < p.n) {
            put_sums<VEC, TPR>(out, unit_column<VEC, TPR>(v, t), p.n, dg[v]);
            put_sums<VEC, TPR>(out + p.n, unit_column<VEC, TPR>(v, t), p.n, db[v]);
        }
}

// dgamma, dbeta = the sum of `parts` partial rows.  A CTA of 1024 threads takes 32 columns of
// one of the two: 32 groups of threads each add every 32nd part, then the groups' sums are added
// in order.
struct LnJoinParams {
    const float *partials;
    void *dgamma, *dbeta;
    int n, parts, param_dtype;
};
__global__ void __launch_bounds__(1024)
layernorm_join_kernel(const LnJoinParams p)
{
    __shared__ float s[32][33];
    grid_launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    void *dst = blockIdx.y ? p.dbeta : p.dgamma;
    if (!dst) return;
    const float *src = p.partials + (long long)blockIdx.y * p.n + c;
    const long long step = 2ll * p.n;
    float a[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < p.n) {
        int i = grp;
        for (; i + 96 < p.parts; i += 128)
#pragma unroll
            for (int u = 0; u < 4; ++u) a[u] += src[(i + 32 * u) * step];
        for (; i < p.parts; i += 32) a[0] += src[i * step];
    }
    s[grp][lane] = (a[0] + a[1]) + (a[2] + a[3]);
    __syncthreads();
    // warp w finishes column w of the CTA
    float sum = s[lane][grp];
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const int col = blockIdx.x * 32 + grp;
    if (lane == 0 && col < p.n) store_from_float(dst, p.param_dtype, col, sum);
}

// Rows too long for registers: one CTA of 1024 threads per row, several passes over the row
// (which stays in L2 between them).
constexpr int kLnLongThreads = 1024;

template <typename T>
__global__ void __launch_bounds__(kLnLongThreads)
layernorm_long_kernel(const LnRowsParams p)
{
    __shared__ float xch1[2][32][1];
    __shared__ float xch2[2][32][2];
    grid_launch_dependents();
    grid_dependency_wait();
    int flip1 = 0, flip2 = 0;
    for (int row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(p.x) + row * p.ldx;
        T *y = static_cast<T *>(p.y) + row * p.ldy;
        float s[1] = {0.f};
        for (int c = threadIdx.x; c < p.n; c += kLnLongThreads) s[0] += elem_to_float(x[c]);
        block_sum<kLnLongThreads, 1>(s, xch1, flip1);
        const float mean0 = s[0] * p.inv_n;
        float d[2] = {0.f, 0.f};
        for (int c = threadIdx.x; c < p.n; c += kLnLongThreads) {
            const float f = elem_to_float(x[c]) - mean0;
            d[0] += f;
            d[1] = fmaf(f, f, d[1]);
        }
        block_sum<kLnLongThreads, 2>(d, xch2, flip2);
        const LnStats st = ln_stats(mean0, d[0], d[1], p);
        for (int c = threadIdx.x; c < p.n; c += kLnLongThreads) {
            const float g = p.gamma ? load_as_float(p.gamma, p.param_dtype, c) : 1.f;
            const float b = p.beta ? load_as_float(p.beta, p.param_dtype, c) : 0.f;
            y[c] = elem_from_float<T>(fmaf(((elem_to_float(x[c]) - mean0) - st.shift) * st.rstd, g, b));
        }
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[row] = mean0 + st.shift;
            if (p.rstd) p.rstd[row] = st.rstd;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kLnLongThreads)
layernorm_long_dx_kernel(const LnRowsParams p)
{
    __shared__ float xch[2][32][2];
    grid_launch_dependents();
    grid_dependency_wait();
    int flip = 0;
    for (int row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(p.x) + row * p.ldx;
        const T *dy = static_cast<const T *>(p.dy) + row * p.lddy;
        T *dx = static_cast<T *>(p.y) + row * p.ldy;
        const float mean = p.mean[row], rstd = p.rstd[row];
        float s[2] = {0.f, 0.f};
        for (int c = threadIdx.x; c < p.n; c += kLnLongThreads) {
            const float g = elem_to_float(dy[c]) * (p.gamma ? load_as_float(p.gamma, p.param_dtype, c) : 1.f);
            s[0] += g;
            s[1] = fmaf(g, (elem_to_float(x[c]) - mean) * rstd, s[1]);
        }
        block_sum<kLnLongThreads, 2>(s, xch, flip);
        const float c1 = s[0] * p.inv_n, c2 = s[1] * p.inv_n;
        for (int c = threadIdx.x; c < p.n; c += kLnLongThreads) {
            const float g = elem_to_float(dy[c]) * (p.gamma ? load_as_float(p.gamma, p.param_dtype, c) : 1.f);
            const float xh = (elem_to_float(x[c]) - mean) * rstd;
            dx[c] = elem_from_float<T>(rstd * (g - fmaf(xh, c2, c1)));
        }
    }
}

// Column sums of long rows: grid (columns / 256, parts), one column per thread.  A sum that adds m values one after
// the other is off by up to m roundings, so 32 rows are added at a time, and then those sums (6000 x 8200 fp32:
// 86 us with the join, 4.6 TB/s; as one chain 109).
constexpr int kLnColumnRows = 32;
template <typename T>
__global__ void __launch_bounds__(256)
layernorm_long_columns_kernel(const LnRowsParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= p.n) return;
    const T *x = static_cast<const T *>(p.x) + c;
    const T *dy = static_cast<const T *>(p.dy) + c;
    float dg = 0.f, db = 0.f;
    long long row = blockIdx.y;
    while (row < p.rows) {
        float g = 0.f, b = 0.f;
        const long long end = min((long long)p.rows, row + (long long)kLnColumnRows * gridDim.y);
#pragma unroll 4
        for (; row < end; row += gridDim.y) {
            const float d = elem_to_float(dy[row * p.lddy]);
            g = fmaf(d, (elem_to_float(x[row * p.ldx]) - p.mean[row]) * p.rstd[row], g);
            b += d;
        }
        dg += g;
        db += b;
    }
    float *out = p.partials + (long long)blockIdx.y * 2 * p.n + c;
    out[0] = dg;
    out[p.n] = db;                                                 // (n + c may pass 2^31)
}

}  // namespace cudallm
