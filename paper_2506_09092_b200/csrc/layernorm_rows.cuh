// LayerNorm over the rows of a matrix, forward and backward.
//
//   forward   mean, rstd = 1 / sqrt(var + eps),  y = (x - mean) rstd gamma + beta
//   backward  xhat = (x - mean) rstd,  g = dy gamma,
//             dx = rstd (g - mean(g) - xhat mean(g xhat)),
//             dgamma = sum_rows dy xhat,  dbeta = sum_rows dy
//
// Bound: HBM (x read once, y written once; dy, x read and dx written once).  A row is
// held in registers between its statistics and its normalisation, so nothing is read
// twice.  The CTAs are persistent: a thread owns the same columns in every row that its
// CTA visits, so gamma and beta are read once per CTA (per row they would cost more L2
// traffic than the row itself), dgamma and dbeta are summed in registers, and the next
// row's loads are issued before the current row's reductions.
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

// Sum of `v` (NV values at once) over the TPR threads that share a row.  `xch` is used
// alternately (`flip`), so one barrier per call is enough.
template <int TPR, int NV>
__device__ __forceinline__ void row_sum(float (&v)[NV], float (*xch)[NV][32], int &flip)
{
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    if (TPR > 32) {
        constexpr int kWarps = TPR / 32;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < NV; ++k) xch[flip][k][warp] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float s = lane < kWarps ? xch[flip][k][lane] : 0.f;
#pragma unroll
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            v[k] = s;
        }
        flip ^= 1;
    }
}

__host__ __device__ constexpr int ln_threads(int tpr) { return tpr == 32 ? 256 : tpr; }

// VPT pieces of VEC elements per thread, TPR threads per row: rows of up to TPR * VPT * VEC
// elements.  Piece v of thread t covers columns (v * TPR + t) * VEC ...: a warp's accesses are
// contiguous.  n is a multiple of VEC.
template <typename T, int VEC, int TPR, int VPT>
__global__ void __launch_bounds__(ln_threads(TPR))
layernorm_rows_kernel(const LnRowsParams p)
{
    __shared__ float xch1[2][1][32];
    __shared__ float xch2[2][2][32];
    constexpr int kRows = ln_threads(TPR) / TPR;                  // rows a CTA works on at a time
    const int t = threadIdx.x % TPR;
    const int stride = gridDim.x * kRows;
    int row = blockIdx.x * kRows + threadIdx.x / TPR;
    const T *x = static_cast<const T *>(p.x);
    T *y = static_cast<T *>(p.y);
    grid_launch_dependents();
    grid_dependency_wait();

    Piece<T, VEC> next[VPT];
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int c = (v * TPR + t) * VEC;
        next[v].clear();
        if (row < p.rows && c < p.n) next[v].load(x + row * p.ldx + c);
    }
    float gamma[VPT][VEC], beta[VPT][VEC];
#pragma unroll
    for (int v = 0; v < VPT; ++v)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int c = (v * TPR + t) * VEC + e;
            gamma[v][e] = (p.gamma && c < p.n) ? load_as_float(p.gamma, p.param_dtype, c) : 1.f;
            beta[v][e] = (p.beta && c < p.n) ? load_as_float(p.beta, p.param_dtype, c) : 0.f;
        }

    int flip1 = 0, flip2 = 0;
    // every thread of a CTA runs the same number of rounds (barriers inside)
    for (int base = blockIdx.x * kRows; base < p.rows; base += stride, row += stride) {
        float f[VPT][VEC];
        float s[1] = {0.f};
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            next[v].unpack(f[v]);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[0] += f[v][e];        // columns beyond n hold zeros
        }
        const long long nrow = (long long)row + stride;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int c = (v * TPR + t) * VEC;
            if (nrow < p.rows && c < p.n) next[v].load(x + nrow * p.ldx + c);
        }
        row_sum<TPR, 1>(s, xch1, flip1);
        const float mean0 = s[0] * p.inv_n;
        // differences to the first mean; their own mean corrects it (a mean far above the
        // spread is off by its fp32 rounding, the differences are not)
        float d[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const bool live = (v * TPR + t) * VEC < p.n;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                f[v][e] = live ? f[v][e] - mean0 : 0.f;
                d[0] += f[v][e];
                d[1] = fmaf(f[v][e], f[v][e], d[1]);
            }
        }
        row_sum<TPR, 2>(d, xch2, flip2);
        const float shift = d[0] * p.inv_n;
        const float var = fmaxf(fmaf(-shift, shift, d[1] * p.inv_n), 0.f);
        // (fmaxf drops a NaN: a row that holds one keeps it in d[1], which is tested here)
        const float rstd = d[1] == d[1] ? 1.f / sqrtf(var + p.eps) : d[1];
        if (row < p.rows) {
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                const int c = (v * TPR + t) * VEC;
                if (c < p.n) {
                    float o[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) o[e] = fmaf((f[v][e] - shift) * rstd, gamma[v][e], beta[v][e]);
                    Piece<T, VEC> out;
                    out.pack(o);
                    out.store(y + row * p.ldy + c);
                }
            }
            if (t == 0) {
                if (p.mean) p.mean[row] = mean0 + shift;
                if (p.rstd) p.rstd[row] = rstd;
            }
        }
    }
}

// Backward.  One reduction per row (mean(g) and mean(g xhat) together).
template <typename T, int VEC, int TPR, int VPT>
__global__ void __launch_bounds__(ln_threads(TPR))
layernorm_rows_bwd_kernel(const LnRowsParams p)
{
    constexpr int kRows = ln_threads(TPR) / TPR;
    constexpr int kCols = TPR * VPT * VEC;
    __shared__ float xch[2][2][32];
    __shared__ float join[kRows > 1 ? kRows : 1][kRows > 1 ? kCols : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int stride = gridDim.x * kRows;
    int row = blockIdx.x * kRows + sub;
    const T *x = static_cast<const T *>(p.x);
    const T *dy = static_cast<const T *>(p.dy);
    T *dx = static_cast<T *>(p.y);
    grid_launch_dependents();
    grid_dependency_wait();

    Piece<T, VEC> nx[VPT], ny[VPT];
    float nmean = 0.f, nrstd = 0.f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int c = (v * TPR + t) * VEC;
        nx[v].clear();
        ny[v].clear();
        if (row < p.rows && c < p.n) {
            nx[v].load(x + row * p.ldx + c);
            ny[v].load(dy + row * p.lddy + c);
        }
    }
    if (row < p.rows) { nmean = p.mean[row]; nrstd = p.rstd[row]; }
    float gamma[VPT][VEC], dg[VPT][VEC], db[VPT][VEC];
#pragma unroll
    for (int v = 0; v < VPT; ++v)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const int c = (v * TPR + t) * VEC + e;
            gamma[v][e] = (p.gamma && c < p.n) ? load_as_float(p.gamma, p.param_dtype, c) : 1.f;
            dg[v][e] = db[v][e] = 0.f;
        }

    int flip = 0;
    for (int base = blockIdx.x * kRows; base < p.rows; base += stride, row += stride) {
        const bool live_row = row < p.rows;
        const float mean = nmean, rstd = nrstd;
        float xh[VPT][VEC], g[VPT][VEC];
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const bool live = live_row && (v * TPR + t) * VEC < p.n;
            nx[v].unpack(xh[v]);
            ny[v].unpack(g[v]);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                xh[v][e] = live ? (xh[v][e] - mean) * rstd : 0.f;
                const float d = live ? g[v][e] : 0.f;             // (a finished row's last values stay in the registers)
                dg[v][e] = fmaf(d, xh[v][e], dg[v][e]);
                db[v][e] += d;
                g[v][e] = d * gamma[v][e];
                s[0] += g[v][e];
                s[1] = fmaf(g[v][e], xh[v][e], s[1]);
            }
        }
        const long long nrow = (long long)row + stride;
        if (nrow < p.rows) {
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                const int c = (v * TPR + t) * VEC;
                if (c < p.n) {
                    nx[v].load(x + nrow * p.ldx + c);
                    ny[v].load(dy + nrow * p.lddy + c);
                }
            }
            nmean = p.mean[nrow];
            nrstd = p.rstd[nrow];
        }
        if (dx) {
            row_sum<TPR, 2>(s, xch, flip);
            const float c1 = s[0] * p.inv_n, c2 = s[1] * p.inv_n;
#pragma unroll
            for (int v = 0; v < VPT; ++v) {
                const int c = (v * TPR + t) * VEC;
                if (live_row && c < p.n) {
                    float o[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) o[e] = rstd * (g[v][e] - fmaf(xh[v][e], c2, c1));
                    Piece<T, VEC> out;
                    out.pack(o);
                    out.store(dx + row * p.ldy + c);
                }
            }
        }
    }

    if (!p.partials) return;
    float *out = p.partials + (long long)blockIdx.x * 2 * p.n;
    if (kRows == 1) {
#pragma unroll
        for (int v = 0; v < VPT; ++v)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int c = (v * TPR + t) * VEC + e;
                if (c < p.n) {
                    out[c] = dg[v][e];
                    out[p.n + c] = db[v][e];
                }
            }
    } else {
        // the CTA's rows join in shared memory, in order
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < VPT; ++v)
#pragma unroll
                for (int e = 0; e < VEC; ++e) join[sub][(v * TPR + t) * VEC + e] = k ? db[v][e] : dg[v][e];
            __syncthreads();
            for (int c = threadIdx.x; c < p.n; c += blockDim.x) {
                float a = 0.f;
#pragma unroll
                for (int r = 0; r < kRows; ++r) a += join[r][c];
                out[(long long)k * p.n + c] = a;
            }
        }
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
template <int NV>
__device__ __forceinline__ void block_sum(float (&v)[NV], float (*xch)[NV][32], int &flip)
{
    row_sum<kLnLongThreads, NV>(v, xch, flip);
}

template <typename T>
__global__ void __launch_bounds__(kLnLongThreads)
layernorm_long_kernel(const LnRowsParams p)
{
    __shared__ float xch1[2][1][32];
    __shared__ float xch2[2][2][32];
    grid_launch_dependents();
    grid_dependency_wait();
    int flip1 = 0, flip2 = 0;
    for (int row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(p.x) + row * p.ldx;
        T *y = static_cast<T *>(p.y) + row * p.ldy;
        float s[1] = {0.f};
        for (int c = threadIdx.x; c < p.n; c += kLnLongThreads) s[0] += elem_to_float(x[c]);
        block_sum<1>(s, xch1, flip1);
        const float mean0 = s[0] * p.inv_n;
        float d[2] = {0.f, 0.f};
        for (int c = threadIdx.x; c < p.n; c += kLnLongThreads) {
            const float f = elem_to_float(x[c]) - mean0;
            d[0] += f;
            d[1] = fmaf(f, f, d[1]);
        }
        block_sum<2>(d, xch2, flip2);
        const float shift = d[0] * p.inv_n;
        const float var = fmaxf(fmaf(-shift, shift, d[1] * p.inv_n), 0.f);
        const float rstd = d[1] == d[1] ? 1.f / sqrtf(var + p.eps) : d[1];
        for (int c = threadIdx.x; c < p.n; c += kLnLongThreads) {
            const float g = p.gamma ? load_as_float(p.gamma, p.param_dtype, c) : 1.f;
            const float b = p.beta ? load_as_float(p.beta, p.param_dtype, c) : 0.f;
            y[c] = elem_from_float<T>(fmaf(((elem_to_float(x[c]) - mean0) - shift) * rstd, g, b));
        }
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[row] = mean0 + shift;
            if (p.rstd) p.rstd[row] = rstd;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kLnLongThreads)
layernorm_long_dx_kernel(const LnRowsParams p)
{
    __shared__ float xch[2][2][32];
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
        block_sum<2>(s, xch, flip);
        const float c1 = s[0] * p.inv_n, c2 = s[1] * p.inv_n;
        for (int c = threadIdx.x; c < p.n; c += kLnLongThreads) {
            const float g = elem_to_float(dy[c]) * (p.gamma ? load_as_float(p.gamma, p.param_dtype, c) : 1.f);
            const float xh = (elem_to_float(x[c]) - mean) * rstd;
            dx[c] = elem_from_float<T>(rstd * (g - fmaf(xh, c2, c1)));
        }
    }
}

// Column sums of long rows: grid (columns / 256, parts), one column per thread.
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
#pragma unroll 4
    for (int row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const float d = elem_to_float(dy[row * p.lddy]);
        dg = fmaf(d, (elem_to_float(x[row * p.ldx]) - p.mean[row]) * p.rstd[row], dg);
        db += d;
    }
    float *out = p.partials + (long long)blockIdx.y * 2 * p.n;
    out[c] = dg;
    out[p.n + c] = db;
}

}  // namespace cudallm
