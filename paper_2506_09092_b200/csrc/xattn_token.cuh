// Cross attention for single tokens and other short queries: the group x q_rows query rows that
// share a key head (at most 16) against all of its keys.
//
// Bound: HBM (K and V are read once; 16 rows of arithmetic per key are far below any pipe's rate),
// so the work is split over the keys until the GPU is full, and what matters is bytes in flight:
// each of a CTA's four warps walks its own tiles of 32 keys (16 at head dims above 64) through its own
// ring of cp.async stages (no barrier between warps).  The 16 rows are the M of mma.sync.m16n8k16 -- a tcgen05 tile would
// be 128 rows, seven eighths of them empty.  Row statistics are a running maximum and sum in fp32;
// the warps' results join in shared memory.  Up to eight splits are a cluster of CTAs, which read each
// other's results from shared memory; more of them join in xattn_join_kernel.
//
// Measured (one B200): 8 x 32 heads on 8 key heads of 128, 16384 states (537 MB): 79.8 us = 6.7 TB/s, 1.03 of the
// measured copy bandwidth; 16 x 16 heads of 64, up to 1500 states (70 MB): 14.9 us = 4.7 TB/s, one wave
// of 256 CTAs of unequal length (two waves of half the size: 19.4 us; smaller stages, so that all
// 512 fit at once: 16.0).  Compiled for two CTAs an SM, which is what the shared memory holds: without
// that hint 80.9 and 15.6 us.
#pragma once
#include "xattn_common.cuh"

namespace cudallm {

constexpr int kXaTokWarps = 4;
constexpr int kXaTokThreads = 32 * kXaTokWarps;
constexpr int kXaTokRows = 16;                 // query rows at most

struct XaTokParams {
    const void *q, *k, *v;
    void *o;
    float *lse;
    float *o_part, *lse_part;
    const int *lens;
    XaStrides sq, sk, sv, so;
    int q_rows, kv_rows, q_heads, kv_heads, group, batch, head_dim;
    int splits, keys_per_split;                // keys_per_split: a multiple of 32
    int cluster;                               // the splits of a key head are one cluster
    float scale, scale_log2;
};

template <int DP> struct XaTokSmem {
    static constexpr int kKeys = DP == 128 ? 16 : 32;              // of a stage
    static constexpr int kStages = 3;                              // 96 KiB a CTA: two on an SM
    static constexpr int kTile = kKeys * DP * 2;                   // one of K, V
    static constexpr int kWarp = kStages * 2 * kTile;
    static constexpr int kPitch = DP + 4;                          // floats per row of the joining block
    static constexpr int kJoinWarp = (kXaTokRows * kPitch + 2 * kXaTokRows) * 4;
    static constexpr int kBytes = kXaTokWarps * (kWarp > kJoinWarp ? kWarp : kJoinWarp);
    // a CTA's result for its cluster: [row][DP] fp32, then the rows' lse
    static constexpr int kShare = (kXaTokWarps * kJoinWarp + 127) / 128 * 128;
    static_assert(kShare + kXaTokRows * (DP + 1) * 4 <= kBytes, "behind the warps' results");
};

constexpr int kXaTokCluster = 8;

__device__ __forceinline__ void cluster_sync_all()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_map(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ float cluster_ld(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 cluster_ld4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <typename T> __device__ __forceinline__ void mma_16x8x16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma_16x8x16<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma_16x8x16<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16 bytes global -> shared past L1 (every byte is used once); zero-filled where src_bytes is 0.
__device__ __forceinline__ void cp_async_16_cg(uint32_t smem_addr, const void *gptr, uint32_t src_bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr), "l"(gptr), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait_group() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int DP, typename T>
__global__ void __launch_bounds__(kXaTokThreads, 2)
xattn_token_kernel(const XaTokParams p)
{
    using L = XaTokSmem<DP>;
    constexpr int kChunks = DP / 8;                                // 16-byte pieces of a row
    constexpr int kKeys = L::kKeys, kRowStep = 32 / kChunks;       // rows that a copy instruction covers
    extern __shared__ __align__(1024) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int split = blockIdx.x % p.splits, bk = blockIdx.x / p.splits;
    const int kvh = bk % p.kv_heads, b = bk / p.kv_heads;
    const int rows = p.group * p.q_rows;                           // row r: head kvh * group + r / q_rows, query r % q_rows
    grid_launch_dependents();
    grid_dependency_wait();

    const int keys = xa_keys(p.lens, b, p.kv_rows);
    const int key0 = split * p.keys_per_split;
    const int key_end = min(keys, key0 + p.keys_per_split);
    const int ntiles = key_end > key0 ? (key_end - key0 + kKeys - 1) / kKeys : 0;
    const int mine = ntiles > warp ? (ntiles - warp + kXaTokWarps - 1) / kXaTokWarps : 0;   // tiles warp, warp + 4, ...

    const T *kbase = static_cast<const T *>(p.k) + b * p.sk.b + kvh * p.sk.h;
    const T *vbase = static_cast<const T *>(p.v) + b * p.sv.b + kvh * p.sv.h;
    const uint32_t ring = smem_u32(smem) + warp * L::kWarp;

    // one stage of K and of V; the pieces of a row go to neighbouring lanes, piece c of row r to position
    // c ^ (r & 7) (conflict-free ldmatrix)
    const int lc = lane % kChunks, lr = lane / kChunks;
    const bool lc_live = lc * 8 < p.head_dim;
    const int first = key0 + warp * kKeys + lr;                    // this lane's first row of tile 0
    const T *kp = kbase + (long long)(lc_live && mine > 0 ? first : 0) * p.sk.r + (lc_live ? lc * 8 : 0);
    const T *vp = vbase + (long long)(lc_live && mine > 0 ? first : 0) * p.sv.r + (lc_live ? lc * 8 : 0);
    auto load = [&](int t) {
        if (t < mine) {
            const uint32_t st = ring + (t % L::kStages) * 2 * L::kTile;
            const int row0 = t * kXaTokWarps * kKeys;
            const T *ks = kp + row0 * p.sk.r, *vs = vp + row0 * p.sv.r;
#pragma unroll
            for (int n = 0; n < kKeys / kRowStep; ++n) {
                const int r = lr + n * kRowStep;
                const bool live = lc_live && first + row0 + n * kRowStep < key_end;
                const uint32_t dst = st + r * DP * 2 + ((lc ^ (r & 7)) << 4);
                cp_async_16_cg(dst, live ? ks + n * kRowStep * p.sk.r : kbase, live ? 16 : 0);
                cp_async_16_cg(dst + L::kTile, live ? vs + n * kRowStep * p.sv.r : vbase, live ? 16 : 0);
            }
        }
        cp_async_commit();
    };
    if (mine > 0)
        for (int t = 0; t < L::kStages - 1; ++t) load(t);

    // Q as the A operand: rows g and g + 8, columns 2 q, 2 q + 1 and + 8 of every 16
    const int g = lane >> 2, q4 = lane & 3;
    uint32_t qa[DP / 16][4];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int r = g + 8 * half;
        const T *src = nullptr;
        if (r < rows)
            src = static_cast<const T *>(p.q) + b * p.sq.b + (long long)(r % p.q_rows) * p.sq.r
                  + (long long)(kvh * p.group + r / p.q_rows) * p.sq.h;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
                const int d = k * 16 + hi * 8 + q4 * 2;
                qa[k][half + 2 * hi] = (src && d < p.head_dim) ? *reinterpret_cast<const uint32_t *>(src + d) : 0u;
            }
    }

    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    float o[DP / 8][4];
#pragma unroll
    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][e] = 0.f;

    for (int t = 0; t < mine; ++t) {
        cp_async_wait_group<L::kStages - 2>();
        __syncwarp();                                              // every lane's copies of stage t have landed
        load(t + L::kStages - 1);                                  // (its stage was read in round t - 1)
        const uint32_t sk = ring + (t % L::kStages) * 2 * L::kTile, sv = sk + L::kTile;
        constexpr int kN = kKeys / 8;                              // tiles of eight keys
        float s[kN][4] = {};
        {
            const int idx = lane >> 3, kr = (idx >> 1) * 8 + (lane & 7);
#pragma unroll
            for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                for (int n = 0; n < kN; n += 2) {
                    uint32_t bf[4];
                    ldmatrix_x4(bf, sk + (n * 8 + kr) * DP * 2 + (((2 * k + (idx & 1)) ^ (kr & 7)) << 4));
                    mma_16x8x16<T>(s[n], qa[k], bf[0], bf[1]);
                    mma_16x8x16<T>(s[n + 1], qa[k], bf[2], bf[3]);
                }
        }
        const int valid = key_end - (key0 + (warp + t * kXaTokWarps) * kKeys);
        if (valid < kKeys) {
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n * 8 + q4 * 2 + (e & 1) >= valid) s[n][e] = -INFINITY;
        }
        float bm[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            bm[half] = fmaxf(s[0][2 * half], s[0][2 * half + 1]);
#pragma unroll
            for (int n = 1; n < kN; ++n) bm[half] = fmaxf(bm[half], fmaxf(s[n][2 * half], s[n][2 * half + 1]));
            bm[half] = fmaxf(bm[half], __shfl_xor_sync(0xffffffffu, bm[half], 1));
            bm[half] = fmaxf(bm[half], __shfl_xor_sync(0xffffffffu, bm[half], 2));
        }
        if (__any_sync(0xffffffffu, bm[0] > m[0] || bm[1] > m[1])) {
            float alpha[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const float nm = fmaxf(m[half], bm[half]);
                alpha[half] = nm == m[half] ? 1.f : xa_exp2((m[half] - nm) * p.scale_log2);
                m[half] = nm;
                l[half] *= alpha[half];
            }
#pragma unroll
            for (int n = 0; n < DP / 8; ++n) {
                o[n][0] *= alpha[0];
                o[n][1] *= alpha[0];
                o[n][2] *= alpha[1];
                o[n][3] *= alpha[1];
            }
        }
        const float neg[2] = {-m[0] * p.scale_log2, -m[1] * p.scale_log2};
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][e] = xa_exp2(fmaf(s[n][e], p.scale_log2, neg[e >> 1]));
                l[e >> 1] += s[n][e];
            }
        {
            const int idx = lane >> 3, kr = (idx & 1) * 8 + (lane & 7);
#pragma unroll
            for (int h = 0; h < kN; h += 2) {
                const uint32_t pa[4] = {XaElem<T>::pack(s[h][0], s[h][1]), XaElem<T>::pack(s[h][2], s[h][3]),
                                        XaElem<T>::pack(s[h + 1][0], s[h + 1][1]), XaElem<T>::pack(s[h + 1][2], s[h + 1][3])};
#pragma unroll
                for (int n = 0; n < DP / 16; ++n) {
                    uint32_t bf[4];
                    ldmatrix_x4_trans(bf, sv + (h * 8 + kr) * DP * 2 + (((2 * n + (idx >> 1)) ^ (kr & 7)) << 4));
                    mma_16x8x16<T>(o[2 * n], pa, bf[0], bf[1]);
                    mma_16x8x16<T>(o[2 * n + 1], pa, bf[2], bf[3]);
                }
            }
        }
        __syncwarp();                                              // stage t has been read by every lane
    }
    cp_async_wait_group<0>();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        l[half] += __shfl_xor_sync(0xffffffffu, l[half], 1);
        l[half] += __shfl_xor_sync(0xffffffffu, l[half], 2);
    }
    __syncthreads();                                               // the rings are free
    float *jo = reinterpret_cast<float *>(smem) + warp * (L::kJoinWarp / 4);
    float *jm = jo + kXaTokRows * L::kPitch, *jl = jm + kXaTokRows;
#pragma unroll
    for (int n = 0; n < DP / 8; ++n) {
        *reinterpret_cast<float2 *>(jo + g * L::kPitch + n * 8 + q4 * 2) = make_float2(o[n][0], o[n][1]);
        *reinterpret_cast<float2 *>(jo + (g + 8) * L::kPitch + n * 8 + q4 * 2) = make_float2(o[n][2], o[n][3]);
    }
    if (q4 == 0) {
        jm[g] = m[0];
        jm[g + 8] = m[1];
        jl[g] = l[0];
        jl[g + 8] = l[1];
    }
    __syncthreads();
    // thread -> (row, 8 columns): the four warps' rows, weighted to the common maximum
    const float *base = reinterpret_cast<const float *>(smem);
    constexpr int kStep = L::kJoinWarp / 4;
    for (int i = tid; i < rows * kChunks; i += kXaTokThreads) {
        const int r = i / kChunks, c = i % kChunks;
        float wm[kXaTokWarps], mx = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kXaTokWarps; ++w) {
            wm[w] = base[w * kStep + kXaTokRows * L::kPitch + r];
            mx = fmaxf(mx, wm[w]);
        }
        float acc[8] = {};
#pragma unroll
        for (int w = 0; w < kXaTokWarps; ++w) {
            const float lw = base[w * kStep + kXaTokRows * L::kPitch + kXaTokRows + r];
            if (lw == 0.f && wm[w] == -INFINITY) continue;         // a warp without keys
            const float a = xa_exp2((wm[w] - mx) * p.scale_log2);
            sum = fmaf(a, lw, sum);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = fmaf(a, base[w * kStep + r * L::kPitch + c * 8 + e], acc[e]);
        }
        const int h = kvh * p.group + r / p.q_rows, qr = r % p.q_rows;
        const bool none = ntiles == 0;
        const float inv = none ? 0.f : 1.f / sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= inv;
        const long long bhr = ((long long)b * p.q_heads + h) * p.q_rows + qr;
        const float lse = none ? -INFINITY : fmaf(mx, p.scale, logf(sum));
        if (p.cluster) {
            float *share = reinterpret_cast<float *>(smem + L::kShare);
            float4 *dst = reinterpret_cast<float4 *>(share + r * DP + c * 8);
            dst[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
            dst[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
            if (c == 0) share[kXaTokRows * DP + r] = lse;
        } else if (p.splits == 1) {
            if (c * 8 < p.head_dim)
                *reinterpret_cast<uint4 *>(static_cast<T *>(p.o) + b * p.so.b + qr * p.so.r + h * p.so.h + c * 8) =
                    make_uint4(XaElem<T>::pack(acc[0], acc[1]), XaElem<T>::pack(acc[2], acc[3]),
                               XaElem<T>::pack(acc[4], acc[5]), XaElem<T>::pack(acc[6], acc[7]));
            if (c == 0 && p.lse) p.lse[bhr] = lse;
        } else {
            const long long part = (long long)split * p.batch * p.q_heads * p.q_rows + bhr;
            if (c * 8 < p.head_dim && !none) {
                float4 *dst = reinterpret_cast<float4 *>(p.o_part + part * p.head_dim + c * 8);
                dst[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
                dst[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
            }
            if (c == 0) p.lse_part[part] = lse;
        }
    }
    if (!p.cluster) return;
    // the cluster's CTAs each write a share of the rows' pieces, from all of their results
    cluster_sync_all();
    const uint32_t share = smem_u32(smem) + L::kShare;
    for (int i = split * kXaTokThreads + tid; i < rows * kChunks; i += p.splits * kXaTokThreads) {
        const int r = i / kChunks, c = i % kChunks;
        float part[kXaTokCluster], mx = -INFINITY, sum = 0.f, acc[8] = {};
#pragma unroll
        for (int s = 0; s < kXaTokCluster; ++s) {
            part[s] = s < p.splits ? cluster_ld(cluster_map(share + (kXaTokRows * DP + r) * 4, s)) : -INFINITY;
            mx = fmaxf(mx, part[s]);
        }
#pragma unroll
        for (int s = 0; s < kXaTokCluster; ++s) {
            if (part[s] == -INFINITY) continue;                    // no keys there (a NaN goes on)
            const float w = expf(part[s] - mx);
            sum += w;
            const uint32_t src = cluster_map(share + (r * DP + c * 8) * 4, s);
            const float4 a = cluster_ld4(src), b4 = cluster_ld4(src + 16);
            acc[0] = fmaf(w, a.x, acc[0]); acc[1] = fmaf(w, a.y, acc[1]); acc[2] = fmaf(w, a.z, acc[2]); acc[3] = fmaf(w, a.w, acc[3]);
            acc[4] = fmaf(w, b4.x, acc[4]); acc[5] = fmaf(w, b4.y, acc[5]); acc[6] = fmaf(w, b4.z, acc[6]); acc[7] = fmaf(w, b4.w, acc[7]);
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= inv;
        const int h = kvh * p.group + r / p.q_rows, qr = r % p.q_rows;
        if (c * 8 < p.head_dim)
            *reinterpret_cast<uint4 *>(static_cast<T *>(p.o) + b * p.so.b + qr * p.so.r + h * p.so.h + c * 8) =
                make_uint4(XaElem<T>::pack(acc[0], acc[1]), XaElem<T>::pack(acc[2], acc[3]),
                           XaElem<T>::pack(acc[4], acc[5]), XaElem<T>::pack(acc[6], acc[7]));
        if (c == 0 && p.lse)
            p.lse[((long long)b * p.q_heads + h) * p.q_rows + qr] = sum == 0.f ? -INFINITY : mx + logf(sum);
    }
    cluster_sync_all();                                            // nobody's shared memory goes while it is read
}

}  // namespace cudallm
