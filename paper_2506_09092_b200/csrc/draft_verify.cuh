// Drafted tokens against the target's probabilities.
//
// Bound: latency where the vocabulary is small (numbers of the drafts -> their probabilities -> the row to draw from, three
// dependent loads), HBM where it is large (one row of p and one of q per sequence are read once).  A
// cluster of CTAs works on a sequence: each decides which drafts hold by itself, sums up its part of the
// row that the next token is drawn from, chunk by chunk, and learns the others' sums from their shared
// memory.  The CTA whose part holds the drawn point reads one chunk again (from L2), element by element.
// 64 sequences of 128000 fp32 values: 15.8 to 16.4 us for 65 MB (floor 10.0): the front, the tail and the two conversions and
// additions in 64 bits of an element (with one of each: 13.8).  The same work an element whatever its type: bf16 17.4 us, fp16 16.9 (floor
// 5.0), certain drafts 15.0 to 16.6.  Two CTAs an SM of 128 registers a thread: three of 80 spill (19.4 us),
// one of 512 threads takes 16.3; parts of 1024 values 21.6, of 256 19.1.
//
// Everything is in 64 bits: products of two fp32 values and differences of two are exact there, and a sum
// is off by 2^-53 of itself per addition, so that the point drawn is the one that any order of summation
// would give but for one in some 10^10.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "elem.cuh"
#include "mma_sync.cuh"
#include "ptx.cuh"

namespace cudallm {

constexpr int kVerifyThreads = 256;
constexpr int kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyChunk = 512;              // elements that a warp sums up at a time (or a multiple, for huge rows)
constexpr int kVerifyChunks = 1024;            // of a CTA at most
constexpr int kVerifyCluster = 8;

struct VerifyParams {
    const void *p, *q;
    const int *drafts, *draft_lens;
    const float *u;
    int *tokens, *accepted;
    long long ldp, ldq;
    int n, vocab, cluster;
    int chunk, chunks;                         // elements of a chunk (a multiple of 512), chunks of a CTA
};

template <typename T> __device__ __forceinline__ double elem_to_double(T v) { return (double)elem_to_float(v); }
__device__ __forceinline__ double cluster_ld_f64(uint32_t addr)
{
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
    return v;
}

// What an element adds to the row that the token is drawn from: p - q where that is positive and finite, in 64 bits.  (fp32 says
// so exactly: a difference of two values is zero there only if they are equal.  As two choices under one predicate: a
// branch for each element costs more than its sum, 24 us instead of 16 for 64 rows of 128000.)
template <typename T> __device__ __forceinline__ double mass(T p, T q)
{
    float x = elem_to_float(p), y = elem_to_float(q);
    asm("{\n\t.reg .pred p;\n\tsetp.gt.f32 p, %2, 0f00000000;\n\tsetp.lt.and.f32 p, %2, 0f7F800000, p;\n\t"
        "selp.f32 %0, %0, 0f00000000, p;\n\tselp.f32 %1, %1, 0f00000000, p;\n\t}"
        : "+f"(x), "+f"(y) : "f"(x - y));
    return (double)x - (double)y;
}

// N elements a lane of the 32 N from `from` on, zeros behind the end; `certain`: the one place where q is one.  VEC elements lie side
// by side in 16 bytes (rows that begin there), else neighbouring lanes have neighbouring elements.
template <int VEC, typename T, int N>
__device__ __forceinline__ void verify_load(const T *prow, const T *qrow, long long from, int vocab, int certain, T (&pv)[N], T (&qv)[N])
{
    const int lane = threadIdx.x & 31;
    const T zero = elem_from_float<T>(0.f), one = elem_from_float<T>(1.f);
    const int left = (int)min((long long)vocab - from, 32LL * N);  // (may be negative)
    int mine = -1;                                                 // the certain one's place among this lane's
    const long long at = certain - from;
    const bool here = certain >= 0 && at >= 0 && at < 32 * N;
    if (VEC > 1 && left == 32 * N) {
        union Piece {
            uint4 w;
            T e[VEC];
            __device__ Piece() {}
        };
#pragma unroll
        for (int i = 0; i < N; i += VEC) {
            Piece x;
            x.w = *reinterpret_cast<const uint4 *>(prow + from + i * 32 + lane * VEC);
#pragma unroll
            for (int e = 0; e < VEC; ++e) pv[i + e] = x.e[e];
        }
#pragma unroll
        for (int i = 0; i < N; i += VEC) {
            Piece x;
            if (qrow) x.w = *reinterpret_cast<const uint4 *>(qrow + from + i * 32 + lane * VEC);
#pragma unroll
            for (int e = 0; e < VEC; ++e) qv[i + e] = qrow ? x.e[e] : zero;
        }
        if (here && (int)at / VEC % 32 == lane) mine = (int)at / (32 * VEC) * VEC + (int)at % VEC;
    } else {
        const T *ps = prow + from + lane, *qs = qrow + from + lane;
#pragma unroll
        for (int i = 0; i < N; ++i) pv[i] = i * 32 + lane < left ? ps[i * 32] : zero;
#pragma unroll
        for (int i = 0; i < N; ++i) qv[i] = qrow && i * 32 + lane < left ? qs[i * 32] : zero;
        if (here && (int)at % 32 == lane) mine = (int)at / 32;
    }
    if (here) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i == mine) qv[i] = one;
    }
}

template <typename T, int VEC>
__global__ void __launch_bounds__(kVerifyThreads, 2)
draft_verify_kernel(const VerifyParams p)
{
    __shared__ double masses[kVerifyChunks], sums[kVerifyChunks], cta_sum;     // of each chunk; up to and with each; of all
    __shared__ int s_accepted;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = blockIdx.x % p.cluster, b = blockIdx.x / p.cluster;
    grid_launch_dependents();
    grid_dependency_wait();

    const T *pp = static_cast<const T *>(p.p) + (long long)b * (p.n + 1) * p.ldp;
    const T *qq = p.q ? static_cast<const T *>(p.q) + (long long)b * p.n * p.ldq : nullptr;
    const int *drafts = p.drafts + (long long)b * p.n;
    const float *u = p.u + (long long)b * (p.n + 1);
    const int m = p.draft_lens ? min(max(p.draft_lens[b], 0), p.n) : p.n;
    const double draw = (double)u[p.n];
    if (warp == 0) {
        int a = m;
        for (int t0 = 0; t0 < p.n; t0 += 32) {                     // (m is not waited for: the drafts behind it are looked at, too)
            const int t = t0 + lane;
            bool good = false;
            if (t < p.n) {
                const int x = drafts[t];
                const float ut = u[t];
                if ((unsigned)x < (unsigned)p.vocab) {
                    const double qx = qq ? elem_to_double(qq[t * p.ldq + x]) : 1.0;
                    good = (double)ut * qx < elem_to_double(pp[t * p.ldp + x]);
                }
            }
            const uint32_t bad = __ballot_sync(0xffffffffu, !good);
            if (bad) {
                a = min(m, t0 + __ffs(bad) - 1);
                break;
            }
        }
        if (lane == 0) s_accepted = a;
    }
    __syncthreads();
    const int a = s_accepted;
    // what is drawn from: max(p_a - q_a, 0) while drafts are left, q_a being a row or 1 at `certain`; else p_a
    const T *prow = pp + a * p.ldp, *qrow = a < m && qq ? qq + a * p.ldq : nullptr;
    int certain = a < m && !qq ? drafts[a] : -1;
    double point, before;                                          // where in the sum of all; the sum of the CTAs before this one
    int owner;                                                     // the CTA that holds the point
    for (int pass = 0;; ++pass) {
        // a warp's chunks, each in parts of 512 elements; the next part is asked for before one is summed up
        const int parts = p.chunk / kVerifyChunk, mine = p.chunks > warp ? ((p.chunks - warp - 1) / kVerifyWarps + 1) * parts : 0;
        auto at = [&](int k) { return ((long long)rank * p.chunks + warp + k / parts * kVerifyWarps) * p.chunk + k % parts * kVerifyChunk; };
        T pv[2][16], qv[2][16];
        double s = 0.0;
        if (mine > 0) verify_load<VEC>(prow, qrow, at(0), p.vocab, certain, pv[0], qv[0]);
        for (int k0 = 0; k0 < mine; k0 += 2) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = k0 + h;
                if (k + 1 < mine) verify_load<VEC>(prow, qrow, at(k + 1), p.vocab, certain, pv[h ^ 1], qv[h ^ 1]);
                if (k >= mine) break;
                double part[4] = {};
#pragma unroll
                for (int i = 0; i < 16; ++i) part[i % 4] += mass(pv[h][i], qv[h][i]);
                s += (part[0] + part[1]) + (part[2] + part[3]);
                if (k % parts == parts - 1) {
#pragma unroll
                    for (int d = 16; d; d /= 2) s += __shfl_xor_sync(0xffffffffu, s, d);
                    if (lane == 0) masses[warp + k / parts * kVerifyWarps] = s;
                    s = 0.0;
                }
            }
        }
        __syncthreads();
        if (warp == 0) {
            double upto = 0.0;
            for (int c0 = 0; c0 < p.chunks; c0 += 32) {
                double s = c0 + lane < p.chunks ? masses[c0 + lane] : 0.0;
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const double x = __shfl_up_sync(0xffffffffu, s, d);
                    if (lane >= d) s += x;
                }
                s += upto;
                if (c0 + lane < p.chunks) sums[c0 + lane] = s;
                upto = __shfl_sync(0xffffffffu, s, 31);
            }
            if (lane == 0) cta_sum = upto;
        }
        __syncthreads();
        double cta[kVerifyCluster], all = 0.0;
        if (p.cluster > 1) cluster_sync_all();
#pragma unroll
        for (int c = 0; c < kVerifyCluster; ++c) {
            cta[c] = c >= p.cluster ? 0.0 : p.cluster > 1 ? cluster_ld_f64(cluster_map(smem_u32(&cta_sum), c)) : cta_sum;
            all += cta[c];
        }
        point = draw * all;
        owner = -1;
        before = 0.0;
        double upto = 0.0;
        int last = -1;
#pragma unroll
        for (int c = 0; c < kVerifyCluster; ++c) {
            if (c == rank) before = upto;
            if (cta[c] > 0.0) {
                last = c;
                if (owner < 0 && upto + cta[c] > point) owner = c;
            }
            upto += cta[c];
        }
        if (owner < 0) owner = last;                               // a point behind the end: the last element with mass
        if (p.cluster > 1) cluster_sync_all();                     // the sums have been read
        if (owner >= 0 || pass == 1 || a == m) break;
        qrow = nullptr;                                            // nothing is left of p_a - q_a: p_a itself
        certain = -1;
    }

    int *out = p.tokens + (long long)b * (p.n + 1);
    if (rank == 0) {
        for (int t = tid; t <= p.n; t += kVerifyThreads)
            if (t != a || owner < 0) out[t] = t < a ? drafts[t] : -1;
        if (tid == 0) p.accepted[b] = a;
    }
    if (rank != owner || warp != 0) return;
    // the chunk that holds the point, or the last one with mass
    int hit = -1, last = 0;
    for (int c0 = 0; c0 < p.chunks && hit < 0; c0 += 32) {
        const int c = c0 + lane;
        const bool some = c < p.chunks && masses[c] > 0.0;
        const uint32_t there = __ballot_sync(0xffffffffu, some), over = __ballot_sync(0xffffffffu, some && before + sums[c] > point);
        if (there) last = c0 + 31 - __clz(there);
        if (over) hit = c0 + __ffs(over) - 1;
    }
    const int c = hit >= 0 ? hit : last;
    double upto = before + (c ? sums[c - 1] : 0.0);
    long long token = -1;
    constexpr int kRows = 8;
    bool found = false;
    for (int part = 0; part < p.chunk && !found; part += 32 * kRows) {
        const long long from = ((long long)rank * p.chunks + c) * p.chunk + part;
        T pv[kRows], qv[kRows];
        verify_load<1>(prow, qrow, from, p.vocab, certain, pv, qv);
        double own[kRows], row[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) row[i] = own[i] = mass(pv[i], qv[i]);
        // the sums of eight rows of 32, side by side; then the scan of the one that holds the point, or else the last with mass
        uint32_t there = 0;
#pragma unroll
        for (int i = 0; i < kRows; ++i) there |= (uint32_t)(__ballot_sync(0xffffffffu, own[i] > 0.0) != 0) << i;
#pragma unroll
        for (int d = 16; d; d /= 2)
#pragma unroll
            for (int i = 0; i < kRows; ++i) row[i] += __shfl_xor_sync(0xffffffffu, row[i], d);
        int pick = -1;
        double below = 0.0;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if ((there >> i & 1) && !found) {
                pick = i;
                below = upto;
                found = upto + row[i] > point;
            }
            upto += row[i];
        }
        if (pick < 0) continue;
        double r = 0.0;
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (i == pick) r = own[i];
        double s = r;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const double x = __shfl_up_sync(0xffffffffu, s, d);
            if (lane >= d) s += x;
        }
        const uint32_t some = __ballot_sync(0xffffffffu, r > 0.0), over = __ballot_sync(0xffffffffu, r > 0.0 && below + s > point);
        token = from + pick * 32 + (over ? __ffs(over) - 1 : 31 - __clz(some));
    }
    if (lane == 0) out[a] = (int)token;
}

}  // namespace cudallm
