// Cross attention, backward.  With P = exp(S - lse) and delta = rowsum(dO * O):
//     dP = dO V^T,  dS = P * (dP - delta),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// Two kernels, each with its result stationary in tensor memory, so nothing is added by atomics
// and equal inputs give equal bits: one owns 128 query rows of a head and walks the keys (S, dP,
// dQ: three products per block, and delta on the way), one owns 128 keys of a key head and walks
// the queries of all heads that share it (S^T, dP^T, dV, dK: four).  Seven products where five
// would do with dQ added up through memory in a fixed order, which has not been tried (1.6 GB of additions
// at the size below).
//
// Both run the same roles: 512 threads on the 128 x 128 blocks (a thread is a row and a quarter of the
// columns), a TMA warp, a warp that issues the products, and (keys) a warp that brings the
// queries' lse and delta.  S and P, dP and dS lie over each other in tensor memory; P and dS, 16
// bits each, are the A operand of the second products straight from there.
//
// Bound: the tensor core at DP = 128 (3 and 4 products of 512 clocks per block) with the
// special-function unit (1024 clocks per block) beside it; the exponentials at DP = 64.
// P and dS are rounded to the operands' type: that is what the tensor core multiplies.
//
// Measured (one B200): 2048 x up to 4096, 4 x 16 heads of 128 (526 GFLOP in five products): 630-650 us
// = 0.81-0.83 PFLOP/s in short bursts, that is 1.13-1.17 PFLOP/s of the seven that are executed, 0.70 of cuBLAS's burst
// rate; over seconds, at the power cap, 723-740 us = 0.72-0.74 of cuBLAS's sustained rate.  Neither shorter chains (a quarter to a
// half of the exponentials by polynomial) nor more warps changed it by more than 2 %.  The same with heads of 64, all
// 4096 states: 631 us = 0.54 PFLOP/s, bound by the exponentials.  A block takes about 2400
// clocks (dQ) and 3000 (dK, dV).
#pragma once
#include "xattn_common.cuh"

namespace cudallm {

constexpr int kXaBwdThreads = 608;             // 16 warps on the blocks, TMA, products, lse / delta
constexpr int kXaBwdWorkers = 512;

struct XaBwdParams {
    const void *o, *d_o;
    void *dq, *dk, *dv;
    const float *lse;
    float *delta;               // [batch][q_heads][q_rows]
    const int *lens;
    XaStrides sq, sk, sv, so;
    int q_rows, kv_rows, q_heads, kv_heads, group, batch, head_dim;
    int q_tiles, kv_tiles;      // of 128 rows
    // Where one kernel's CTAs are too few to fill the GPU, the axis that they walk is cut into parts
    // (gridDim.y), whose fp32 results are added in order by xattn_grad_join_kernel.
    float *dq_part;             // [part][batch][q_heads][q_rows][head_dim], or NULL: one part
    float *dk_part, *dv_part;   // [part][batch][kv_heads][kv_rows][head_dim], or NULL
    int dq_blocks, dkv_blocks;  // blocks per part
    float scale, scale_log2;
    int *status;
    int skip_loads;
    unsigned long long wait_limit_ns;
};

// Shared memory: the two stationary tiles, a ring of three tiles (the operand that serves two
// products: K or Q), a ring of two (V or dO), lse and delta of two blocks.
template <int DP> struct XaBwdSmem {
    static constexpr int kTile = DP / 64 * kXaChunkBytes;
    static constexpr int kLong = 3, kShort = 2;
    static constexpr int kRingL = 2 * kTile, kRingS = kRingL + kLong * kTile;
    static constexpr int kRows = kRingS + kShort * kTile;          // floats: [2][lse 128, delta 128]
    static constexpr int kBars = kRows + 2 * 2 * kXaRows * 4;
    static constexpr int kNumBars = 24;
    static constexpr int kMisc = kBars + kNumBars * 8;
    static constexpr int kBytes = kMisc + 16;
};
static_assert(XaBwdSmem<128>::kBytes <= 232448, "shared memory budget");
static_assert(XaBwdSmem<64>::kBytes > 114 * 1024, "one CTA per SM (each takes all of tensor memory)");

// Barriers, 8 bytes each from XaBwdSmem::kBars.
enum : int { kBwStat = 0, kBwS = 1 /* 2 */, kBwDp = 3, kBwP = 4, kBwDs = 5, kBwDone = 6, kBwLFull = 7 /* 3 */,
             kBwLEmpty = 10 /* 3 */, kBwSFull = 13 /* 2 */, kBwSEmpty = 15 /* 2 */, kBwRowsFull = 17 /* 2 */,
             kBwRowsEmpty = 19 /* 2 */, kBwDrain = 21 };

// The TMA warp of both kernels: the stationary tiles, then `n` pairs of tiles.  coords(i, h, row) gives
// the head and first row of pair i.  Returns false if a wait ran out; `nl` and `ns`: tiles asked for in each ring.
template <int DP, typename Coords>
__device__ __forceinline__ bool xa_bwd_load(uint32_t sbase, const CUtensorMap *stat_a, const CUtensorMap *stat_b, int stat_h,
                                            int stat_row, const CUtensorMap *ring_l, const CUtensorMap *ring_s, int b, int n,
                                            Coords coords, volatile int *abort_flag, unsigned long long limit, int &nl,
                                            int &ns)
{
    using L = XaBwdSmem<DP>;
    const uint32_t bars = sbase + L::kBars;
    mbar_expect_tx(bars + 8 * kBwStat, 2 * L::kTile);
    xa_load_tile<DP>(stat_a, sbase, bars + 8 * kBwStat, stat_h, stat_row, b);
    xa_load_tile<DP>(stat_b, sbase + L::kTile, bars + 8 * kBwStat, stat_h, stat_row, b);
    bool ok = true;
    for (int i = 0; i < n && ok; ++i) {
        int h, row;
        coords(i, h, row);
        const int sl = i % L::kLong, ss = i % L::kShort;
        if (i >= L::kLong) ok = mbar_wait(bars + 8 * (kBwLEmpty + sl), (i / L::kLong - 1) & 1, abort_flag, limit);
        if (!ok) break;
        mbar_expect_tx(bars + 8 * (kBwLFull + sl), L::kTile);
        xa_load_tile<DP>(ring_l, sbase + L::kRingL + sl * L::kTile, bars + 8 * (kBwLFull + sl), h, row, b);
        ++nl;
        if (i >= L::kShort) ok = mbar_wait(bars + 8 * (kBwSEmpty + ss), (i / L::kShort - 1) & 1, abort_flag, limit);
        if (!ok) break;
        mbar_expect_tx(bars + 8 * (kBwSFull + ss), L::kTile);
        xa_load_tile<DP>(ring_s, sbase + L::kRingS + ss * L::kTile, bars + 8 * (kBwSFull + ss), h, row, b);
        ++ns;
    }
    return ok;
}

// By warp 0: one barrier per lane.
template <int DP>
__device__ __forceinline__ void xa_bwd_init(uint32_t bars, int lane, volatile int *abort_flag)
{
    const bool workers = lane == kBwP || lane == kBwDs || lane == kBwRowsEmpty || lane == kBwRowsEmpty + 1;
    if (lane == 0) *abort_flag = 0;
    if (lane < XaBwdSmem<DP>::kNumBars) mbar_init(bars + 8 * lane, workers ? kXaBwdWorkers / 32 : 1);   // (one arrival per warp)
    fence_mbar_init();
}

// End of both kernels, by all threads.  After a failed wait the copies (lane 0 of warp 16 asked for nl and ns tiles)
// and products in flight are waited for; then tensor memory is released by warp 17.
template <int DP>
__device__ __forceinline__ void xa_bwd_finish(uint32_t bars, uint32_t tmem, volatile int *abort_flag, int nl, int ns)
{
    using L = XaBwdSmem<DP>;
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag && nl > 0) {
        volatile int never = 0;
        mbar_wait(bars + 8 * kBwStat, 0, &never);
        xa_ring_landed<L::kLong>(bars + 8 * kBwLFull, nl, &never);
        xa_ring_landed<L::kShort>(bars + 8 * kBwSFull, ns, &never);
    }
    if (threadIdx.x >> 5 == 17) {
        tc_fence_after();
        if (*abort_flag) xa_products_done(bars + 8 * kBwDrain);
        tmem_dealloc(tmem, 512);
    }
}

// Columns [col, end) of a row of zeros.
template <typename T>
__device__ __forceinline__ void xa_bwd_zero(T *row, int col, int end)
{
    for (; col < end; col += 16 / (int)sizeof(T)) *reinterpret_cast<uint4 *>(row + col) = make_uint4(0, 0, 0, 0);
}

// ---------------------------------------------------------------- dQ --
// Tensor memory: S of even and odd blocks at 0 and 128 (dS over them), dP at 256, dQ at 384.
// When a block's dS is there, three products follow: dP of the next block, this block's part of
// dQ, and S of the block after next, into the place that dS leaves.
template <int DP, typename T>
__global__ void __launch_bounds__(kXaBwdThreads, 1)
xattn_dq_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_do, const XaBwdParams p)
{
    using L = XaBwdSmem<DP>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sbase = smem_u32(smem), bars = sbase + L::kBars;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + L::kMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L::kMisc + 4);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int qt = blockIdx.x % p.q_tiles, bh = blockIdx.x / p.q_tiles;
    const int h = bh % p.q_heads, b = bh / p.q_heads, kvh = h / p.group;
    const int row0 = qt * kXaRows;

    if (warp == 0) xa_bwd_init<DP>(bars, lane, abort_flag);
    if (warp == 17) {
        tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_launch_dependents();
    grid_dependency_wait();
    const int keys = xa_keys(p.lens, b, p.kv_rows);
    const int blk0 = blockIdx.y * p.dq_blocks;                       // (the first of this part's blocks)
    const int nblk = min(p.dq_blocks, (keys + kXaRows - 1) / kXaRows - blk0);
    const unsigned long long limit = p.wait_limit_ns;
    int nl = 0, ns = 0;

    if (warp == 16) {
        if (lane == 0 && nblk > 0 && !p.skip_loads) {
            const bool ok = xa_bwd_load<DP>(sbase, &tm_q, &tm_do, h, row0, &tm_k, &tm_v, b, nblk,
                                            [&](int i, int &hh, int &row) { hh = kvh; row = (blk0 + i) * kXaRows; }, abort_flag, limit, nl, ns);
            if (!ok) xa_report(p.status, kXaRoleDq, 1);
        }
    } else if (warp == 17) {
        if (nblk > 0) {
            constexpr uint32_t idesc_s = xa_idesc<T>(128, 0), idesc_o = xa_idesc<T>(DP, 1);
            const uint32_t t0 = __shfl_sync(0xffffffffu, tmem, 0), s0 = sbase, bar0 = s0 + L::kBars;
            auto wait = [&](int bar, int parity) {
                return __all_sync(0xffffffffu, mbar_wait(bar0 + 8 * bar, parity & 1, abort_flag, limit)) != 0;
            };
            auto k_tile = [&](int i) { return s0 + L::kRingL + (i % L::kLong) * L::kTile; };
            auto wait_k = [&](int i) { return wait(kBwLFull + i % L::kLong, i / L::kLong); };
            auto wait_v = [&](int i) { return wait(kBwSFull + i % L::kShort, i / L::kShort); };
            auto issue_s = [&](int i) {                                  // (by one lane, like the next)
                xa_product_nt<DP>(t0 + (i & 1) * 128, s0, k_tile(i), idesc_s);
                umma_commit(bar0 + 8 * (kBwS + (i & 1)));
            };
            auto issue_dp = [&](int i) {
                const int ss = i % L::kShort;
                xa_product_nt<DP>(t0 + 256, s0 + L::kTile, s0 + L::kRingS + ss * L::kTile, idesc_s);
                umma_commit(bar0 + 8 * kBwDp);
                umma_commit(bar0 + 8 * (kBwSEmpty + ss));
            };
            bool ok = wait(kBwStat, 0) && wait_k(0) && wait_v(0) && (nblk < 2 || wait_k(1));
            if (ok) {
                tc_fence_after();
                if (elect_one()) {
                    issue_s(0);
                    issue_dp(0);
                    if (nblk > 1) issue_s(1);
                }
                __syncwarp();
            }
            for (int i = 0; i < nblk && ok; ++i) {
                ok = (i + 1 >= nblk || wait_v(i + 1)) && wait(kBwDs, i);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    if (i + 1 < nblk) issue_dp(i + 1);
                    xa_product_tn<2, 32>(t0 + 384, t0 + (i & 1) * 128, k_tile(i), idesc_o, i > 0);
                    umma_commit(bar0 + 8 * (kBwLEmpty + i % L::kLong));
                    if (i + 1 == nblk) umma_commit(bar0 + 8 * kBwDone);
                }
                __syncwarp();
                if (i + 2 < nblk) {
                    ok = wait_k(i + 2);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) issue_s(i + 2);
                    __syncwarp();
                }
            }
            if (!ok && lane == 0) xa_report(p.status, kXaRoleDq, 2);
        }
    } else if (warp < 16) {
        const int quarter = warp >> 2, t = (warp & 3) * 32 + lane;        // 32 columns of the block; its row
        const uint32_t t_lane = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const int row = row0 + t;
        const bool live = row < p.q_rows;
        const long long bhr = (long long)bh * p.q_rows + row;
        // delta = rowsum(dO * O): DP / 8 neighbouring lanes a row (16 bytes each), the sums by way of shared memory
        float *delta_s = reinterpret_cast<float *>(smem + L::kRows);
        {
            constexpr int kLanes = DP / 8;
            const int piece = lane % kLanes;
#pragma unroll
            for (int k = 0; k < 8 * kLanes / 32; ++k) {
                const int r = warp * 8 + k * (32 / kLanes) + lane / kLanes;
                float part = 0.f;
                if (row0 + r < p.q_rows && piece * 8 < p.head_dim) {
                    const long long at = b * p.so.b + (row0 + r) * p.so.r + h * p.so.h + piece * 8;
                    const uint4 ov = *reinterpret_cast<const uint4 *>(static_cast<const T *>(p.o) + at);
                    const uint4 gv = *reinterpret_cast<const uint4 *>(static_cast<const T *>(p.d_o) + at);
                    const T *oe = reinterpret_cast<const T *>(&ov), *ge = reinterpret_cast<const T *>(&gv);
#pragma unroll
                    for (int e = 0; e < 8; ++e) part = fmaf(float(oe[e]), float(ge[e]), part);
                }
#pragma unroll
                for (int o = kLanes / 2; o; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
                if (piece == 0) delta_s[r] = part;
            }
        }
        named_bar_sync(1, kXaBwdWorkers);
        const float delta = delta_s[t];
        if (live && quarter == 0 && blockIdx.y == 0) p.delta[bhr] = delta;
        const float lse2 = live ? p.lse[bhr] * 1.4426950408889634f : INFINITY;      // rows that do not exist: P = 0
        bool ok = true;
        for (int i = 0; i < nblk; ++i) {
            ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * (kBwS + (i & 1)), (i >> 1) & 1, abort_flag, limit));
            if (!ok) break;
            tc_fence_after();
            const uint32_t t_s = tmem + (i & 1) * 128 + quarter * 32 + t_lane, t_dp = tmem + 256 + quarter * 32 + t_lane;
            const int valid = keys - (blk0 + i) * kXaRows - quarter * 32;        // of this thread's 32 columns
            uint32_t s[32], r[32], w[16];
            tmem_ld_32x32b_x32(t_s, s);
            tmem_ld_wait_for(s);
#pragma unroll
            for (int k = 0; k < 32; ++k)
                s[k] = __float_as_uint(xa_exp2(fmaf(__uint_as_float(s[k]), p.scale_log2, -lse2)));
            ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * kBwDp, i & 1, abort_flag, limit));
            if (!ok) break;
            tc_fence_after();
            if (quarter == 0 && keys - (blk0 + i) * kXaRows < kXaRows && keys < p.kv_rows) {
                if (t >= keys - (blk0 + i) * kXaRows) xa_zero_row<DP>(sbase + L::kRingL + (i % L::kLong) * L::kTile, t);
                fence_proxy_async_smem();
            }
            tmem_ld_32x32b_x32(t_dp, r);
            tmem_ld_wait_for(r);
#pragma unroll
            for (int k = 0; k < 32; ++k) r[k] = __float_as_uint(__uint_as_float(s[k]) * (__uint_as_float(r[k]) - delta));
            if (valid < 32) {
#pragma unroll
                for (int k = 0; k < 32; ++k)
                    if (k >= valid) r[k] = 0;
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) w[k] = XaElem<T>::pack(__uint_as_float(r[2 * k]), __uint_as_float(r[2 * k + 1]));
            tmem_st_32x32b_x16(t_s, w);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 8 * kBwDs);
        }
        if (ok && nblk > 0) ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * kBwDone, 0, abort_flag, limit));
        if (ok) {
            // this warp's rows, 32 columns, staged where the tiles were
            const int first = row0 + (warp & 3) * 32, rows = p.q_rows - first, col = quarter * 32, left = p.head_dim - col;
            const uint32_t stage = sbase + warp * 4096, t_dq = tmem + 384 + t_lane + col;
            float *part = p.dq_part + ((long long)blockIdx.y * p.batch * p.q_heads * p.q_rows + (long long)bh * p.q_rows + first) * p.head_dim;
            T *dst = static_cast<T *>(p.dq) + b * p.sq.b + first * p.sq.r + h * p.sq.h;
            if (nblk > 0 && col < DP) {
                tc_fence_after();
                if (p.dq_part) xa_store_part<32>(t_dq, stage, lane, 1.f, part + col, p.head_dim, rows, left);
                else xa_store_result<32, T>(t_dq, stage, lane, p.scale, dst + col, p.sq.r, rows, left);
            } else if (nblk <= 0 && live) {
                const int end = min(col + 32, p.head_dim);
                if (p.dq_part) xa_bwd_zero(part + lane * p.head_dim, col, end);
                else xa_bwd_zero(dst + lane * p.sq.r, col, end);
            }
        } else if (lane == 0) {
            xa_report(p.status, kXaRoleDq, 3);
        }
    }
    xa_bwd_finish<DP>(bars, tmem, abort_flag, nl, ns);
}

// ------------------------------------------------------------- dK, dV --
// Tensor memory: S^T at 0 (P^T over it), dP^T at 128 (dS^T over it), dV at 256, dK at 384.  While
// the exponentials of a block run, the tensor core adds the last block's dK and computes dP^T;
// while dS^T is formed, it adds dV and computes the next S^T.
template <int DP, typename T>
__global__ void __launch_bounds__(kXaBwdThreads, 1)
xattn_dkv_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                 const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_do, const XaBwdParams p)
{
    using L = XaBwdSmem<DP>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sbase = smem_u32(smem), bars = sbase + L::kBars;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + L::kMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L::kMisc + 4);
    float *rows_buf = reinterpret_cast<float *>(smem + L::kRows);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int kt = blockIdx.x % p.kv_tiles, bk = blockIdx.x / p.kv_tiles;
    const int kvh = bk % p.kv_heads, b = bk / p.kv_heads;
    const int key0 = kt * kXaRows;

    if (warp == 0) xa_bwd_init<DP>(bars, lane, abort_flag);
    if (warp == 17) {
        tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_launch_dependents();
    grid_dependency_wait();
    const int keys = xa_keys(p.lens, b, p.kv_rows);
    // block i: head i / q_tiles of the group; blk0: the first of this part's blocks
    const int blk0 = blockIdx.y * p.dkv_blocks;
    const int nblk = key0 < keys ? min(p.dkv_blocks, p.group * p.q_tiles - blk0) : 0;
    const unsigned long long limit = p.wait_limit_ns;
    int nl = 0, ns = 0;

    if (warp == 16) {
        if (lane == 0 && nblk > 0 && !p.skip_loads) {
            const bool ok = xa_bwd_load<DP>(sbase, &tm_k, &tm_v, kvh, key0, &tm_q, &tm_do, b, nblk,
                                            [&](int i, int &hh, int &row) {
                                                hh = kvh * p.group + (blk0 + i) / p.q_tiles;
                                                row = ((blk0 + i) % p.q_tiles) * kXaRows;
                                            }, abort_flag, limit, nl, ns);
            if (!ok) xa_report(p.status, kXaRoleDkv, 1);
        }
    } else if (warp == 17) {
        if (nblk > 0) {
            constexpr uint32_t idesc_s = xa_idesc<T>(128, 0), idesc_o = xa_idesc<T>(DP, 1);
            const uint32_t t0 = __shfl_sync(0xffffffffu, tmem, 0), s0 = sbase, bar0 = s0 + L::kBars;
            auto wait = [&](int bar, int parity) {
                return __all_sync(0xffffffffu, mbar_wait(bar0 + 8 * bar, parity & 1, abort_flag, limit)) != 0;
            };
            auto q_tile = [&](int i) { return s0 + L::kRingL + (i % L::kLong) * L::kTile; };
            auto do_tile = [&](int i) { return s0 + L::kRingS + (i % L::kShort) * L::kTile; };
            auto wait_q = [&](int i) { return wait(kBwLFull + i % L::kLong, i / L::kLong); };
            auto wait_do = [&](int i) { return wait(kBwSFull + i % L::kShort, i / L::kShort); };
            auto issue_s = [&](int i) {                                  // (by one lane, like the next)
                xa_product_nt<DP>(t0, s0, q_tile(i), idesc_s);
                umma_commit(bar0 + 8 * kBwS);
            };
            auto issue_dp = [&](int i) {
                xa_product_nt<DP>(t0 + 128, s0 + L::kTile, do_tile(i), idesc_s);
                umma_commit(bar0 + 8 * kBwDp);
            };
            bool ok = wait(kBwStat, 0) && wait_q(0) && wait_do(0);
            if (ok) {
                tc_fence_after();
                if (elect_one()) {
                    issue_s(0);
                    issue_dp(0);
                }
                __syncwarp();
            }
            for (int i = 0; i < nblk && ok; ++i) {
                const bool more = i + 1 < nblk;
                ok = (!more || wait_q(i + 1)) && wait(kBwP, i);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    xa_product_tn<2, 32>(t0 + 256, t0, do_tile(i), idesc_o, i > 0);
                    umma_commit(bar0 + 8 * (kBwSEmpty + i % L::kShort));
                    if (more) issue_s(i + 1);
                }
                __syncwarp();
                ok = (!more || wait_do(i + 1)) && wait(kBwDs, i);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    xa_product_tn<2, 32>(t0 + 384, t0 + 128, q_tile(i), idesc_o, i > 0);
                    umma_commit(bar0 + 8 * (kBwLEmpty + i % L::kLong));
                    if (more) issue_dp(i + 1);
                    else umma_commit(bar0 + 8 * kBwDone);
                }
                __syncwarp();
            }
            if (!ok && lane == 0) xa_report(p.status, kXaRoleDkv, 2);
        }
    } else if (warp == 18) {
        // lse (in units of log2) and delta of each block's queries; a query that does not exist has P = 0
        bool ok = true;
        for (int i = 0; i < nblk && ok; ++i) {
            const int j = i & 1;
            if (i >= 2) ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * (kBwRowsEmpty + j), ((i >> 1) - 1) & 1, abort_flag, limit));
            if (!ok) break;
            const int row0 = ((blk0 + i) % p.q_tiles) * kXaRows;
            const long long base = ((long long)b * p.q_heads + kvh * p.group + (blk0 + i) / p.q_tiles) * p.q_rows;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int r = lane + 32 * u, row = row0 + r;
                rows_buf[j * 256 + r] = row < p.q_rows ? p.lse[base + row] * 1.4426950408889634f : INFINITY;
                rows_buf[j * 256 + 128 + r] = row < p.q_rows ? p.delta[base + row] : 0.f;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 8 * (kBwRowsFull + j));
        }
    } else {
        const int quarter = warp >> 2;                               // 32 columns (queries) of the block
        const uint32_t t_lane = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + quarter * 32 + t_lane, t_dp = tmem + 128 + quarter * 32 + t_lane;
        bool ok = true;
        for (int i = 0; i < nblk; ++i) {
            const int j = i & 1;
            const float4 *lse4 = reinterpret_cast<const float4 *>(rows_buf + j * 256 + quarter * 32);
            const float4 *delta4 = lse4 + 32;
            ok = mbar_wait(bars + 8 * (kBwRowsFull + j), (i >> 1) & 1, abort_flag, limit)
                 && mbar_wait(bars + 8 * kBwS, i & 1, abort_flag, limit);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            uint32_t s[32], w[16];
            tmem_ld_32x32b_x32(t_s, s);
            tmem_ld_wait_for(s);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float4 l4 = lse4[k];
                const float e0 = xa_exp2(fmaf(__uint_as_float(s[4 * k]), p.scale_log2, -l4.x));
                const float e1 = xa_exp2(fmaf(__uint_as_float(s[4 * k + 1]), p.scale_log2, -l4.y));
                const float e2 = xa_exp2(fmaf(__uint_as_float(s[4 * k + 2]), p.scale_log2, -l4.z));
                const float e3 = xa_exp2(fmaf(__uint_as_float(s[4 * k + 3]), p.scale_log2, -l4.w));
                s[4 * k] = __float_as_uint(e0);
                s[4 * k + 1] = __float_as_uint(e1);
                s[4 * k + 2] = __float_as_uint(e2);
                s[4 * k + 3] = __float_as_uint(e3);
                w[2 * k] = XaElem<T>::pack(e0, e1);
                w[2 * k + 1] = XaElem<T>::pack(e2, e3);
            }
            tmem_st_32x32b_x16(t_s, w);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 8 * kBwP);
            ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * kBwDp, i & 1, abort_flag, limit));
            if (!ok) break;
            tc_fence_after();
            uint32_t r[32];
            tmem_ld_32x32b_x32(t_dp, r);
            tmem_ld_wait_for(r);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float4 d4 = delta4[k];
                w[2 * k] = XaElem<T>::pack(__uint_as_float(s[4 * k]) * (__uint_as_float(r[4 * k]) - d4.x),
                                           __uint_as_float(s[4 * k + 1]) * (__uint_as_float(r[4 * k + 1]) - d4.y));
                w[2 * k + 1] = XaElem<T>::pack(__uint_as_float(s[4 * k + 2]) * (__uint_as_float(r[4 * k + 2]) - d4.z),
                                               __uint_as_float(s[4 * k + 3]) * (__uint_as_float(r[4 * k + 3]) - d4.w));
            }
            tmem_st_32x32b_x16(t_dp, w);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(bars + 8 * (kBwRowsEmpty + j));
                mbar_arrive(bars + 8 * kBwDs);
            }
        }
        if (ok && nblk > 0) ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * kBwDone, 0, abort_flag, limit));
        if (ok) {
            // this warp's states: half of the columns of dV (quarters 0, 1) or of dK, staged where the tiles were;
            // rows from `keys` on are padding, and get no gradient
            const bool is_k = quarter >= 2;
            const int first = key0 + (warp & 3) * 32, rows = keys - first, col = (quarter & 1) * (DP / 2), left = p.head_dim - col;
            const uint32_t stage = sbase + warp * 4096, t_g = tmem + (is_k ? 384 : 256) + t_lane + col;
            const long long at = (((long long)blockIdx.y * p.batch * p.kv_heads + bk) * p.kv_rows + first) * p.head_dim;
            float *part = (is_k ? p.dk_part : p.dv_part) + at;
            const XaStrides st = is_k ? p.sk : p.sv;
            T *dst = static_cast<T *>(is_k ? p.dk : p.dv) + b * st.b + first * st.r + kvh * st.h;
            if (nblk > 0) {
                tc_fence_after();
                if (p.dk_part) xa_store_part<DP / 2>(t_g, stage, lane, 1.f, part + col, p.head_dim, rows, left);
                else xa_store_result<DP / 2, T>(t_g, stage, lane, is_k ? p.scale : 1.f, dst + col, st.r, rows, left);
            }
            if (first + lane < p.kv_rows && (lane >= rows || nblk <= 0)) {
                const int end = min(col + DP / 2, p.head_dim);
                if (p.dk_part) xa_bwd_zero(part + lane * p.head_dim, col, end);
                else xa_bwd_zero(dst + lane * st.r, col, end);
            }
        } else if (lane == 0) {
            xa_report(p.status, kXaRoleDkv, 3);
        }
    }
    xa_bwd_finish<DP>(bars, tmem, abort_flag, nl, ns);
}

// Adds the parts of one or two gradients in order and rounds the sums, times f0 and f1.  A thread takes four
// columns of a row.
struct XaGradJoinParams {
    const float *part[2];
    void *out[2];
    XaStrides st[2];
    float f[2];
    int parts, rows, heads, head_dim;
    long long rows_all;             // batch * heads * rows
};
template <typename T>
__global__ void __launch_bounds__(256)
xattn_grad_join_kernel(const XaGradJoinParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const int per_row = p.head_dim / 4, a = blockIdx.y;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.rows_all * per_row) return;
    const long long row = i / per_row;
    const int col = (int)(i % per_row) * 4;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < p.parts; ++s) {
        const float4 v = *reinterpret_cast<const float4 *>(p.part[a] + (s * p.rows_all + row) * p.head_dim + col);
        sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
    }
    const float f = p.f[a];
    const long long r = row % p.rows, bh = row / p.rows, h = bh % p.heads, b = bh / p.heads;
    *reinterpret_cast<uint2 *>(static_cast<T *>(p.out[a]) + b * p.st[a].b + r * p.st[a].r + h * p.st[a].h + col) =
        make_uint2(XaElem<T>::pack(sum.x * f, sum.y * f), XaElem<T>::pack(sum.z * f, sum.w * f));
}

}  // namespace cudallm
