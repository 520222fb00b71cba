// Cross attention, forward: O = softmax(scale Q K^T) V per head, keys from kv_len on masked.
//
// A CTA owns two tiles of 128 query rows of one head and walks the keys in blocks of 128.
//   warps 0-15      softmax: eight warps per tile; a row is a lane of tensor memory, its 128 scores
//                   are shared by two threads (of warps w and w + 4) with 64 in registers each
//   warp 16         TMA: the queries once, then K and V tiles through a ring
//   warp 17         the tensor core: S = Q K^T into tensor memory, O += P V with P read from tensor
//                   memory
// While one tile's softmax runs, the tensor core works for the other.  One pass over the keys: the
// row's reference maximum is only moved (and O rescaled in tensor memory) when a block's maximum
// passes it by more than 2^8, since any reference gives the same quotient; probabilities stay
// below 2^8, far inside every type's range.
//
// Bound: at DP = 128 the chain softmax -> P V -> next S of a tile, which only the other tile's
// chain covers: tensor memory (S 2 x 128 columns, O 2 x 128) has no room for a second S, and P lies
// over S (with P in shared memory the next S could start earlier: not tried).  At DP = 64 P has columns of its own, the next S starts as soon as this one is in
// registers, and the special-function unit (16 exponentials per clock) is the bound; the tiles take
// turns at it, since together they would also leave it together (66 instead of 58 us below).
//
// Measured (one B200): 2048 queries x up to 4096 states, 4 x 16 heads of 128, lengths 3/8 to 1 (210
// GFLOP): 185-207 us = 1.02-1.14 PFLOP/s, 0.62-0.69 of the measured cuBLAS burst, at the power cap when
// it runs for seconds (217 us).  512 x 4096, 74 heads of 64: 58 us = 0.69 PFLOP/s.
// Tried and not kept: 5 to 8 of 16 exponentials by polynomial on the FMA pipe (221 to 236 us when the kernel
// without them took 213 to 217); blocks of 64 keys with two places for S (254 us: with N = 64 a product
// is bound by reading the queries from shared memory, 48 clocks instead of 32); exponentials before the
// halves of a row have exchanged their maxima (198 to 210 us instead of 198 at DP = 128, 73 at 64).
#pragma once
#include "xattn_common.cuh"

namespace cudallm {

constexpr int kXaFwdThreads = 576;

struct XaFwdParams {
    void *o;
    float *lse;                 // [batch][q_heads][q_rows], or NULL
    float *o_part, *lse_part;   // splits > 1: [split][batch][q_heads][q_rows]([head_dim]) partial results
    const int *lens;
    XaStrides so;
    int q_rows, kv_rows, q_heads, group, batch, head_dim;
    int q_tiles;                // pairs of query tiles per head
    int splits, tiles_per_split;
    float scale, scale_log2;    // scale, and scale * log2(e)
    int *status;
    int skip_loads;             // self-test of the bounded waits: nothing is loaded, every wait runs out
    unsigned long long wait_limit_ns;
};

__device__ __forceinline__ float xa_max32(const uint32_t (&r)[32])
{
    float m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = max3_nan(__uint_as_float(r[i]), __uint_as_float(r[i + 4]), __uint_as_float(r[i + 8]));
#pragma unroll
    for (int k = 12; k < 28; k += 8)
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = max3_nan(m[i], __uint_as_float(r[k + i]), __uint_as_float(r[k + 4 + i]));
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = max3_nan(m[i], __uint_as_float(r[28 + i]), __uint_as_float(r[28 + i]));
    return max3_nan(max3_nan(m[0], m[1], m[2]), m[3], m[3]);
}

template <int DP> struct XaFwdSmem {
    static constexpr int kTile = DP / 64 * kXaChunkBytes;
    static constexpr int kStages = DP == 128 ? 4 : 7;
    static constexpr int kRing = 2 * kTile;
    static constexpr int kBars = kRing + kStages * kTile;
    // q_full, s_full[2], p_full[2], pv_done[2], s_read[2], p_half[2], turn[2], full[kStages], empty[kStages], drain
    static constexpr int kNumBars = 14 + 2 * kStages;
    static constexpr int kMisc = kBars + kNumBars * 8;
    static constexpr int kXch = kMisc + 16 + 8 * (kNumBars & 1);   // floats: [tile][parity][half][row]
    // 4 KiB per softmax warp for the output's rows: where the queries were (two tiles of 32 KiB), or behind
    static constexpr int kEnd = kXch + 2 * 2 * 2 * kXaRows * 4;
    static constexpr int kStore = DP == 128 ? 0 : (kEnd + 127) / 128 * 128;
    static constexpr int kBytes = DP == 128 ? kEnd : kStore + 16 * 4096;
    // tensor memory: S of tile j, P of tile j, O of tile j
    static constexpr bool kOwnP = DP == 64;
    static constexpr int kTmemS = 0, kTmemP = kOwnP ? 256 : 0, kStepP = kOwnP ? 64 : 128, kTmemO = kOwnP ? 384 : 256;
};
static_assert(XaFwdSmem<128>::kBytes <= 232448 && XaFwdSmem<64>::kBytes > 114 * 1024, "one CTA per SM");

template <int DP, typename T>
__global__ void __launch_bounds__(kXaFwdThreads, 1)
xattn_fwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                 const __grid_constant__ CUtensorMap tm_v, const XaFwdParams p)
{
    using L = XaFwdSmem<DP>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sbase = smem_u32(smem);
    const uint32_t bars = sbase + L::kBars;
    const uint32_t q_full = bars, s_full = bars + 8, p_full = bars + 24, pv_done = bars + 40, s_read = bars + 56,
                   p_half = bars + 72, turn = bars + 88, full = bars + 104, empty = full + 8 * L::kStages,
                   drain = empty + 8 * L::kStages;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + L::kMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L::kMisc + 4);

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int qt = blockIdx.x % p.q_tiles;
    const int bh = blockIdx.x / p.q_tiles;
    const int h = bh % p.q_heads, b = bh / p.q_heads;
    const int kvh = h / p.group;
    const int row0 = qt * 2 * kXaRows;
    const int tiles = p.q_rows - row0 > kXaRows ? 2 : 1;

    if (tid == 0) *abort_flag = 0;
    if (warp == 0) {
        // one barrier per lane: p_full, s_read, p_half, turn take one arrival per warp of a tile, the others one
        static_assert(L::kNumBars <= 32, "barriers");
        if (lane < L::kNumBars) mbar_init(bars + 8 * lane, (lane == 3 || lane == 4 || (lane >= 7 && lane < 13)) ? 8 : 1);
        fence_mbar_init();
    }
    if (warp == 17) {
        tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // only now: the next kernel of the stream may start once every CTA of this one holds its tensor memory
    grid_launch_dependents();
    grid_dependency_wait();

    const int keys = xa_keys(p.lens, b, p.kv_rows);
    const int key0 = blockIdx.y * p.tiles_per_split * kXaRows;
    const int nkeys = min(p.tiles_per_split * kXaRows, keys - key0);                      // <= 0: no keys here
    const int nblk = (nkeys + kXaRows - 1) / kXaRows;
    int loads = 0;                                                                       // (lane 0 of warp 16: tiles asked for)

    if (warp == 16) {
        if (lane == 0 && nblk > 0 && !p.skip_loads) {
            mbar_expect_tx(q_full, tiles * L::kTile);
            for (int j = 0; j < tiles; ++j) xa_load_tile<DP>(&tm_q, sbase + j * L::kTile, q_full, h, row0 + j * kXaRows, b);
            bool ok = true;
            for (int i = 0; i < nblk && ok; ++i) {
                for (int w = 0; w < 2; ++w) {                             // K, then V
                    const int s = loads % L::kStages, use = loads / L::kStages;
                    if (use > 0) ok = mbar_wait(empty + 8 * s, (use - 1) & 1, abort_flag, p.wait_limit_ns);
                    if (!ok) break;
                    mbar_expect_tx(full + 8 * s, L::kTile);
                    xa_load_tile<DP>(w ? &tm_v : &tm_k, sbase + L::kRing + s * L::kTile, full + 8 * s, kvh,
                                     key0 + i * kXaRows, b);
                    ++loads;
                }
            }
            if (!ok) xa_report(p.status, kXaRoleLoad, 1);
        }
    } else if (warp == 17) {
        if (nblk > 0) {
            constexpr uint32_t idesc_s = xa_idesc<T>(kXaRows, 0), idesc_o = xa_idesc<T>(DP, 1);
            const uint32_t t0 = __shfl_sync(0xffffffffu, tmem, 0), s0 = sbase, ring = s0 + L::kRing;
            const uint32_t b0 = s0 + L::kBars, b_s = b0 + 8, b_p = b0 + 24, b_pv = b0 + 40, b_read = b0 + 56, b_half = b0 + 72, b_full = b0 + 104,
                           b_empty = b_full + 8 * L::kStages;
            auto wait = [&](uint32_t bar, int parity) {
                return __all_sync(0xffffffffu, mbar_wait(bar, parity & 1, abort_flag, p.wait_limit_ns)) != 0;
            };
            // ring position of K of block i: 2 i, of V: 2 i + 1
            auto stage = [&](int pos) { return pos % L::kStages; };
            auto wait_tile = [&](int pos) { return wait(b_full + 8 * stage(pos), pos / L::kStages); };
            auto tile_at = [&](int pos) { return ring + stage(pos) * L::kTile; };
            auto issue_s = [&](int j, int i) {                            // (by one lane, like the next)
                xa_product_nt<DP>(t0 + L::kTmemS + 128 * j, s0 + j * L::kTile, tile_at(2 * i), idesc_s);
                umma_commit(b_s + 8 * j);
                if (j + 1 == tiles) umma_commit(b_empty + 8 * stage(2 * i));
            };
            auto issue_pv_half = [&](int j, int i) {
                xa_product_tn<4, 64, 1>(t0 + L::kTmemO + DP * j, t0 + L::kTmemP + L::kStepP * j, tile_at(2 * i + 1), idesc_o, i > 0);
            };
            auto issue_pv = [&](int j, int i) {
                if (L::kOwnP)
                    xa_product_tn<4, 32>(t0 + L::kTmemO + DP * j, t0 + L::kTmemP + L::kStepP * j, tile_at(2 * i + 1), idesc_o, i > 0);
                else
                    xa_product_tn<4, 64, 2>(t0 + L::kTmemO + DP * j, t0 + L::kTmemP + L::kStepP * j, tile_at(2 * i + 1), idesc_o, true);
                umma_commit(b_pv + 8 * j);
                if (j + 1 == tiles) umma_commit(b_empty + 8 * stage(2 * i + 1));
            };
            bool ok = wait(b0, 0) && wait_tile(0);
            if (ok) {
                tc_fence_after();
                if (elect_one())
                    for (int j = 0; j < tiles; ++j) issue_s(j, 0);
                __syncwarp();
            }
            for (int i = 0; i < nblk && ok; ++i) {
                const bool more = i + 1 < nblk;
                ok = wait_tile(2 * i + 1) && (!more || wait_tile(2 * i + 2));
                if (L::kOwnP) {
                    // the next scores of each tile as soon as these have been read
                    for (int j = 0; j < tiles && ok && more; ++j) {
                        ok = wait(b_read + 8 * j, i);
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_one()) issue_s(j, i + 1);
                        __syncwarp();
                    }
                }
                for (int j = 0; j < tiles && ok; ++j) {
                    if (!L::kOwnP) {
                        // the first half of P is multiplied while the exponentials of the second run
                        ok = wait(b_half + 8 * j, i);
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_one()) issue_pv_half(j, i);
                        __syncwarp();
                    }
                    ok = wait(b_p + 8 * j, i);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        // (products of one issuing thread run in order: the next S, which overwrites P where
                        // they share their place, starts after this product has read it)
                        issue_pv(j, i);
                        if (!L::kOwnP && more) issue_s(j, i + 1);
                    }
                    __syncwarp();
                }
            }
            if (!ok && lane == 0) xa_report(p.status, kXaRoleMma, 1);
        }
    } else {
        const int j = warp >> 3, half = (warp >> 2) & 1;                 // tile, half of the block's keys
        const int t = (warp & 3) * 32 + lane;                            // row of the tile = lane of tensor memory
        if (j < tiles && nblk > 0) {
            const uint32_t t_lane = static_cast<uint32_t>((warp & 3) * 32) << 16;
            const uint32_t t_s = tmem + L::kTmemS + 128 * j + 64 * half + t_lane, t_o = tmem + L::kTmemO + DP * j + t_lane;
            const uint32_t t_p = tmem + L::kTmemP + L::kStepP * j + (L::kOwnP ? 32 : 64) * half + t_lane;
            float *xch = reinterpret_cast<float *>(smem + L::kXch) + j * 4 * kXaRows;     // [parity][half][row]
            float m = -INFINITY, l = 0.f;
            bool ok = true;
            auto wait = [&](uint32_t bar, int parity) {
                return __all_sync(0xffffffffu, mbar_wait(bar, parity & 1, abort_flag, p.wait_limit_ns)) != 0;
            };
            for (int i = 0; i < nblk; ++i) {
                ok = ok && wait(s_full + 8 * j, i);
                tc_fence_after();
                uint32_t r[2][32];
                float bm = -INFINITY;
                if (ok) {
                    tmem_ld_32x32b_x32(t_s, r[0]);
                    tmem_ld_32x32b_x32(t_s + 32, r[1]);
                    tmem_ld_wait_for(r[0]);
                    tmem_ld_wait_for(r[1]);
                    if (L::kOwnP) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(s_read + 8 * j);
                    }
                    const int valid = nkeys - i * kXaRows;                // keys of this block that exist
                    if (valid < kXaRows) {
#pragma unroll
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if (half * 64 + c * 32 + k >= valid) r[c][k] = 0xFF800000u;         // -inf
                        if (j == 0 && half == 0 && key0 + nkeys < p.kv_rows) {
                            // rows of V that are padding, not beyond the tensor's end
                            const int sv = (2 * i + 1) % L::kStages;
                            ok = wait(full + 8 * sv, (2 * i + 1) / L::kStages);
                            if (ok && t >= valid) xa_zero_row<DP>(sbase + L::kRing + sv * L::kTile, t);
                            fence_proxy_async_smem();
                        }
                    }
                    bm = max3_nan(xa_max32(r[0]), xa_max32(r[1]), -INFINITY);
                }
                // the other half of the row; a wait that failed for one warp ends the loop for all of the
                // tile's, so that none is missing at a later barrier
                xch[((i & 1) * 2 + half) * kXaRows + t] = bm;
                ok = named_bar_all(1 + j, 2 * kXaRows, ok);
                if (!ok) break;
                bm = max3_nan(bm, xch[((i & 1) * 2 + (half ^ 1)) * kXaRows + t], bm);
                const bool move = !((bm - m) * p.scale_log2 <= 8.f);      // (always for the first block, and with a NaN)
                if (i == 0) {
                    m = bm;
                } else if (__any_sync(0xffffffffu, move)) {
                    const float alpha = move ? xa_exp2((m - bm) * p.scale_log2) : 1.f;
                    if (move) m = bm;
                    l *= alpha;
                    // (block i - 2's product is complete: its P was read before block i - 1's was formed)
                    ok = wait(pv_done + 8 * j, i - 1);
                    tc_fence_after();
                    if (ok) {
#pragma unroll
                        for (int c = 0; c < DP / 32; ++c) {               // half of O's columns
                            uint32_t o[16];
                            tmem_ld_32x32b_x16(t_o + half * (DP / 2) + 16 * c, o);
                            tmem_ld_wait_for(o);
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                            tmem_st_32x32b_x16(t_o + half * (DP / 2) + 16 * c, o);
                        }
                    }
                }
                if (L::kOwnP && i > 0) {                                  // the last block's P has been read
                    ok = ok && wait(pv_done + 8 * j, i - 1);
                    tc_fence_after();
                }
                if (L::kOwnP && tiles == 2 && (i > 0 || j > 0)) ok = ok && wait(turn + 8 * j, j ? i : i - 1);
                const float neg = -m * p.scale_log2;
                const uint64_t scale2 = f32x2(p.scale_log2, p.scale_log2), neg2 = f32x2(neg, neg);
                uint64_t sum[2] = {0, 0};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float lo, hi;
                        f32x2_split(f32x2_fma(f32x2(__uint_as_float(r[c][2 * k]), __uint_as_float(r[c][2 * k + 1])), scale2, neg2),
                                    lo, hi);
                        lo = xa_exp2(lo);
                        hi = xa_exp2(hi);
                        sum[k & 1] = f32x2_add(sum[k & 1], f32x2(lo, hi));
                        w[k] = XaElem<T>::pack(lo, hi);
                    }
                    tmem_st_32x32b_x16(t_p + 16 * c, w);                  // (over S it is this thread's own half)
                    if (c == 0) {
                        if (!L::kOwnP) {
                            tmem_st_wait();
                            tc_fence_before();
                        }
                        __syncwarp();
                        if (lane == 0) mbar_arrive(L::kOwnP ? turn + 8 * (j ^ 1) : p_half + 8 * j);
                    }
                }
                float s0, s1;
                f32x2_split(f32x2_add(sum[0], sum[1]), s0, s1);
                l += s0 + s1;
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8 * j);
            }
            // the row's output: the halves' sums join, each thread stores half of the columns
            // (block nblk - 2's product is complete: see above)
            ok = ok && wait(pv_done + 8 * j, nblk - 1);
            xch[((nblk & 1) * 2 + half) * kXaRows + t] = l;
            ok = named_bar_all(1 + j, 2 * kXaRows, ok);
            if (ok) {
                tc_fence_after();
                l += xch[((nblk & 1) * 2 + (half ^ 1)) * kXaRows + t];
                const float inv = 1.f / l;
                const int first = row0 + j * kXaRows + (warp & 3) * 32, rows = p.q_rows - first;    // this warp's rows
                const int col = half * (DP / 2), left = p.head_dim - col;
                const long long bhr = (long long)bh * p.q_rows + first;
                const long long part = (long long)blockIdx.y * p.batch * p.q_heads * p.q_rows + bhr;
                const uint32_t stage = sbase + L::kStore + ((j * 2 + half) * 4 + (warp & 3)) * 4096;
                if (p.splits == 1)
                    xa_store_result<DP / 2, T>(t_o + col, stage, lane, inv,
                                               static_cast<T *>(p.o) + b * p.so.b + first * p.so.r + h * p.so.h + col, p.so.r, rows, left);
                else
                    xa_store_part<DP / 2>(t_o + col, stage, lane, inv, p.o_part + part * p.head_dim + col, p.head_dim, rows, left);
                if (lane < rows && half == 0) {
                    const float lse = fmaf(m, p.scale, logf(l));
                    if (p.splits > 1) p.lse_part[part + lane] = lse;
                    else if (p.lse) p.lse[bhr + lane] = lse;
                }
            } else if (lane == 0) {
                xa_report(p.status, kXaRoleSoftmax, 1);
            }
        } else if (j < tiles) {
            // no keys: the output is zero, the sum of no exponentials is zero
            const int row = row0 + j * kXaRows + t;
            if (row < p.q_rows && half == 0) {
                const long long bhr = (long long)bh * p.q_rows + row;
                if (p.splits > 1) {
                    p.lse_part[(long long)blockIdx.y * p.batch * p.q_heads * p.q_rows + bhr] = -INFINITY;
                } else {
                    T *dst = static_cast<T *>(p.o) + b * p.so.b + row * p.so.r + h * p.so.h;
                    for (int c = 0; c < p.head_dim; c += 8) *reinterpret_cast<uint4 *>(dst + c) = make_uint4(0, 0, 0, 0);
                    if (p.lse) p.lse[bhr] = -INFINITY;
                }
            }
        }
    }
    __syncwarp();
    // All copies and products have been waited for (pv_done), or a wait ran out.  Then those in flight are waited for
    // here, whichever role gave up and when, before shared and tensor memory are another CTA's.
    tc_fence_before();
    __syncthreads();
    if (*abort_flag && warp == 16 && lane == 0 && loads > 0) {
        volatile int never = 0;
        mbar_wait(q_full, 0, &never);
        xa_ring_landed<L::kStages>(full, loads, &never);
    }
    if (warp == 17) {
        tc_fence_after();
        if (*abort_flag) xa_products_done(drain);
        tmem_dealloc(tmem, 512);
    }
}

// Joins the partial results of `splits` parts of the keys: weights exp(lse_s - lse), a part without
// keys (lse = -inf) is not read.  One warp per row.
struct XaJoinParams {
    const float *o_part, *lse_part;
    void *o;
    float *lse;
    XaStrides so;
    int q_rows, q_heads, head_dim, splits;
    long long rows_all;
};
template <typename T>
__global__ void __launch_bounds__(256)
xattn_join_kernel(const XaJoinParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (row >= p.rows_all) return;
    const int r = (int)(row % p.q_rows);
    const int h = (int)(row / p.q_rows % p.q_heads), b = (int)(row / p.q_rows / p.q_heads);
    const float part = lane < p.splits ? p.lse_part[lane * p.rows_all + row] : -INFINITY;
    float mx = part;
#pragma unroll
    for (int o = 16; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    // (-inf and NaN scores: a NaN part must make the row NaN)
    float w = part == -INFINITY ? 0.f : expf(part - mx), sum = w;
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float inv = mx == -INFINITY && sum == 0.f ? 0.f : 1.f / sum;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const int col = lane * 4;
    for (int s = 0; s < p.splits; ++s) {
        // (a weight that has vanished still multiplies: 0 x inf must make the row NaN, as it does in one part)
        const float ws = __shfl_sync(0xffffffffu, w, s) * inv;
        const bool keys = __shfl_sync(0xffffffffu, part, s) != -INFINITY;
        if (!keys || col >= p.head_dim) continue;
        const float4 v = *reinterpret_cast<const float4 *>(p.o_part + (s * p.rows_all + row) * p.head_dim + col);
        acc.x = fmaf(ws, v.x, acc.x);
        acc.y = fmaf(ws, v.y, acc.y);
        acc.z = fmaf(ws, v.z, acc.z);
        acc.w = fmaf(ws, v.w, acc.w);
    }
    if (col < p.head_dim)
        *reinterpret_cast<uint2 *>(static_cast<T *>(p.o) + b * p.so.b + r * p.so.r + h * p.so.h + col) =
            make_uint2(XaElem<T>::pack(acc.x, acc.y), XaElem<T>::pack(acc.z, acc.w));
    if (lane == 0 && p.lse) p.lse[row] = sum == 0.f ? -INFINITY : mx + logf(sum);
}

}  // namespace cudallm
