// Cross attention, forward: O = softmax(scale Q K^T) V per head, keys from kv_len on masked.
//
// A CTA owns two tiles of 128 query rows of one head and walks the keys in blocks of 128.
//   warps 0-3, 4-7  softmax of the first and second tile: a thread is a row (a lane of tensor
//                   memory), so the row's maximum and sum need no exchange between threads
//   warp 8          TMA: the queries once, then K and V tiles through a ring
//   warp 9          the tensor core: S_j = Q_j K^T into tensor memory, O_j += P_j V with P_j read
//                   from tensor memory (it lies over S_j, as 16-bit values)
// While one tile's softmax runs, the tensor core works for the other.  One pass over the keys: the
// row's reference maximum is only moved (and O_j rescaled in tensor memory) when a block's maximum
// passes it by more than 2^8, since any reference gives the same quotient; probabilities stay
// below 2^8, far inside every type's range.
//
// Bound: the tensor core (two products of 2 x 128 x 128 x DP multiply-adds per block and pair of
// tiles) and, close behind it at DP = 64, the special-function unit (16 exponentials per clock).
// Tensor memory: S_0 and S_1 128 columns each, O_0 and O_1 DP columns each: all 512 at DP = 128.
#pragma once
#include "xattn_common.cuh"

namespace cudallm {

constexpr int kXaFwdThreads = 320;

struct XaFwdParams {
    void *o;
    float *lse;                 // [batch][q_heads][q_rows], or NULL
    float *o_part, *lse_part;   // splits > 1: [split][batch][q_heads][q_rows]([head_dim]) partial results
    const int *lens;
    XaStrides so;
    int q_rows, kv_rows, q_heads, group, batch, head_dim;
    int q_tiles;                // pairs of query tiles per head
    int splits, blocks_per_split;
    float scale, scale_log2;    // scale, and scale * log2(e)
    int *status;
    int skip_loads;             // self-test of the bounded waits: nothing is loaded, every wait runs out
    unsigned long long wait_limit_ns;
};

template <int DP> struct XaFwdSmem {
    static constexpr int kTile = DP / 64 * kXaChunkBytes;
    static constexpr int kStages = DP == 128 ? 5 : 10;
    static constexpr int kRing = 2 * kTile;
    static constexpr int kBars = kRing + kStages * kTile;
    // q_full, s_full[2], p_full[2], pv_done[2], full[kStages], empty[kStages]
    static constexpr int kNumBars = 7 + 2 * kStages;
    static constexpr int kMisc = kBars + kNumBars * 8;
    static constexpr int kBytes = kMisc + 16;
};

template <int DP, typename T>
__global__ void __launch_bounds__(kXaFwdThreads, 1)
xattn_fwd_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                 const __grid_constant__ CUtensorMap tm_v, const XaFwdParams p)
{
    using L = XaFwdSmem<DP>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sbase = smem_u32(smem);
    const uint32_t bars = sbase + L::kBars;
    const uint32_t q_full = bars, s_full = bars + 8, p_full = bars + 24, pv_done = bars + 40, full = bars + 56,
                   empty = full + 8 * L::kStages;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + L::kMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L::kMisc + 4);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int qt = blockIdx.x % p.q_tiles;
    const int bh = blockIdx.x / p.q_tiles;
    const int h = bh % p.q_heads, b = bh / p.q_heads;
    const int kvh = h / p.group;
    const int row0 = qt * 2 * kXaRows;
    const int tiles = p.q_rows - row0 > kXaRows ? 2 : 1;

    if (tid == 0) {
        *abort_flag = 0;
        mbar_init(q_full, 1);
        for (int j = 0; j < 2; ++j) {
            mbar_init(s_full + 8 * j, 1);
            mbar_init(p_full + 8 * j, kXaRows);
            mbar_init(pv_done + 8 * j, 1);
        }
        for (int s = 0; s < L::kStages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        fence_mbar_init();
    }
    if (warp == 9) {
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
    const int blk0 = blockIdx.y * p.blocks_per_split;
    const int nblk = min(p.blocks_per_split, (keys + kXaRows - 1) / kXaRows - blk0);      // <= 0: no keys here

    if (warp == 8) {
        if (lane == 0 && nblk > 0 && !p.skip_loads) {
            mbar_expect_tx(q_full, tiles * L::kTile);
            for (int j = 0; j < tiles; ++j) xa_load_tile<DP>(&tm_q, sbase + j * L::kTile, q_full, h, row0 + j * kXaRows, b);
            bool ok = true;
            int it = 0;
            for (int i = 0; i < nblk && ok; ++i) {
                for (int w = 0; w < 2; ++w, ++it) {                       // K, then V
                    const int s = it % L::kStages, use = it / L::kStages;
                    if (use > 0) ok = mbar_wait(empty + 8 * s, (use - 1) & 1, abort_flag, p.wait_limit_ns);
                    if (!ok) break;
                    mbar_expect_tx(full + 8 * s, L::kTile);
                    xa_load_tile<DP>(w ? &tm_v : &tm_k, sbase + L::kRing + s * L::kTile, full + 8 * s, kvh,
                                     (blk0 + i) * kXaRows, b);
                }
            }
            if (!ok) {
                // another role gave up: the copies in flight must land before the CTA ends
                xa_report(p.status, kXaRoleLoad, 1);
                volatile int never = 0;
                mbar_wait(q_full, 0, &never, p.wait_limit_ns);
                for (int s = 0; s < L::kStages; ++s) {
                    const int uses = (it - s + L::kStages - 1) / L::kStages;      // loads issued into stage s
                    if (uses > 0) mbar_wait(full + 8 * s, (uses - 1) & 1, &never, p.wait_limit_ns);
                }
            }
        }
    } else if (warp == 9) {
        if (lane == 0 && nblk > 0) {
            constexpr uint32_t idesc_s = xa_idesc<T>(128, 0), idesc_o = xa_idesc<T>(DP, 1);
            const uint32_t t_s = tmem, t_o = tmem + 256;
            bool ok = mbar_wait(q_full, 0, abort_flag, p.wait_limit_ns);
            ok = ok && mbar_wait(full, 0, abort_flag, p.wait_limit_ns);
            if (ok) {
                tc_fence_after();
                for (int j = 0; j < tiles; ++j) {
                    xa_product_nt<DP>(t_s + 128 * j, sbase + j * L::kTile, sbase + L::kRing, idesc_s);
                    umma_commit(s_full + 8 * j);
                }
                umma_commit(empty);
            }
            for (int i = 0; i < nblk && ok; ++i) {
                const int iv = 2 * i + 1, ik = 2 * i + 2;                 // ring positions of V(i) and K(i + 1)
                const int sv = iv % L::kStages, sk = ik % L::kStages;
                const bool more = i + 1 < nblk;
                for (int j = 0; j < tiles && ok; ++j) {
                    if (j == 0) ok = mbar_wait(full + 8 * sv, (iv / L::kStages) & 1, abort_flag, p.wait_limit_ns);
                    ok = ok && mbar_wait(p_full + 8 * j, i & 1, abort_flag, p.wait_limit_ns);
                    if (!ok) break;
                    tc_fence_after();
                    // (products of one issuing thread run in order: S_j of the next block, which
                    // overwrites P_j, starts after this product has read it)
                    xa_product_tn<32>(t_o + DP * j, t_s + 128 * j, sbase + L::kRing + sv * L::kTile, idesc_o, i > 0);
                    umma_commit(pv_done + 8 * j);
                    if (more) {
                        if (j == 0) ok = mbar_wait(full + 8 * sk, (ik / L::kStages) & 1, abort_flag, p.wait_limit_ns);
                        if (!ok) break;
                        xa_product_nt<DP>(t_s + 128 * j, sbase + j * L::kTile, sbase + L::kRing + sk * L::kTile, idesc_s);
                        umma_commit(s_full + 8 * j);
                    }
                }
                if (ok) {
                    umma_commit(empty + 8 * sv);
                    if (more) umma_commit(empty + 8 * sk);
                }
            }
            if (!ok) xa_report(p.status, kXaRoleMma, 1);
        }
    } else {
        const int j = warp >> 2;
        if (j < tiles && nblk > 0) {
            const int t = tid & (kXaRows - 1);                           // row of the tile = lane of tensor memory
            const uint32_t t_lane = static_cast<uint32_t>((warp & 3) * 32) << 16;
            const uint32_t t_s = tmem + 128 * j + t_lane, t_o = tmem + 256 + DP * j + t_lane;
            float m = -INFINITY, l = 0.f;
            bool ok = true;
            for (int i = 0; i < nblk; ++i) {
                ok = __all_sync(0xffffffffu, mbar_wait(s_full + 8 * j, i & 1, abort_flag, p.wait_limit_ns));
                if (!ok) break;
                tc_fence_after();
                uint32_t r[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld_32x32b_x32(t_s + 32 * c, r[c]);
                tmem_ld_wait();
                const int valid = keys - (blk0 + i) * kXaRows;            // keys of this block that exist
                if (valid < kXaRows) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (c * 32 + k >= valid) r[c][k] = 0xFF800000u;                 // -inf
                    if (j == 0 && keys < p.kv_rows) {
                        // rows of V that are padding, not beyond the tensor's end
                        const int iv = 2 * i + 1, sv = iv % L::kStages;
                        ok = __all_sync(0xffffffffu, mbar_wait(full + 8 * sv, (iv / L::kStages) & 1, abort_flag, p.wait_limit_ns));
                        if (!ok) break;
                        xa_zero_rows<DP>(sbase + L::kRing + sv * L::kTile, t, valid);
                        fence_proxy_async_smem();
                    }
                }
                float mx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx[c] = __uint_as_float(r[c][0]);
#pragma unroll
                    for (int k = 1; k < 32; ++k) mx[c] = fmaxf(mx[c], __uint_as_float(r[c][k]));
                }
                const float bm = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                if (i == 0) {
                    m = bm;
                } else {
                    const bool move = (bm - m) * p.scale_log2 > 8.f;
                    if (__any_sync(0xffffffffu, move)) {
                        const float alpha = move ? xa_exp2((m - bm) * p.scale_log2) : 1.f;
                        if (move) m = bm;
                        l *= alpha;
                        ok = __all_sync(0xffffffffu, mbar_wait(pv_done + 8 * j, (i - 1) & 1, abort_flag, p.wait_limit_ns));
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll
                        for (int c = 0; c < DP / 16; ++c) {               // (16 at a time: the block's scores
                            uint32_t o[16];                               // stay in registers meanwhile)
                            tmem_ld_32x32b_x16(t_o + 16 * c, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                            tmem_st_32x32b_x16(t_o + 16 * c, o);
                        }
                    }
                }
                const float neg = -m * p.scale_log2;
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int k = 0; k < 32; k += 2) {
                        const float e0 = xa_exp2(fmaf(__uint_as_float(r[c][k]), p.scale_log2, neg));
                        const float e1 = xa_exp2(fmaf(__uint_as_float(r[c][k + 1]), p.scale_log2, neg));
                        sum[k & 2] += e0;
                        sum[(k & 2) + 1] += e1;
                        w[k >> 1] = XaElem<T>::pack(e0, e1);
                    }
                    tmem_st_32x32b_x16(t_s + 16 * c, w);                  // over S, which is in registers
                }
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                tmem_st_wait();
                tc_fence_before();
                mbar_arrive(p_full + 8 * j);
            }
            // the row's output
            if (ok) ok = __all_sync(0xffffffffu, mbar_wait(pv_done + 8 * j, (nblk - 1) & 1, abort_flag, p.wait_limit_ns));
            if (ok) {
                tc_fence_after();
                const int row = row0 + j * kXaRows + t;
                const bool live = row < p.q_rows;
                const float inv = 1.f / l;
                const float lse = fmaf(m, p.scale, logf(l));
                const long long bhr = (long long)bh * p.q_rows + row;
                const long long rows_all = (long long)p.batch * p.q_heads * p.q_rows;
                const long long part = (long long)blockIdx.y * rows_all + bhr;
                T *dst = static_cast<T *>(p.o) + b * p.so.b + row * p.so.r + h * p.so.h;
                float *dst_part = p.o_part + part * p.head_dim;
#pragma unroll
                for (int c = 0; c < DP / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld_32x32b_x32(t_o + 32 * c, o);
                    tmem_ld_wait();
                    float v[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(o[k]) * inv;
                    const int left = p.head_dim - c * 32;
                    if (live) {
                        if (p.splits == 1) {
                            xa_store_32(dst + c * 32, v, left);
                        } else {
#pragma unroll
                            for (int g = 0; g < 8; ++g)
                                if (g * 4 < left)
                                    *reinterpret_cast<float4 *>(dst_part + c * 32 + g * 4) =
                                        make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
                        }
                    }
                }
                if (live) {
                    if (p.splits > 1) p.lse_part[part] = lse;
                    else if (p.lse) p.lse[bhr] = lse;
                }
            } else if (lane == 0) {
                xa_report(p.status, kXaRoleSoftmax, 1);
            }
        } else if (j < tiles) {
            // no keys: the output is zero, the sum of no exponentials is zero
            const int row = row0 + j * kXaRows + (tid & (kXaRows - 1));
            if (row < p.q_rows) {
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
    // all products have been waited for (the last pv_done), or the kernel gave up after a failed wait;
    // then the tensor core's queue is drained before tensor memory is released
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        if (*abort_flag) {
            if (lane == 0) {
                volatile int never = 0;
                mbar_init(q_full, 1);
                fence_mbar_init();
                umma_commit(q_full);
                mbar_wait(q_full, 0, &never, p.wait_limit_ns);
            }
            __syncwarp();
        }
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
        const float ws = __shfl_sync(0xffffffffu, w, s) * inv;
        if (ws == 0.f || col >= p.head_dim) continue;
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
