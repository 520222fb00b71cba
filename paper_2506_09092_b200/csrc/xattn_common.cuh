// What the cross-attention kernels share: parameters, 4-D TMA loads, tcgen05 wrappers with the A
// operand in shared or tensor memory, and the tile layout.
//
// A tile is 128 rows of one head in shared memory, its head dimension padded with zeros to DP =
// 64 or 128 (by TMA, which fills what lies outside the tensor): DP / 64 chunks of 64 columns, each
// 128 rows x 128 bytes in the 128-byte swizzle.  The same bytes serve the tensor core as a K-major
// operand (contraction over the head dimension) and as an MN-major one (contraction over the rows).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "elem.cuh"
#include "ptx.cuh"

namespace cudallm {

constexpr int kXaRows = 128;                   // rows of a tile
constexpr int kXaChunkBytes = kXaRows * 128;   // one 64-column chunk of a tile

struct XaStrides { long long b, r, h; };       // elements between batch items, rows, heads

// status detail codes of the attention kernels' bounded waits: (role << 8) | barrier
enum : int { kXaRoleLoad = 0x10, kXaRoleMma = 0x11, kXaRoleSoftmax = 0x12, kXaRoleDq = 0x20, kXaRoleDkv = 0x30 };

__device__ __forceinline__ void xa_report(int *status, int role, int what)
{
    if (atomicCAS(status, 0, -9 /* CUDALLM_ERR_DEVICE_TIMEOUT */) == 0) status[1] = (role << 8) | what;
}

// One 64-column chunk of a tile: columns 64 c .., head h, rows row .. row + 127, batch item b.
__device__ __forceinline__ void xa_load_chunk(const CUtensorMap *tm, uint32_t dst, uint32_t bar, int c, int h, int row, int b)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(c * 64), "r"(h), "r"(row), "r"(b), "r"(bar) : "memory");
}
template <int DP>
__device__ __forceinline__ void xa_load_tile(const CUtensorMap *tm, uint32_t dst, uint32_t bar, int h, int row, int b)
{
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) xa_load_chunk(tm, dst + c * kXaChunkBytes, bar, c, h, row, b);
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// D (tensor memory) (+)= A B with A and B in shared memory, or with A in tensor memory.
__device__ __forceinline__ void xa_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void xa_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}

// One lane of a converged warp.  The warp that issues products runs its loop as a whole, so that
// descriptors and addresses are uniform values, and only the instructions themselves are one lane's.
__device__ __forceinline__ bool elect_one()
{
    int one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.s32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}

// Product over the head dimension: D = A B^T, both tiles K-major (idesc says how many rows of B).
template <int DP>
__device__ __forceinline__ void xa_product_nt(uint32_t d, uint32_t a_tile, uint32_t b_tile, uint32_t idesc)
{
    const uint64_t a0 = make_smem_desc_sw128(a_tile, 16, 1024), b0 = make_smem_desc_sw128(b_tile, 16, 1024);
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        const uint64_t o = (k / 4) * (kXaChunkBytes >> 4) + (k % 4) * 2;
        xa_mma_ss(d, a0 + o, b0 + o, idesc, k > 0);
    }
}
// Product over a tile's rows: D (+)= P T, P (128 x 128, 16-bit) in tensor memory, tile T MN-major.  P lies in
// groups of 16 GROUP values, each STEP tensor-memory columns after the last.  HALVES says which half of each
// four steps of 16 takes part: 1 the first, 2 the second, 3 both.
template <int GROUP, int STEP, int HALVES = 3>
__device__ __forceinline__ void xa_product_tn(uint32_t d, uint32_t p_tmem, uint32_t tile, uint32_t idesc, bool accumulate)
{
    const uint64_t b0 = make_smem_desc_sw128(tile, kXaChunkBytes, 1024);
#pragma unroll
    for (int k = 0; k < kXaRows / 16; ++k)
        if ((k % 4 < 2 ? 1 : 2) & HALVES)
            xa_mma_ts(d, p_tmem + (k / GROUP) * STEP + (k % GROUP) * 8, b0 + k * (2048 >> 4), idesc,
                      accumulate || k > (HALVES == 2 ? 2 : 0));
}

// Instruction descriptor: kind::f16, both operands T, fp32 accumulator, A K-major, M = 128.
template <typename T> struct XaElem;
template <> struct XaElem<__nv_bfloat16> {
    static constexpr uint32_t kFormat = 1;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16x2(lo, hi); }
};
template <> struct XaElem<__half> {
    static constexpr uint32_t kFormat = 0;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
};
template <typename T>
__host__ __device__ constexpr uint32_t xa_idesc(int n, int b_mn_major)
{
    return (1u << 4) | (XaElem<T>::kFormat << 7) | (XaElem<T>::kFormat << 10) | ((uint32_t)b_mn_major << 16)
         | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kXaRows >> 4) << 24);
}

// 32 lanes x 16 consecutive columns, registers -> tensor memory and back.
__device__ __forceinline__ void tmem_st_32x32b_x16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
                   "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld_32x32b_x16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait()
{
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// Waits for the warp's loads from tensor memory; the registers are tied to the wait, so that no use
// of theirs can be moved ahead of it.
template <int N>
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&r)[N])
{
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}

// Maximum of three values; a NaN among them is the result.
__device__ __forceinline__ float max3_nan(float a, float b, float c)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// 2^x by the special-function unit (relative error ~2^-22); -inf gives 0.
__device__ __forceinline__ float xa_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Named barrier over `threads` threads that also tells each whether `ok` held for all of them.
__device__ __forceinline__ bool named_bar_all(int id, int threads, bool ok)
{
    int all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %3, 0;\n\tbar.red.and.pred q, %1, %2, p;\n\t"
                 "selp.s32 %0, 1, 0, q;\n\t}" : "=r"(all) : "r"(id), "r"(threads), "r"((int)ok) : "memory");
    return all != 0;
}

// What is left to wait for when a kernel has given up: the last copy into each stage of a ring of STAGES (`loads` of
// them were issued, in turn), and the products in flight.  With the library's own limit: the caller's may have
// run out because it is short, and copies must not land in what is another CTA's shared memory by then.
template <int STAGES>
__device__ __forceinline__ void xa_ring_landed(uint32_t full, int loads, volatile int *never)
{
    for (int s = 0; s < STAGES; ++s) {
        const int uses = (loads - s + STAGES - 1) / STAGES;
        if (uses > 0) mbar_wait(full + 8 * s, (uses - 1) & 1, never);
    }
}
// (by the warp that issued the products; the same lane is elected each time, and a commit covers what that lane has issued)
__device__ __forceinline__ void xa_products_done(uint32_t drain)
{
    if (elect_one()) {
        volatile int never = 0;
        umma_commit(drain);
        mbar_wait(drain, 0, &never);
    }
    __syncwarp();
}

// Valid keys of batch item b.
__device__ __forceinline__ int xa_keys(const int *lens, int b, int kv_rows)
{
    if (!lens) return kv_rows;
    const int n = lens[b];
    return n < 0 ? 0 : (n < kv_rows ? n : kv_rows);
}

// Zero a row of a tile that TMA has written: a padded row may hold anything, and 0 x NaN would reach
// the product's sums.  The writes must be followed by fence_proxy_async_smem() before the tensor core
// may read them.
template <int DP>
__device__ __forceinline__ void xa_zero_row(uint32_t tile, int row)
{
#pragma unroll
    for (int c = 0; c < DP / 64; ++c)
#pragma unroll
        for (int k = 0; k < 8; ++k) st_shared_v4_b32(tile + c * kXaChunkBytes + row * 128 + k * 16, 0, 0, 0, 0);
}

// Rows that a warp's lanes hold (lane t row t, PIECES x 16 bytes of it) to memory.  A store instruction whose
// lanes write 32 different rows takes as long as 32 lines do, so the rows pass through `stage` (32 x
// PIECES x 16 bytes of shared memory that only this warp uses; pieces of a row exchanged so that no two
// lanes meet in a bank) and leave as whole rows, PIECES lanes each.  Of the rows `rows` exist, of their
// pieces `pieces`.
template <int PIECES>
__device__ __forceinline__ void xa_store_rows(uint32_t stage, int lane, const uint4 (&v)[PIECES], uint8_t *dst, long long pitch,
                                              int rows, int pieces)
{
    static_assert(PIECES == 4 || PIECES == 8, "64 or 128 bytes");
    auto at = [&](int row, int i) {
        return stage + row * (PIECES * 16) + ((i ^ ((PIECES == 8 ? row : row >> 1) & (PIECES - 1))) << 4);
    };
#pragma unroll
    for (int i = 0; i < PIECES; ++i) st_shared_v4_b32(at(lane, i), v[i].x, v[i].y, v[i].z, v[i].w);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        const int row = (k * 32 + lane) / PIECES, i = lane % PIECES;
        uint4 w;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(at(row, i)) : "memory");
        if (row < rows && i < pieces) *reinterpret_cast<uint4 *>(dst + row * pitch + i * 16) = w;
    }
    __syncwarp();
}

// A warp's 32 rows x NC (32 or 64) columns of an fp32 result in tensor memory (from column `t_addr` on), row t times
// f, to rows of T (`dst`: row 0, first of the columns; `pitch` in elements; `left` columns exist).
template <int NC, typename T>
__device__ __forceinline__ void xa_store_result(uint32_t t_addr, uint32_t stage, int lane, float f, T *dst, long long pitch, int rows, int left)
{
    uint4 v[NC / 8];
#pragma unroll
    for (int c = 0; c < NC / 32; ++c) {
        uint32_t r[32];
        tmem_ld_32x32b_x32(t_addr + 32 * c, r);
        tmem_ld_wait_for(r);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                w[k] = XaElem<T>::pack(__uint_as_float(r[8 * g + 2 * k]) * f, __uint_as_float(r[8 * g + 2 * k + 1]) * f);
            v[4 * c + g] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    xa_store_rows<NC / 8>(stage, lane, v, reinterpret_cast<uint8_t *>(dst), pitch * (long long)sizeof(T), rows, left / 8);
}
// The same to rows of fp32.
template <int NC>
__device__ __forceinline__ void xa_store_part(uint32_t t_addr, uint32_t stage, int lane, float f, float *dst, long long pitch, int rows, int left)
{
#pragma unroll
    for (int c = 0; c < NC / 32; ++c) {
        uint32_t r[32];
        tmem_ld_32x32b_x32(t_addr + 32 * c, r);
        tmem_ld_wait_for(r);
        uint4 v[8];
#pragma unroll
        for (int g = 0; g < 8; ++g)
            v[g] = make_uint4(__float_as_uint(__uint_as_float(r[4 * g]) * f), __float_as_uint(__uint_as_float(r[4 * g + 1]) * f),
                              __float_as_uint(__uint_as_float(r[4 * g + 2]) * f), __float_as_uint(__uint_as_float(r[4 * g + 3]) * f));
        xa_store_rows<8>(stage, lane, v, reinterpret_cast<uint8_t *>(dst + 32 * c), pitch * 4, rows, (left - 32 * c) / 4);
    }
}

}  // namespace cudallm
