// Attention of the newest tokens over pages where many rows (query heads of a key head x new tokens) share a
// key head: drafts under wide groups, prompts.
//
// One CTA an SM, made of independent roles that walk the same segments (items, key heads, row tiles and blocks of
// 128 keys, dealt out in equal shares as in paged_attn.cuh):
//   warps 0-7    softmax: 128 rows are the lanes of tensor memory, a row's 128 scores are shared by two
//                threads; then the rows' results
//   warp 8       the tensor core: S = Q K^T into one of two places in tensor memory, O += P V with P written over S
//   warps 9, 10  TMA: the pages of a block of K, and those of V, into a ring of tiles, a lane a page (a TMA instruction
//                takes its warp some 120 clocks: one warp for both was the bound with pages of 16 rows); needs pages of 8, 16, 32,
//                64 or a multiple of 128 rows, so that they fill a tile and begin on a swizzle's boundary
//   warp 11      the queries of a segment
// While the softmax of one block runs, the scores of the next are formed; the copies run ahead by the ring, into
// the next segment too.  tcgen05 has 128 rows whether they are used or not, but the products of a block take a
// third of the time that its bytes take from HBM, no registers and no issue slots of the other warps; mma.sync
// with the same rows (paged_walk_wide) is bound by those.
// Drafts (16 sequences of 16384 states, 5 tokens of 32 heads on 4 key heads of 128, 40 rows): 98-104 us, 5.2 TB/s; what it lacks are
// some 6 us until the first block's scores and 4 for the join.  Prompts (one of 32000 tokens, 8 heads on each of 4 key
// heads of 128): 9.3 ms, 0.90 PFLOP/s; 4 of 1000 behind 3000, 8 on 8: 586 us, 0.78; heads of 64: half of that rate, since
// the exponentials of a block are as many and its products half as large.  Sixteen softmax warps had 96 registers a
// thread, spilled and were slower.
#pragma once
#include "paged_attn.cuh"

namespace cudallm {

constexpr int kPtSoftmaxWarps = 8, kPtMmaWarp = 8, kPtLoadWarp = 9, kPtQueryWarp = 11;
constexpr int kPtThreads = 32 * (kPtQueryWarp + 1);        // 12 warps: three to a quarter of the SM, 168 registers each
constexpr int kPtMaskSlots = 8;                // blocks whose masks are kept: more than the copies can be ahead of the softmax
constexpr int kPtWords = kXaRows / 32;         // masks of a block: a bit a key

enum : int { kXaRolePagedLoad = 0x40, kXaRolePagedMma = 0x41, kXaRolePagedSoftmax = 0x42, kXaRolePagedQuery = 0x43 };

template <int DP> struct PagedTileSmem {
    static constexpr int kRows = kXaRows, kBlock = kXaRows;
    static constexpr int kTile = DP / 64 * kXaChunkBytes;          // 128 rows of Q, K or V
    static constexpr int kStages = DP == 128 ? 6 : 12;             // (even: K and V each have every second)
    static constexpr int kRing = kTile;                            // behind the queries
    static constexpr int kBars = kRing + kStages * kTile;
    // q_full, q_empty, pv_done, drain, s_full[2], p_full[2], full[kStages], empty[kStages]
    static constexpr int kNumBars = 8 + 2 * kStages;
    static constexpr int kMisc = kBars + kNumBars * 8;             // tensor memory's address, the abort flag
    static constexpr int kXch = kMisc + 16;                        // floats [parity][half][row]
    static constexpr int kMask = kXch + 2 * 2 * kXaRows * 4;       // words [slot][32 keys]: keys that are there
    static constexpr int kBad = kMask + kPtMaskSlots * kPtWords * 4;   // the same: keys whose values were set aside
    static constexpr int kBytes = kBad + kPtMaskSlots * kPtWords * 4;
    static_assert(kBytes <= 227 * 1024 && kBytes > 114 * 1024, "one CTA an SM");
    static constexpr int kSlot = kRows * (DP + 1);                 // floats of a part's result
    static constexpr int kTmemO = 256;                             // S and P: columns 0 and 128
};
// Pages that TMA can bring into tiles.
inline bool paged_tile_pages(long long page_rows) { return page_rows % 8 == 0 && (kXaRows % page_rows == 0 || page_rows % kXaRows == 0); }

struct PagedTileParams {
    PagedParams a;
    int *status;
    int skip_loads;             // self-test of the bounded waits: nothing is loaded, every wait runs out
    unsigned long long wait_limit_ns;
};

// 16-byte piece c of row r of a tile in the 128-byte swizzle, 64 columns a chunk.
__device__ __forceinline__ uint32_t tile_piece(int r, int c)
{
    return (uint32_t)((c >> 3) * kXaChunkBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}

// Values that were set aside (see the softmax), of keys in the blocks from `aside` on: added to this row's half of the columns of
// O in tensor memory, from scores taken anew.  A warp's lanes together, those without a row of their own among them: such a lane sees
// nothing (seen = 0), so that no query is read for it.  `block`: the number behind the segment's last.
template <int DP, typename T>
__device__ __noinline__ void add_set_aside(const PagedParams &p, const int *pages, int b, int kvh, int row, int seen, float m, int d0,
                                           uint32_t t_o, volatile uint32_t *bads, int key0, int block, int blocks, int aside)
{
    using L = PagedTileSmem<DP>;
    for (int i = aside; i < blocks; ++i)
        for (int w = 0; w < kPtWords; ++w)
            for (uint32_t rest = bads[(block - blocks + i) % kPtMaskSlots * kPtWords + w]; rest; rest &= rest - 1) {
                const int key = key0 + i * L::kBlock + w * 32 + __ffs(rest) - 1;
                const int pc = (int)fast_div((uint32_t)key, p.by_page_rows), in_page = key - pc * p.page_rows;
                const long long page = pages[pc];
                const T *k = static_cast<const T *>(p.k) + page * p.sk.page + in_page * p.sk.row + kvh * p.sk.head;
                const T *v = static_cast<const T *>(p.v) + page * p.sv.page + in_page * p.sv.row + kvh * p.sv.head + d0;
                float weight = 0.f;
                if (key < seen) {
                    const T *q = paged_q_row<T>(p, b, kvh, row);
                    float s = 0.f;
                    for (int d = 0; d < p.head_dim; ++d) s = fmaf(elem_to_float(q[d]), elem_to_float(k[d]), s);
                    weight = m == -INFINITY ? 0.f : xa_exp2((s - m) * p.scale_log2);       // (all its scores are -inf)
                }
                for (int c = 0; c < DP / 2; c += 16) {
                    uint32_t o[16];
                    tmem_ld_32x32b_x16(t_o + c, o);
                    tmem_ld_wait_for(o);
#pragma unroll
                    for (int n = 0; n < 16; ++n)
                        if (key < seen && d0 + c + n < p.head_dim)
                            o[n] = __float_as_uint(fmaf(weight, elem_to_float(v[c + n]), __uint_as_float(o[n])));
                    tmem_st_32x32b_x16(t_o + c, o);
                    tmem_st_wait();
                }
            }
}

// Rows from `row` on of a page and key head, 64 columns.
__device__ __forceinline__ void paged_load_box(const CUtensorMap *tm, uint32_t dst, uint32_t bar, int c, int head, int row, int page)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(c * 64), "r"(head), "r"(row), "r"(page), "r"(bar) : "memory");
}

template <int DP, typename T>
__global__ void __launch_bounds__(kPtThreads, 1)
paged_tile_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const __grid_constant__ PagedTileParams tp)
{
    using L = PagedTileSmem<DP>;
    constexpr int kChunks = DP / 8;
    extern __shared__ __align__(1024) uint8_t tile_smem[];
    uint8_t *const smem = tile_smem;
    const PagedParams &p = tp.a;
    const uint32_t sbase = smem_u32(smem), bars = sbase + L::kBars;
    const uint32_t q_full = bars, q_empty = bars + 8, pv_done = bars + 16, drain = bars + 24, s_full = bars + 32, p_full = bars + 48,
                   full = bars + 64, empty = full + 8 * L::kStages;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem + L::kMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + L::kMisc + 4);
    volatile uint32_t *masks = reinterpret_cast<volatile uint32_t *>(smem + L::kMask);
    volatile uint32_t *bads = reinterpret_cast<volatile uint32_t *>(smem + L::kBad);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

    if (tid == 0) *abort_flag = 0;
    if (warp == 0) {
        // arrivals: the softmax warps at p_full, one at the others
        static_assert(L::kNumBars <= 32, "barriers");
        if (lane < L::kNumBars) mbar_init(bars + 8 * lane, lane == 6 || lane == 7 ? kPtSoftmaxWarps : 1);
        fence_mbar_init();
    }
    if (warp == kPtMmaWarp) {
        tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (warp == kPtLoadWarp && lane == 0) {
        prefetch_tensormap(&tm_k);
        prefetch_tensormap(&tm_v);
    }
    // only now: the next kernel of the stream may start once every CTA of this one holds its tensor memory
    grid_launch_dependents();
    grid_dependency_wait();

    long long per;
    PagedSegments<L::kRows, L::kBlock> seg(p);
    const bool some = seg.locate(smem, per);
    const int cta = blockIdx.x;
    // (a whole warp waits; what fails for one lane ends it for all)
    auto wait = [&](uint32_t bar, int parity) {
        return __all_sync(0xffffffffu, mbar_wait(bar, parity & 1, abort_flag, tp.wait_limit_ns)) != 0;
    };
    int segments = 0, block = 0;                                   // of this CTA so far, those without keys not counted
    bool ok = true;

    if (warp == kPtQueryWarp) {
        for (bool more = some; ok && more; more = seg.next()) {
            const int rows = seg.rows();
            if (seg.live() == 0) continue;
            if (segments > 0) ok = wait(q_empty, segments - 1);     // the segment before has formed its last scores
            if (!ok) break;
            // (rows that do not exist are the tensor core's own affair: they reach no other row's result)
            constexpr int kRowStep = 32 / kChunks;                 // rows that an instruction covers
            const int c = lane % kChunks, row0 = seg.rt * L::kRows;
            const bool live = c * 8 < p.head_dim;
#pragma unroll 2
            for (int r = lane / kChunks; r < rows; r += kRowStep)
                cp_async_16_cg(sbase + tile_piece(r, c), paged_q_row<T>(p, seg.b, seg.kvh, row0 + r) + (live ? c * 8 : 0), live ? 16 : 0);
            cp_async_wait_all();
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);
            ++segments;
        }
        if (!ok && lane == 0) xa_report(tp.status, kXaRolePagedQuery, 1);
    } else if (warp > kPtMmaWarp) {
        // the pages of a block: lane j has the j-th, up to 16 of them; of larger ones the part that the block is
        const int box = min(p.page_rows, L::kBlock), pages = L::kBlock / box;
        const int kv = warp - kPtLoadWarp;
        const CUtensorMap *tm = kv ? &tm_v : &tm_k;
        ok = !tp.skip_loads;
        for (bool more = some; ok && more; more = seg.next()) {
            const int blocks = seg.live(), key0 = seg.key0(), key_end = seg.key_end();
            int page = -1, in_page = 0;                            // this lane's page of the next block
            auto look_up = [&](int i) {
                page = -1;
                const int key = key0 + i * L::kBlock + lane * box;
                if (i < blocks && lane < pages && key < key_end) {
                    const int c = (int)fast_div((uint32_t)key, p.by_page_rows);
                    in_page = key - c * p.page_rows;
                    page = seg.it.row[c];
                }
            };
            look_up(0);
            for (int i = 0; i < blocks && ok; ++i, ++block) {
                const int at = page, from = in_page;
                const bool there = (unsigned)at < (unsigned)p.pages;
                const uint32_t have = __ballot_sync(0xffffffffu, there);
                look_up(i + 1);
                const int tile = 2 * block + kv, stage = tile % L::kStages, use = tile / L::kStages;
                if (use > 0) ok = wait(empty + 8 * stage, use - 1);
                if (!ok) break;
                if (kv == 0) {
#pragma unroll
                    for (int w = 0; w < kPtWords; ++w) {
                        const int r = w * 32 + lane;
                        const uint32_t word = __ballot_sync(0xffffffffu, (have >> (r / box) & 1) && key0 + i * L::kBlock + r < key_end);
                        if (lane == 0) masks[block % kPtMaskSlots * kPtWords + w] = word;
                    }
                    __syncwarp();
                }
                // (the pages go round by shuffle and one lane asks for all of them: their addresses are uniform values then)
                if (lane == 0) mbar_expect_tx(full + 8 * stage, __popc(have) * box * (DP / 64) * 128);
                __syncwarp();
                uint32_t dst = sbase + L::kRing + stage * L::kTile;
                for (int j = 0; j < pages; ++j, dst += box * 128) {
                    const int pg = __shfl_sync(0xffffffffu, at, j), row = __shfl_sync(0xffffffffu, from, j);
                    if ((have >> j & 1) && elect_one()) {
#pragma unroll
                        for (int c = 0; c < DP / 64; ++c)
                            paged_load_box(tm, dst + c * kXaChunkBytes, full + 8 * stage, c, seg.kvh, row, pg);
                    }
                    __syncwarp();
                }
            }
        }
        if (!ok && lane == 0 && !tp.skip_loads) xa_report(tp.status, kXaRolePagedLoad, 1);
    } else if (warp == kPtMmaWarp) {
        constexpr uint32_t idesc_s = xa_idesc<T>(kXaRows, 0), idesc_o = xa_idesc<T>(DP, 1);
        const uint32_t t0 = __shfl_sync(0xffffffffu, tmem, 0);
        auto tile_at = [&](int tile) { return sbase + L::kRing + tile % L::kStages * L::kTile; };
        auto wait_tile = [&](int tile) { return wait(full + 8 * (tile % L::kStages), tile / L::kStages); };
        // scores of block g; the segment's last ones free its queries
        auto scores = [&](int g, bool last) {
            ok = ok && wait_tile(2 * g);
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
                xa_product_nt<DP>(t0 + 128 * (g & 1), sbase, tile_at(2 * g), idesc_s);
                umma_commit(s_full + 8 * (g & 1));
                umma_commit(empty + 8 * (2 * g % L::kStages));
                if (last) umma_commit(q_empty);
            }
            __syncwarp();
        };
        for (bool more = some; ok && more; more = seg.next()) {
            const int blocks = seg.live();
            if (blocks == 0) continue;
            ok = wait(q_full, segments);
            scores(block, blocks == 1);
            for (int i = 0; i < blocks && ok; ++i, ++block) {
                if (i + 1 < blocks) scores(block + 1, i + 2 == blocks);
                ok = ok && wait_tile(2 * block + 1) && wait(p_full + 8 * (block & 1), block >> 1);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    xa_product_tn<4, 64>(t0 + L::kTmemO, t0 + 128 * (block & 1), tile_at(2 * block + 1), idesc_o, i > 0);
                    umma_commit(pv_done);
                    umma_commit(empty + 8 * ((2 * block + 1) % L::kStages));
                }
                __syncwarp();
            }
            ++segments;
        }
        if (!ok && lane == 0) xa_report(tp.status, kXaRolePagedMma, 1);
    } else {
        const int half = warp >> 2, t = (warp & 3) * 32 + lane;    // half of a block's keys; row of the tile = lane of tensor memory
        const uint32_t t_lane = static_cast<uint32_t>((warp & 3) * 32) << 16, t_o = tmem + L::kTmemO + half * (DP / 2) + t_lane;
        float *xch = reinterpret_cast<float *>(smem + L::kXch);
        // the two warps that share rows meet at a barrier of their own, and agree there on whether to go on
        auto meet = [&]() { ok = named_bar_all(1 + (warp & 3), 64, ok); };
        for (bool more = some; ok && more; more = seg.next()) {
            const int blocks = seg.live(), rows = seg.rows(), key0 = seg.key0(), seen_lo = seg.seen_lo();
            const int row = seg.rt * L::kRows + t, token = paged_token(p, row), h = seg.kvh * p.group + row - token * p.group;
            const bool mine = t < rows, warp_rows = (warp & 3) * 32 < rows;
            const int seen = mine ? paged_seen(seg.it, token) : 0x7fffffff;       // (rows that do not exist may see anything)
            float m = -INFINITY, l = 0.f;
            bool any = false;
            for (int i = 0; i < blocks; ++i, ++block) {
                ok = ok && wait(s_full + 8 * (block & 1), block >> 1);
                tc_fence_after();
                uint32_t r[2][32];
                float bm = -INFINITY;
                const uint32_t t_s = tmem + 128 * (block & 1) + 64 * half + t_lane;
                if (ok && warp_rows) {
                    tmem_ld_32x32b_x32(t_s, r[0]);
                    tmem_ld_32x32b_x32(t_s + 32, r[1]);
                    const int first = key0 + i * L::kBlock + half * 64;
                    uint32_t see[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        see[c] = masks[block % kPtMaskSlots * kPtWords + half * 2 + c] & low_bits(seen - first - 32 * c);
                        any |= see[c] != 0;
                    }
                    tmem_ld_wait_for(r[0]);
                    tmem_ld_wait_for(r[1]);
                    if (__any_sync(0xffffffffu, (see[0] & see[1]) != 0xffffffffu)) {
#pragma unroll
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if (!(see[c] >> k & 1)) r[c][k] = 0xFF800000u;      // -inf
                    }
                    bm = max3_nan(xa_max32(r[0]), xa_max32(r[1]), -INFINITY);
                }
                // the other half of the row
                xch[((block & 1) * 2 + half) * kXaRows + t] = bm;
                meet();
                if (!ok) break;
                if (warp_rows) {
                    bm = max3_nan(bm, xch[((block & 1) * 2 + (half ^ 1)) * kXaRows + t], bm);
                    // The reference is moved only when it is passed by more than 2^8 (or there was none, or with a NaN): any
                    // reference gives the same quotient, and probabilities below 2^8 are far inside every type's range.
                    const bool move = m == -INFINITY ? !(bm == -INFINITY) : !((bm - m) * p.scale_log2 <= 8.f);
                    if (__any_sync(0xffffffffu, move)) {
                        const float alpha = move && m != -INFINITY ? xa_exp2((m - bm) * p.scale_log2) : 1.f;
                        if (move) m = bm;
                        l *= alpha;
                        if (i > 0) {
                            ok = wait(pv_done, block - 1);
                            tc_fence_after();
#pragma unroll
                            for (int c = 0; c < DP / 32; ++c) {    // half of O's columns
                                uint32_t o[16];
                                tmem_ld_32x32b_x16(t_o + 16 * c, o);
                                tmem_ld_wait_for(o);
#pragma unroll
                                for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                                tmem_st_32x32b_x16(t_o + 16 * c, o);
                            }
                        }
                    }
                    // (a row that has seen nothing yet: all its scores are -inf, and so are their differences to 0)
                    const float neg = m == -INFINITY ? 0.f : -m * p.scale_log2;
                    const uint64_t scale2 = f32x2(p.scale_log2, p.scale_log2), neg2 = f32x2(neg, neg);
                    uint64_t sum2[2] = {0, 0};
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
                            sum2[k & 1] = f32x2_add(sum2[k & 1], f32x2(lo, hi));
                            w[k] = XaElem<T>::pack(lo, hi);
                        }
                        tmem_st_32x32b_x16(t_s + 16 * c, w);       // (over this thread's own half of S)
                    }
                    float s0, s1;
                    f32x2_split(f32x2_add(sum2[0], sum2[1]), s0, s1);
                    l += s0 + s1;
                    tmem_st_wait();
                }
                // What must not meet P = 0 in the product, since 0 x NaN is NaN: rows of V that are not there become zero,
                // and so do those that some of the rows do not see if they hold a value that is not finite (who sees
                // them adds them by hand at the end).  Thread t has row t.
                if (half == 0) {
                    const uint32_t word = masks[block % kPtMaskSlots * kPtWords + warp];
                    const int hidden = seen_lo - (key0 + i * L::kBlock);   // rows from here on are not seen by all
                    uint32_t aside = 0;
                    if (word != 0xffffffffu || hidden < warp * 32 + 32) {
                        const int tile = 2 * block + 1, stage = tile % L::kStages;
                        ok = ok && wait(full + 8 * stage, tile / L::kStages);
                        const uint32_t at = sbase + L::kRing + stage * L::kTile;
                        bool bad = false;
                        if (ok && (word >> lane & 1) && t >= hidden)
                            for (int c = 0; c < kChunks; ++c) bad |= any_not_finite<T>(ld_shared_v4(at + tile_piece(t, c)));
                        if (ok && (bad || !(word >> lane & 1)))
                            for (int c = 0; c < kChunks; ++c) st_shared_v4_b32(at + tile_piece(t, c), 0, 0, 0, 0);
                        fence_proxy_async_smem();
                        aside = __ballot_sync(0xffffffffu, bad);
                    }
                    if (lane == 0) bads[block % kPtMaskSlots * kPtWords + warp] = aside;
                }
                // The product of the block before is over before this one's may start: so a wait for it, here and at the
                // segment's end, is never for a phase two behind (whose parity would pass for the one that is meant).
                if (i > 0) ok = ok && wait(pv_done, block - 1);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8 * (block & 1));
            }
            // The row's result: the halves' sums join, each thread has half of the columns.  (A wait that failed for one of the
            // two warps in the last block is both's here.)
            if (blocks > 0) {
                ok = ok && wait(pv_done, block - 1);
                // scores of -inf alone are not the same as no scores: a mark that no sum is
                if (any && m == -INFINITY && l == 0.f) l = -1.f;
                xch[((block & 1) * 2 + half) * kXaRows + t] = l;
                meet();
                if (!ok) break;
                tc_fence_after();
                l += xch[((block & 1) * 2 + (half ^ 1)) * kXaRows + t];
                meet();                                            // (the next segment's first maxima go to the same place)
            }
            if (blocks > 0 && warp_rows)
                add_set_aside<DP, T>(p, seg.it.row, seg.b, seg.kvh, row, mine ? seen : 0, m, half * (DP / 2), t_o, bads, key0, block, blocks,
                                     min(blocks, max(0, seen_lo - key0) / L::kBlock));
            const bool whole = seg.whole();
            // (a mark: the maximum is both halves', so the other's sum is 0 or a mark, too)
            PagedNorm norm = paged_norm(l < 0.f ? kPaOnlyInf : m, l < 0.f ? 0.f : l, p.scale);
            if (whole) norm = paged_whole(norm);
            float *part = p.part + (2LL * cta + (seg.blk0 == 0)) * L::kSlot;
            if (warp_rows) {
#pragma unroll
                for (int c = 0; c < DP / 64; ++c) {
                    uint32_t r[32];
                    if (blocks > 0) {
                        tmem_ld_32x32b_x32(t_o + 32 * c, r);
                        tmem_ld_wait_for(r);
                    } else {
#pragma unroll
                        for (int k = 0; k < 32; ++k) r[k] = 0;
                    }
                    const int d0 = half * (DP / 2) + 32 * c;       // this thread's first column of the 32
                    if (mine) {
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            float v[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(r[8 * g + k]) * norm.inv;
                            if (whole) {
                                paged_store<T>(p, seg.b, token, h, d0 / 8 + g, v);
                            } else {
                                float4 *dst = reinterpret_cast<float4 *>(part + t * DP + d0 + 8 * g);
                                dst[0] = make_float4(v[0], v[1], v[2], v[3]);
                                dst[1] = make_float4(v[4], v[5], v[6], v[7]);
                            }
                        }
                    }
                }
                if (mine && half == 0) {
                    if (whole) paged_store_lse(p, seg.b, token, h, norm.lse);
                    else part[L::kRows * DP + t] = norm.lse;
                }
            }
            if (tid == 0 && seg.blk0 == 0 && !whole) seg.describe(per);
        }
        if (!ok && lane == 0) xa_report(tp.status, kXaRolePagedSoftmax, 1);
    }
    __syncwarp();
    // All copies and products have been waited for, or a wait ran out.  Then those in flight are waited for here,
    // before shared and tensor memory are another CTA's.
    tc_fence_before();
    __syncthreads();
    if (*abort_flag && (warp == kPtLoadWarp || warp == kPtLoadWarp + 1) && lane == 0) {
        // the last copy into each stage of this warp's: every second one
        volatile int never = 0;
        constexpr int kOwn = L::kStages / 2;
        for (int s = 0; s < kOwn; ++s) {
            const int uses = (block - s + kOwn - 1) / kOwn;
            if (uses > 0) mbar_wait(full + 8 * (2 * s + warp - kPtLoadWarp), (uses - 1) & 1, &never);
        }
    }
    if (warp == kPtMmaWarp) {
        tc_fence_after();
        if (*abort_flag) xa_products_done(drain);
        tmem_dealloc(tmem, 512);
    }
}

}  // namespace cudallm
