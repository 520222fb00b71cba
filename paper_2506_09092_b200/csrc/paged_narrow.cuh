// Paged attention where up to 16 rows (query heads of a key head x new tokens) share a key head: single tokens, few drafts.
//
// Each warp has tiles, a ring of stages and sums of its own, in one line over the CTA's segments: when a segment's tiles are
// over, the next one's first two are asked for and its queries read before the warps' sums join, in the stage that
// is free, so that no segment begins with an empty ring (48 sequences of 1024 to 4096 states, 8 key heads of 128: 84 us, 6.1 TB/s;
// 128 of 250 to 1000: 63 us).  Three stages of two CTAs an SM: two stages and three CTAs were slower.  Short sequences
// are bound by what a segment takes besides its tiles, some 1700 instructions a warp (512 sequences of 200: 109 us for 65 of
// bytes).
#pragma once
#include "paged_attn.cuh"

namespace cudallm {

template <int DP> struct PagedNarrowSmem : PagedSizes<DP> {
    using S = PagedSizes<DP>;
    static constexpr int kRows = 16;
    static constexpr int kWarp = S::kStages * 2 * S::kTile;        // a warp's ring
    static_assert(kRows * DP * 4 <= 2 * S::kTile, "a warp's sums in a stage");
    static constexpr int kStats = S::kRing;                        // floats [warp][maxima, sums of exponentials][row]
    static constexpr int kShare = kStats + kPaWarps * 2 * kRows * 4;       // a CTA's result for its cluster: [row][DP] fp32, lse
    static constexpr int kBytes = kShare + kRows * (DP + 1) * 4;
    static_assert(2 * (kBytes + 1024) <= 228 * 1024, "two CTAs on an SM");
};

// Four columns (piece c) of row r of a warp's sums: neighbouring rows lie in different banks.
__device__ __forceinline__ int paged_sum_at(int dp, int r, int c) { return r * dp + ((c ^ (r & 7)) << 2); }

template <int DP, typename T>
__global__ void __launch_bounds__(kPaThreads, 2)
paged_narrow_kernel(const PagedParams p)
{
    using L = PagedNarrowSmem<DP>;
    using Loader = PagedLoader<DP, T>;
    using Segments = PagedSegments<L::kRows, L::kBlock>;
    constexpr int kChunks = DP / 8, kKeys = L::kKeys, kN = kKeys / 8;      // kN: tiles of eight keys
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q4 = lane & 3;
    grid_launch_dependents();
    grid_dependency_wait();

    Segments seg(p);
    long long per = 1;
    const int cta = blockIdx.x, rank = p.cluster ? cta % p.cluster : 0;
    if (!(p.cluster ? paged_cluster_segment(p, seg, rank) : seg.locate(smem, per))) return;

    const uint32_t ring = smem_u32(smem) + warp * L::kWarp;
    auto stage_at = [&](int stage) { return (uint32_t)(stage * 2 * L::kTile); };
    auto step = [](int stage) { return stage == L::kStages - 1 ? 0 : stage + 1; };
    // tiles of 16 or 32 keys of a segment: warp, warp + 4, ... are this warp's
    auto tiles_of = [&](const Segments &s) {
        const int keys = s.key_end() - s.key0();
        return keys > 0 ? (int)((unsigned)(keys + kKeys - 1) / (unsigned)kKeys) : 0;
    };
    auto mine_of = [&](int tiles) { return tiles > warp ? (tiles - warp + kPaWarps - 1) / kPaWarps : 0; };
    int turn = 0;                                                  // the stage that the segment's first tile goes to
    int tiles = tiles_of(seg), mine = mine_of(tiles);
    Loader ld(p, ring);
    ld.set(seg.it, seg.kvh, seg.key0() + warp * kKeys, seg.key_end(), mine);
    ld.look_up(0);
    uint32_t there[2] = {ld.load(0, stage_at(turn), L::kTile), 0};         // of the next two tiles
    there[1] = ld.load(1, stage_at(step(turn)), L::kTile);
    uint32_t qa[DP / 16][4];
    paged_load_q<DP, T>(p, seg.b, seg.kvh, seg.rt * L::kRows, seg.rows(), qa);

    for (;;) {
        Segments nxt = seg;                                        // the next segment, and its first tile's pages
        bool more = false;
        int page = -1, in_page = 0;
        if (!p.cluster) {
            more = nxt.next();
            if (more) {
                Loader first(p, ring);
                first.set(nxt.it, nxt.kvh, nxt.key0() + warp * kKeys, nxt.key_end(), mine_of(tiles_of(nxt)));
                first.look_up(0);
                page = first.page;
                in_page = first.in_page;
            }
        }
        const int rows = seg.rows(), seen_lo = seg.seen_lo();
        int seen[2];                                               // keys that a row sees lie below this
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        bool any[2] = {false, false};
        float o[DP / 8][4];
#pragma unroll
        for (int half = 0; half < 2; ++half)
            seen[half] = g + 8 * half < rows ? paged_seen(seg.it, paged_token(p, seg.rt * L::kRows + g + 8 * half)) : 0x7fffffff;
#pragma unroll
        for (int n = 0; n < DP / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] = 0.f;

        int stage = turn;
        for (int t = 0; t < mine; ++t) {
            cp_async_wait_group<1>();
            __syncwarp();                                          // every lane's copies of this stage have landed
            const uint32_t mask = there[0];
            there[0] = there[1];
            there[1] = ld.load(t + 2, stage_at(step(step(stage))), L::kTile);      // (its stage was read in the last round)
            const uint32_t sk = ring + stage_at(stage), sv = sk + L::kTile;
            stage = step(stage);
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
            const int pos0 = ld.first + t * L::kBlock;
            const bool full = mask == Loader::kAll && pos0 + kKeys <= seen_lo;     // every row sees every key
            if (!full) {
#pragma unroll
                for (int n = 0; n < kN; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = n * 8 + q4 * 2 + (e & 1);
                        if (!(mask >> key & 1) || pos0 + key >= seen[e >> 1]) s[n][e] = -INFINITY;
                    }
            }
            float bm[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float v = fmaxf(s[0][2 * half], s[0][2 * half + 1]);
#pragma unroll
                for (int n = 1; n < kN; ++n) v = fmaxf(v, fmaxf(s[n][2 * half], s[n][2 * half + 1]));
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
                bm[half] = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
                any[half] |= full || (mask & low_bits(seen[half] - pos0)) != 0;
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
            // (a row that has seen nothing yet: all its scores are -inf, and so are their differences to 0)
            const float neg[2] = {m[0] == -INFINITY ? 0.f : -m[0] * p.scale_log2, m[1] == -INFINITY ? 0.f : -m[1] * p.scale_log2};
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[n][e] = xa_exp2(fmaf(s[n][e], p.scale_log2, neg[e >> 1]));
                    l[e >> 1] += s[n][e];
                }
            // Keys that some of the rows do not see: 0 x a value that is not finite would reach those rows through
            // the product, so such a value's rows are added by hand and it becomes zero.
            uint32_t partly = full ? 0u : mask & ~low_bits(seen_lo - pos0);
            while (partly) {
                const int j = __ffs(partly) - 1;
                partly &= partly - 1;
                const uint32_t row = sv + j * DP * 2;
                const bool bad = lane < kChunks && any_not_finite<T>(ld_shared_v4(row + ((lane ^ (j & 7)) << 4)));
                if (!__any_sync(0xffffffffu, bad)) continue;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float w = 0.f;
#pragma unroll
                    for (int n = 0; n < kN; ++n)
                        w = select(n == j >> 3, select(j & 1, s[n][2 * half + 1], s[n][2 * half]), w);
                    w = __shfl_sync(0xffffffffu, w, (lane & ~3) | ((j & 7) >> 1));
                    if (pos0 + j < seen[half]) {
#pragma unroll
                        for (int n = 0; n < DP / 8; ++n) {
                            const float2 f = unpack2<T>(ld_shared_u32(row + ((n ^ (j & 7)) << 4) + q4 * 4));
                            o[n][2 * half] = fmaf(w, f.x, o[n][2 * half]);
                            o[n][2 * half + 1] = fmaf(w, f.y, o[n][2 * half + 1]);
                        }
                    }
                }
                __syncwarp();
                if (lane < kChunks) st_shared_v4_b32(row + (lane << 4), 0, 0, 0, 0);
                __syncwarp();
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
            __syncwarp();                                          // the stage has been read by every lane
        }
        // The next segment's first tiles and queries; the warps' sums join in the third stage, the same for all.
        int next_turn = turn;
        for (int k = (int)((unsigned)(tiles + kPaWarps - 1) / (unsigned)kPaWarps % (unsigned)L::kStages); k > 0; --k) next_turn = step(next_turn);
        const int joint = step(step(next_turn));
        if (more) {
            tiles = tiles_of(nxt);
            mine = mine_of(tiles);
            ld.set(nxt.it, nxt.kvh, nxt.key0() + warp * kKeys, nxt.key_end(), mine);
            ld.page = page;
            ld.in_page = in_page;
            there[0] = ld.load(0, stage_at(next_turn), L::kTile);
            there[1] = ld.load(1, stage_at(step(next_turn)), L::kTile);
            paged_load_q<DP, T>(p, nxt.b, nxt.kvh, nxt.rt * L::kRows, nxt.rows(), qa);
        }
        float *sums = reinterpret_cast<float *>(smem + warp * L::kWarp + stage_at(joint));
        float *stats = reinterpret_cast<float *>(smem + L::kStats);
#pragma unroll
        for (int n = 0; n < DP / 8; ++n) {
            *reinterpret_cast<float2 *>(sums + paged_sum_at(DP, g, 2 * n + (q4 >> 1)) + (q4 & 1) * 2) = make_float2(o[n][0], o[n][1]);
            *reinterpret_cast<float2 *>(sums + paged_sum_at(DP, g + 8, 2 * n + (q4 >> 1)) + (q4 & 1) * 2) = make_float2(o[n][2], o[n][3]);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            l[half] += __shfl_xor_sync(0xffffffffu, l[half], 1);
            l[half] += __shfl_xor_sync(0xffffffffu, l[half], 2);
            if (any[half] && m[half] == -INFINITY && l[half] == 0.f) m[half] = kPaOnlyInf;
            if (q4 == 0) {
                stats[warp * 2 * L::kRows + g + 8 * half] = m[half];
                stats[warp * 2 * L::kRows + L::kRows + g + 8 * half] = l[half];
            }
        }
        __syncthreads();
        // thread -> (row, 8 columns): the warps' sums, weighted to the common maximum.  Whole results leave at once, parts go to
        // the cluster's or the call's scratch.
        const bool whole = seg.whole() && p.cluster <= 1;
        float *slot = p.cluster ? reinterpret_cast<float *>(smem + L::kShare) : p.part + (2LL * cta + (seg.blk0 == 0)) * L::kRows * (DP + 1);
        for (int i = tid; i < rows * kChunks; i += kPaThreads) {
            const int r = i / kChunks, c = i % kChunks;
            float wm[kPaWarps], wl[kPaWarps], mx = -INFINITY, sum = 0.f, acc[8] = {};
#pragma unroll
            for (int w = 0; w < kPaWarps; ++w) {
                wm[w] = stats[w * 2 * L::kRows + r];
                wl[w] = stats[w * 2 * L::kRows + L::kRows + r];
                mx = fmaxf(mx, wm[w]);
            }
#pragma unroll
            for (int w = 0; w < kPaWarps; ++w) {
                if (wl[w] == 0.f && wm[w] == -INFINITY) continue;  // a warp without keys
                const float a = xa_exp2((wm[w] - mx) * p.scale_log2);
                sum = fmaf(a, wl[w], sum);
                const float *src = reinterpret_cast<const float *>(smem + w * L::kWarp + stage_at(joint));
                const float4 x = *reinterpret_cast<const float4 *>(src + paged_sum_at(DP, r, 2 * c));
                const float4 y = *reinterpret_cast<const float4 *>(src + paged_sum_at(DP, r, 2 * c + 1));
                acc[0] = fmaf(a, x.x, acc[0]); acc[1] = fmaf(a, x.y, acc[1]); acc[2] = fmaf(a, x.z, acc[2]); acc[3] = fmaf(a, x.w, acc[3]);
                acc[4] = fmaf(a, y.x, acc[4]); acc[5] = fmaf(a, y.y, acc[5]); acc[6] = fmaf(a, y.z, acc[6]); acc[7] = fmaf(a, y.w, acc[7]);
            }
            PagedNorm norm = paged_norm(mx, sum, p.scale);
            if (whole) norm = paged_whole(norm);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] *= norm.inv;
            if (whole) {
                const int row = seg.rt * L::kRows + r, t = paged_token(p, row), h = seg.kvh * p.group + row - t * p.group;
                paged_store<T>(p, seg.b, t, h, c, acc);
                if (c == 0) paged_store_lse(p, seg.b, t, h, norm.lse);
            } else {
                paged_store_part<DP, L::kRows>(slot, r, c, acc, norm.lse);
            }
        }
        if (tid == 0 && !p.cluster && seg.blk0 == 0 && !whole) seg.describe(per);
        if (!more) break;
        __syncthreads();                                           // the sums have been read
        seg = nxt;
        turn = next_turn;
    }
    cp_async_wait_group<0>();
    if (p.cluster > 1) paged_join_cluster<DP, T>(p, seg, smem_u32(smem) + L::kShare, rank);
}

}  // namespace cudallm
