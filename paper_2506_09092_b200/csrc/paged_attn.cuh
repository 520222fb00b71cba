// Attention of the newest tokens of each sequence over its pages, and writing their keys and values there.
//
// O = softmax(scale Q K^T) V with a running maximum m, a sum l of exponentials and an unnormalised O per row: one pass over the keys,
// o <- o 2^((m - m') s) + P V.  Parts of the keys join by their lse: -inf for a part without keys, kPaOnlyInf for one
// whose scores are all -inf.  Its weight beside any other part is zero, too, but if there are only such parts the row is no number
// (0 / 0), where a row without keys is zero.
//
// Scores, maxima, sums and O are fp32 throughout.  The probabilities alone are rounded to the operands' 16 bits, since the tensor core
// multiplies them with V: half a step each, relative to themselves, which an average over many keys mostly evens out (48 sequences, bf16:
// O is off by 2.2e-3 of itself against 64 bits, 1.7e-3 of it its own rounding; fp16, 16 sequences: 2.9e-4 and 2.1e-4).
//
// Bound: HBM (K and V of every sequence are read once; 16 or 32 rows of arithmetic per key are far below
// any pipe's rate), so what matters is bytes in flight and an even split.  The rows that share a key head (query heads x new
// tokens) share its reading.  Up to 16 of them are one tile of mma.sync.m16n8k16 (paged_narrow.cuh: 4 sequences of 64000 states,
// 8 key heads of 128, 4 rows: 160 us for 1.05 GB, at the copy rate; 16 rows need a tenth of mma.sync's rate at the full speed of
// HBM, and a tcgen05 tile would be 128 rows, most of them empty).  More are tiles of 128 on tcgen05 (paged_tile.cuh) if TMA can
// bring the pages, else two to four tiles of 16 that share their stages (paged_wide_kernel, here).
//
// The mma.sync kernels' CTAs have four warps, each with its own tiles of 32 keys (16 at head dims above 64) in a ring of
// cp.async stages, 96 KiB a CTA and two CTAs an SM.  A lane looks up the page of "its" row of the next tile one tile ahead, and
// the rows' offsets go round by shuffle, so pages may have any number of rows.
//
// Only the device knows the lengths, so the split is made there, in one of two ways:
//  * a cluster of CTAs per (item, key head, row tile), each with an equal share of its keys; they join
//    through each other's shared memory.  One launch, but as long as the longest sequence takes (plan_attn has
//    the rule and both sides' times).
//  * equal shares: all blocks of keys of all items in one line, cut into equal pieces, as many as CTAs fit for
//    every key head.  Neighbouring CTAs have the same piece for the different heads: where the heads of a token lie side by
//    side they read the same DRAM pages at the same time (32 x 64000 keys of 64, a CTA's piece in a line that
//    ran through the heads, too: 101 us against 86).  A piece may begin and end inside an item; such parts go to scratch
//    (two slots a CTA) and paged_join_kernel adds them up in order.
#pragma once
#include "fast_div.cuh"
#include "mma_sync.cuh"
#include "xattn_common.cuh"

namespace cudallm {

constexpr int kPaWarps = 4;
constexpr int kPaThreads = 32 * kPaWarps;
constexpr int kPaCluster = 8;
constexpr float kPaOnlyInf = -3.402823466e38f;         // the lowest number: e to its power is zero, its difference to itself not

struct PagedStrides { long long page, row, head; };

struct PagedParams {
    const void *q, *k, *v;
    void *o;
    float *lse;
    float *part;                               // equal shares: parts' results, two slots a CTA ...
    int *desc;                                 // ... and kPaDesc words a CTA
    const int *table, *lens, *slot_of, *new_lens;
    XaStrides sq, so;
    PagedStrides sk, sv;
    long long table_stride;
    int batch, q_rows, q_heads, kv_heads, group, head_dim;
    FastDiv by_group;
    int pages, page_rows, slots, cap;          // cap: states that a row of the table holds
    FastDiv by_page_rows;
    int row_tiles;                             // tiles of 16 to 128 rows of an item and key head at most
    int cluster;                               // CTAs per item, key head and row tile; 0: equal shares
    int shares;                                // of a key head; CTA = share * kv_heads + key head
    // who counts what (locate): items a thread, or 2^count_shift threads an item, count_tiles row tiles each
    int count_items, count_shift, count_tiles;
    float scale, scale_log2;
};
constexpr int kPaDesc = 4;                     // parts (0: none begins here) and 2^16 x rows, item, key head, row tile

template <int DP> struct PagedSizes {
    static constexpr int kKeys = DP == 128 ? 16 : 32;              // of a stage and warp
    static constexpr int kBlock = kKeys * kPaWarps;                // of a round of the four warps: unit of the split
    static constexpr int kStages = 3;                              // 96 KiB a CTA: two on an SM
    static constexpr int kTile = kKeys * DP * 2;                   // a warp's one of K, V
    static constexpr int kRing = kPaWarps * kStages * 2 * kTile;
};
// Two to four row tiles.
template <int DP, int MT> struct PagedSmem : PagedSizes<DP> {
    using S = PagedSizes<DP>;
    static constexpr int kRows = 16 * MT;
    // the result of the walk: [row][DP] fp32, the rows' maxima, their sums
    static constexpr int kPitch = DP + 4;                          // floats per row
    static constexpr int kPart = (kRows * kPitch + 2 * kRows) * 4;
    // a CTA's result for its cluster: [row][DP] fp32, then the rows' lse
    static constexpr int kShare = (kPart + 127) / 128 * 128;
    static_assert(kShare + kRows * (DP + 1) * 4 <= S::kRing, "behind the result");
    static constexpr bool kQInSmem = MT > 3;                       // queries of four row tiles do not fit into registers
    static constexpr int kMax = S::kRing + (kQInSmem ? kRows * DP * 2 : 0);    // warps' maxima of each row
    static constexpr int kBytes = kMax + kRows * kPaWarps * 4;
    static_assert(2 * (kBytes + 1024) <= 228 * 1024, "two CTAs on an SM");
};

// An item: its row of the table, its states, its new tokens (0: none, or the item is not there).
struct PagedItem { const int *row; int len, news; };
__device__ __forceinline__ PagedItem paged_item(const int *table, long long stride, const int *lens, const int *slot_of,
                                                const int *new_lens, int b, int slots, int cap, int q_rows)
{
    const int slot = slot_of ? slot_of[b] : b;
    if ((unsigned)slot >= (unsigned)slots) return PagedItem{table, 0, 0};
    const int len = min(max(lens[slot], 0), cap);
    const int news = new_lens ? min(max(new_lens[b], 0), q_rows) : q_rows;
    return PagedItem{table + slot * stride, len, news};
}
__device__ __forceinline__ PagedItem paged_item(const PagedParams &p, int b)
{
    return paged_item(p.table, p.table_stride, p.lens, p.slot_of, p.new_lens, b, p.slots, p.cap, p.q_rows);
}
// States that token t sees; states that a row tile's last token sees; its blocks of keys (at least one, so that
// somebody writes the result; none without rows).
__device__ __forceinline__ int paged_seen(const PagedItem &it, int t) { return max(it.len - it.news + t + 1, 0); }
__device__ __forceinline__ int paged_token(const PagedParams &p, int row) { return (int)fast_div((uint32_t)row, p.by_group); }
__device__ __forceinline__ int paged_tile_seen(const PagedParams &p, const PagedItem &it, int rows, int rt)
{
    return paged_seen(it, paged_token(p, min(it.news * p.group, (rt + 1) * rows) - 1));
}
__device__ __forceinline__ int paged_blocks(const PagedParams &p, const PagedItem &it, int rows, int rt, int block)
{
    if (rt * rows >= it.news * p.group) return 0;
    return max(1, (int)((unsigned)(paged_tile_seen(p, it, rows, rt) + block - 1) / (unsigned)block));
}

// (as an instruction: a choice among registers must not become an address into a copy of them in local memory)
__device__ __forceinline__ float select(bool first, float a, float b)
{
    float r;
    asm("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %3, 0;\n\tselp.f32 %0, %1, %2, p;\n\t}" : "=f"(r) : "f"(a), "f"(b), "r"((int)first));
    return r;
}

// The lowest n bits.
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1; }

template <typename T> __device__ __forceinline__ bool any_not_finite(uint4 v);
template <> __device__ __forceinline__ bool any_not_finite<__nv_bfloat16>(uint4 v)
{
    bool bad = false;
    for (uint32_t w : {v.x, v.y, v.z, v.w}) bad |= (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
    return bad;
}
template <> __device__ __forceinline__ bool any_not_finite<__half>(uint4 v)
{
    bool bad = false;
    for (uint32_t w : {v.x, v.y, v.z, v.w}) bad |= (w & 0x7C00u) == 0x7C00u || (w & 0x7C000000u) == 0x7C000000u;
    return bad;
}
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr)
{
    uint4 w;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(addr) : "memory");
    return w;
}
__device__ __forceinline__ uint32_t ld_shared_u32(uint32_t addr)
{
    uint32_t w;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(addr) : "memory");
    return w;
}
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w)
{
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}

// Eight columns of a row of the result, rounded once.
template <typename T>
__device__ __forceinline__ void paged_store(const PagedParams &p, int b, int t, int h, int c, const float (&v)[8])
{
    if (c * 8 < p.head_dim)
        *reinterpret_cast<uint4 *>(static_cast<T *>(p.o) + b * p.so.b + t * p.so.r + h * p.so.h + c * 8) =
            make_uint4(XaElem<T>::pack(v[0], v[1]), XaElem<T>::pack(v[2], v[3]), XaElem<T>::pack(v[4], v[5]),
                       XaElem<T>::pack(v[6], v[7]));
}
__device__ __forceinline__ void paged_store_lse(const PagedParams &p, int b, int t, int h, float lse)
{
    if (p.lse) p.lse[((long long)b * p.q_heads + h) * p.q_rows + t] = lse;
}

// A warp's rows of the stages of a ring: pages looked up one tile ahead, copies past L1.  The pieces of a row go to
// neighbouring lanes, piece c of row r to position c ^ (r & 7) (conflict-free ldmatrix).
template <int DP, typename T> struct PagedLoader {
    using L = PagedSizes<DP>;
    static constexpr int kChunks = DP / 8, kRowStep = 32 / kChunks;        // 16-byte pieces of a row; rows that a copy instruction covers
    static constexpr uint32_t kAll = L::kKeys == 32 ? 0xffffffffu : (1u << L::kKeys) - 1;
    const PagedParams &p;
    const T *kbase, *vbase;
    const int *row;
    uint32_t to;                               // this warp's rows of K in stage 0
    int first, key_end, tiles, lane;           // the warp's tile t begins at key first + t * kBlock
    int page = -1, in_page = 0;                // this lane's row of the next tile

    __device__ __forceinline__ PagedLoader(const PagedParams &p_, uint32_t to_) : p(p_), to(to_), lane(threadIdx.x & 31) {}
    // From now on the warp's tiles of these keys; no page has been looked up.
    __device__ __forceinline__ void set(const PagedItem &it, int kvh, int first_, int key_end_, int tiles_)
    {
        kbase = static_cast<const T *>(p.k) + kvh * p.sk.head;
        vbase = static_cast<const T *>(p.v) + kvh * p.sv.head;
        row = it.row;
        first = first_;
        key_end = key_end_;
        tiles = tiles_;
    }
    __device__ __forceinline__ void look_up(int t)
    {
        page = -1;
        const int pos = first + t * L::kBlock + (lane & (L::kKeys - 1));
        if (t < tiles && pos < key_end) {
            const int col = (int)fast_div((uint32_t)pos, p.by_page_rows);
            in_page = pos - col * p.page_rows;
            page = row[col];
        }
    }
    // Tile t to stage `stage` bytes behind stage 0, values `values` bytes behind the keys.  Returns which rows are
    // there; the others become zeros.
    __device__ __forceinline__ uint32_t load(int t, uint32_t stage, uint32_t values)
    {
        uint32_t mask = 0;
        if (t < tiles) {
            const int lc = lane % kChunks, lr = lane / kChunks;
            const bool lc_live = lc * 8 < p.head_dim, ok = (unsigned)page < (unsigned)p.pages;
            const bool same = p.sk.page == p.sv.page && p.sk.row == p.sv.row;
            mask = __ballot_sync(0xffffffffu, ok) & kAll;
            const long long off_k = ok ? page * p.sk.page + in_page * p.sk.row : 0;
            const long long off_v = ok && !same ? page * p.sv.page + in_page * p.sv.row : 0;
            look_up(t + 1);
#pragma unroll
            for (int n = 0; n < L::kKeys / kRowStep; ++n) {
                const int r = lr + n * kRowStep;
                const uint32_t bytes = lc_live && (mask >> r & 1) ? 16 : 0;
                const uint32_t dst = to + stage + r * DP * 2 + ((lc ^ (r & 7)) << 4);
                const long long at_k = __shfl_sync(0xffffffffu, off_k, r);
                const long long at_v = same ? at_k : __shfl_sync(0xffffffffu, off_v, r);
                const int col = lc_live ? lc * 8 : 0;
                cp_async_16_cg(dst, kbase + at_k + col, bytes);
                cp_async_16_cg(dst + values, vbase + at_v + col, bytes);
            }
        }
        cp_async_commit();
        return mask;
    }
};

// Row r of a row tile: token (rt * kRows + r) / group, query head (rt * kRows + r) % group of the key head.
template <typename T>
__device__ __forceinline__ const T *paged_q_row(const PagedParams &p, int b, int kvh, int row)
{
    const int t = paged_token(p, row), h = row - t * p.group;
    return static_cast<const T *>(p.q) + b * p.sq.b + t * p.sq.r + (long long)(kvh * p.group + h) * p.sq.h;
}
// The A operands of 16 rows from `row` on (up to `rows`): rows g and g + 8, columns 2 q, 2 q + 1 and + 8 of every 16.
template <int DP, typename T>
__device__ __forceinline__ void paged_load_q(const PagedParams &p, int b, int kvh, int row, int rows, uint32_t (&qa)[DP / 16][4])
{
    const int g = (threadIdx.x & 31) >> 2, q4 = threadIdx.x & 3;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const T *src = g + 8 * half < rows ? paged_q_row<T>(p, b, kvh, row + g + 8 * half) : nullptr;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
                const int d = k * 16 + hi * 8 + q4 * 2;
                qa[k][half + 2 * hi] = (src && d < p.head_dim) ? *reinterpret_cast<const uint32_t *>(src + d) : 0u;
            }
    }
}

// Blocks blk0 .. blk1 - 1 of an item's keys for one key head and row tile.  Leaves sums, not yet normalised, at the start of
// shared memory: rows x DP, then the rows' maxima (of the scores), then the sums of exponentials.  A row that has
// seen no state has maximum -inf and sum 0, one whose scores are all -inf the maximum kPaOnlyInf.
//
// Two to four row tiles: registers do not hold a whole result per warp, so the warps share a stage.  Each takes its
// own keys' scores for all rows (S = Q K^T), they agree on the rows' maxima, the probabilities go to shared memory (where the
// stage's keys were), and each multiplies all of them with its own quarter of the columns of V.  Two
// barriers a stage.  Bound by issue slots and those barriers (16 sequences of 16000 states, 4 key heads of 128, 40 rows: 132 us where
// the tcgen05 kernel takes 98), so it serves pages that TMA cannot bring into tiles, and short tables of up to 32 rows.
template <int DP, int MT, typename T>
__device__ __forceinline__ void paged_walk_wide(const PagedParams &p, uint8_t *smem, const PagedItem &it, int b, int kvh, int rt,
                                                int blk0, int blk1)
{
    using L = PagedSmem<DP, MT>;
    using Loader = PagedLoader<DP, T>;
    constexpr int kKeys = L::kKeys, kN = kKeys / 8, kChunks = DP / 8;
    constexpr int kAllTile = kPaWarps * L::kTile, kStage = 2 * kAllTile;   // a stage: all warps' keys, all warps' values
    constexpr int kProb = L::kBlock * 2;                           // bytes of a row of probabilities
    constexpr int kSlice = DP / kPaWarps / 8;                      // 8-column tiles of V that a warp multiplies with
    static_assert(L::kRows * kProb <= kAllTile, "where the keys were");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rows = min(it.news * p.group - rt * L::kRows, L::kRows);
    const int seen_lo = paged_seen(it, paged_token(p, rt * L::kRows));
    const int key0 = blk0 * L::kBlock, key_end = min(paged_tile_seen(p, it, L::kRows, rt), blk1 * L::kBlock);
    const int tiles = key_end > key0 ? (key_end - key0 + L::kBlock - 1) / L::kBlock : 0;
    const uint32_t ring = smem_u32(smem), maxima = ring + L::kMax;
    Loader ld(p, ring + warp * L::kTile);
    ld.set(it, kvh, key0 + warp * kKeys, key_end, tiles);
    ld.look_up(0);
    uint32_t there[L::kStages - 1];
#pragma unroll
    for (int t = 0; t < L::kStages - 1; ++t) there[t] = ld.load(t, t * kStage, kAllTile);

    const int g = lane >> 2, q4 = lane & 3;
    uint32_t qa[L::kQInSmem ? 1 : MT][DP / 16][4];
    const uint32_t qs = ring + L::kRing;
    if constexpr (!L::kQInSmem) {
#pragma unroll
        for (int i = 0; i < MT; ++i) paged_load_q<DP, T>(p, b, kvh, rt * L::kRows + i * 16, rows - i * 16, qa[i]);
    } else {
        for (int i = tid; i < L::kRows * kChunks; i += kPaThreads) {
            const int r = i / kChunks, c = i % kChunks;
            uint4 w = make_uint4(0, 0, 0, 0);
            if (r < rows && c * 8 < p.head_dim)
                w = *reinterpret_cast<const uint4 *>(paged_q_row<T>(p, b, kvh, rt * L::kRows + r) + c * 8);
            st_shared_v4_b32(qs + r * DP * 2 + ((c ^ (r & 7)) << 4), w.x, w.y, w.z, w.w);
        }
        __syncthreads();
    }
    int seen[MT][2];
    float m[MT][2], l[MT][2], o[MT][kSlice][4];
    bool any[MT][2];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int r = i * 16 + g + 8 * half;
            seen[i][half] = r < rows ? paged_seen(it, paged_token(p, rt * L::kRows + r)) : 0x7fffffff;
            m[i][half] = -INFINITY;
            l[i][half] = 0.f;
            any[i][half] = false;
        }
#pragma unroll
        for (int n = 0; n < kSlice; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][n][e] = 0.f;
    }

    for (int t = 0; t < tiles; ++t) {
        cp_async_wait_group<L::kStages - 2>();
        __syncwarp();                                              // this warp's rows of stage t have landed
        const uint32_t stage = ring + (t % L::kStages) * kStage, sk = stage + warp * L::kTile, sv = sk + kAllTile;
        const uint32_t mask = there[0];
        float s[MT][kN][4] = {};
        {
            const int idx = lane >> 3, kr = (idx >> 1) * 8 + (lane & 7);
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) {
                uint32_t a[MT][4];
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if constexpr (!L::kQInSmem) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) a[i][e] = qa[i][k][e];
                    } else {
                        const int r = i * 16 + (lane & 15);
                        ldmatrix_x4(a[i], qs + r * DP * 2 + (((2 * k + (lane >> 4)) ^ (r & 7)) << 4));
                    }
                }
#pragma unroll
                for (int n = 0; n < kN; n += 2) {
                    uint32_t bf[4];
                    ldmatrix_x4(bf, sk + (n * 8 + kr) * DP * 2 + (((2 * k + (idx & 1)) ^ (kr & 7)) << 4));
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        mma_16x8x16<T>(s[i][n], a[i], bf[0], bf[1]);
                        mma_16x8x16<T>(s[i][n + 1], a[i], bf[2], bf[3]);
                    }
                }
            }
        }
        const int pos0 = ld.first + t * L::kBlock;
        const bool full = mask == Loader::kAll && pos0 + kKeys <= seen_lo;     // every row sees every key
        if (!full) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int n = 0; n < kN; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = n * 8 + q4 * 2 + (e & 1);
                        if (!(mask >> key & 1) || pos0 + key >= seen[i][e >> 1]) s[i][n][e] = -INFINITY;
                    }
        }
        // values that are not finite of keys that some of the rows do not see (see below)
        bool bad = false;
        for (uint32_t partly = full ? 0u : mask & ~low_bits(seen_lo - pos0); partly; partly &= partly - 1)
            bad |= lane < kChunks && any_not_finite<T>(ld_shared_v4(sv + (__ffs(partly) - 1) * DP * 2 + (lane << 4)));
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float v = fmaxf(s[i][0][2 * half], s[i][0][2 * half + 1]);
#pragma unroll
                for (int n = 1; n < kN; ++n) v = fmaxf(v, fmaxf(s[i][n][2 * half], s[i][n][2 * half + 1]));
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
                any[i][half] |= full || (mask & low_bits(seen[i][half] - pos0)) != 0;
                if (q4 == 0)
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(maxima + (i * 16 + g + 8 * half) * 16 + warp * 4), "f"(v) : "memory");
            }
        bad = __syncthreads_or(bad);                               // all have read the stage's keys, and stage t - 1 to its end
#pragma unroll
        for (int i = 0; i + 1 < L::kStages - 1; ++i) there[i] = there[i + 1];
        const int next = t + L::kStages - 1;
        there[L::kStages - 2] = ld.load(next, next % L::kStages * kStage, kAllTile);
        float nm[MT][2];
        bool more = false;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint4 w = ld_shared_v4(maxima + (i * 16 + g + 8 * half) * 16);
                nm[i][half] = fmaxf(m[i][half], fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)),
                                                      fmaxf(__uint_as_float(w.z), __uint_as_float(w.w))));
                more |= nm[i][half] > m[i][half];
            }
        if (__any_sync(0xffffffffu, more)) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                float alpha[2];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    alpha[half] = nm[i][half] == m[i][half] ? 1.f : xa_exp2((m[i][half] - nm[i][half]) * p.scale_log2);
                    m[i][half] = nm[i][half];
                    l[i][half] *= alpha[half];
                }
#pragma unroll
                for (int n = 0; n < kSlice; ++n) {
                    o[i][n][0] *= alpha[0];
                    o[i][n][1] *= alpha[0];
                    o[i][n][2] *= alpha[1];
                    o[i][n][3] *= alpha[1];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const float neg[2] = {m[i][0] == -INFINITY ? 0.f : -m[i][0] * p.scale_log2,
                                  m[i][1] == -INFINITY ? 0.f : -m[i][1] * p.scale_log2};
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float p0 = xa_exp2(fmaf(s[i][n][2 * half], p.scale_log2, neg[half]));
                    const float p1 = xa_exp2(fmaf(s[i][n][2 * half + 1], p.scale_log2, neg[half]));
                    l[i][half] += p0 + p1;
                    const int r = i * 16 + g + 8 * half;
                    asm volatile("st.shared.b32 [%0], %1;"
                                 ::"r"(stage + r * kProb + (((warp * kN + n) ^ (r & 7)) << 4) + q4 * 4), "r"(XaElem<T>::pack(p0, p1)) : "memory");
                }
        }
        __syncthreads();                                           // the probabilities are there
        // 0 x a value that is not finite would reach rows that do not see it through the product: such a value is
        // added by hand where it is seen, and becomes zero.  (A warp reads and clears its own columns only.)
        if (bad) {
            const int tile0 = key0 + t * L::kBlock;
            for (int j = max(seen_lo - tile0, 0); j < L::kBlock; ++j) {
                const uint32_t row = stage + kAllTile + j * DP * 2, own = row + (((warp * kSlice + lane) ^ (j & 7)) << 4);
                if (!__any_sync(0xffffffffu, lane < kSlice && any_not_finite<T>(ld_shared_v4(lane < kSlice ? own : row)))) continue;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int r = i * 16 + g + 8 * half;
                        const float2 both = unpack2<T>(ld_shared_u32(stage + r * kProb + (((j >> 3) ^ (r & 7)) << 4) + (j & 6) * 2));
                        const float weight = j & 1 ? both.y : both.x;
                        if (tile0 + j < seen[i][half]) {
#pragma unroll
                            for (int n = 0; n < kSlice; ++n) {
                                const float2 f = unpack2<T>(ld_shared_u32(row + (((warp * kSlice + n) ^ (j & 7)) << 4) + q4 * 4));
                                o[i][n][2 * half] = fmaf(weight, f.x, o[i][n][2 * half]);
                                o[i][n][2 * half + 1] = fmaf(weight, f.y, o[i][n][2 * half + 1]);
                            }
                        }
                    }
                __syncwarp();
                if (lane < kSlice) st_shared_v4_b32(own, 0, 0, 0, 0);
                __syncwarp();
            }
        }
        {
            const int idx = lane >> 3, kr = (idx & 1) * 8 + (lane & 7);
#pragma unroll
            for (int k = 0; k < L::kBlock / 16; ++k) {
                uint32_t a[MT][4];
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const int r = i * 16 + (lane & 15);
                    ldmatrix_x4(a[i], stage + r * kProb + (((2 * k + (lane >> 4)) ^ (r & 7)) << 4));
                }
#pragma unroll
                for (int n = 0; n < kSlice; n += 2) {
                    uint32_t bf[4];
                    ldmatrix_x4_trans(bf, stage + kAllTile + (k * 16 + kr) * DP * 2 + (((warp * kSlice + n + (idx >> 1)) ^ (kr & 7)) << 4));
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        mma_16x8x16<T>(o[i][n], a[i], bf[0], bf[1]);
                        mma_16x8x16<T>(o[i][n + 1], a[i], bf[2], bf[3]);
                    }
                }
            }
        }
    }
    cp_async_wait_group<0>();
    __syncthreads();                                               // the ring is free
    float *jo = reinterpret_cast<float *>(smem), *jm = jo + L::kRows * L::kPitch, *jl = jm + L::kRows;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
        for (int n = 0; n < kSlice; ++n) {
            float *at = jo + (i * 16 + g) * L::kPitch + (warp * kSlice + n) * 8 + q4 * 2;
            *reinterpret_cast<float2 *>(at) = make_float2(o[i][n][0], o[i][n][1]);
            *reinterpret_cast<float2 *>(at + 8 * L::kPitch) = make_float2(o[i][n][2], o[i][n][3]);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            l[i][half] += __shfl_xor_sync(0xffffffffu, l[i][half], 1);
            l[i][half] += __shfl_xor_sync(0xffffffffu, l[i][half], 2);
            // scores of -inf alone are not the same as no scores: a mark that no sum is
            if (any[i][half] && m[i][half] == -INFINITY && l[i][half] == 0.f) l[i][half] = -1.f;
            if (q4 == 0)
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(maxima + (i * 16 + g + 8 * half) * 16 + warp * 4), "f"(l[i][half]) : "memory");
            if (q4 == 0 && warp == 0) jm[i * 16 + g + 8 * half] = m[i][half];
        }
    }
    __syncthreads();
    if (tid < L::kRows) {
        const uint4 w = ld_shared_v4(maxima + tid * 16);
        const float sum = (__uint_as_float(w.x) + __uint_as_float(w.y)) + (__uint_as_float(w.z) + __uint_as_float(w.w));
        jl[tid] = sum < 0.f ? 0.f : sum;                           // (marks: the maximum is the CTA's, so the other warps' sums are 0)
        if (sum < 0.f) jm[tid] = kPaOnlyInf;
    }
    __syncthreads();
}

// Equal shares: for each key head all blocks of keys in one line, items in order, in each the row tiles; a CTA's share of it in
// pieces (segments) that each belong to one item and row tile.  Every row tile has kPaStart units in the line before its
// blocks: what beginning and ending a segment costs, in blocks.  One number for all kernels, although their blocks differ (us with
// 0, 1, 2, 3.  One new token on 8 key heads, 128 sequences of 250 to 1000 states: heads of 128 70.0, 66.8, 63.1, 62.4, of 64
// 45.2, 41.4, 39.8, 39.6; 48 of 1024 to 4096: 87.5, 87.8, 83.8, 83.4 and 50.5, 48.3, 48.4, 48.4.  Tiles, 40 rows on 4 key heads, 128 of
// 300 to 1200: heads of 128 67.4, 62.8, 61.6, 60.4, of 64 57.4, 52.5, 52.9, 53.4; 48 of 1024 to 4096: 60.8, 59.1, 58.6, 58.1 and 53.0,
// 51.9, 53.2, 53.1).
constexpr int kPaStart = 3;
template <int ROWS, int BLOCK> struct PagedSegments {
    const PagedParams &p;
    long long pos, end;                        // in units: behind the segment, the share's end
    int at;                                    // behind the segment, of its row tile
    PagedItem it;
    int b, kvh, rt, blk0, blk1, blocks;        // blocks: of the item and row tile

    __device__ __forceinline__ explicit PagedSegments(const PagedParams &p_) : p(p_) {}
    PagedSegments(const PagedSegments &) = default;
    __device__ __forceinline__ PagedSegments &operator=(const PagedSegments &s)        // (of the same call)
    {
        pos = s.pos; end = s.end; at = s.at;
        it = s.it;
        b = s.b; kvh = s.kvh; rt = s.rt; blk0 = s.blk0; blk1 = s.blk1; blocks = s.blocks;
        return *this;
    }
    __device__ __forceinline__ static int units(int blocks) { return blocks > 0 ? blocks + kPaStart : 0; }
    __device__ __forceinline__ void enter(int b_, int rt_)
    {
        if (b_ != b) it = paged_item(p, b_);
        b = b_;
        rt = rt_;
        at = 0;
        blocks = paged_blocks(p, it, ROWS, rt, BLOCK);
    }
    __device__ __forceinline__ static long long divide(long long a, long long d)
    {
        return (a | d) >> 32 ? a / d : (long long)((unsigned)a / (unsigned)d);
    }
    // The next segment; false: there are no more.
    __device__ __forceinline__ bool next()
    {
        while (pos < end) {
            const int own = units(blocks);
            if (at < own) {
                const int upto = (int)min((long long)own, at + (end - pos));
                blk0 = max(at - kPaStart, 0);
                blk1 = max(upto - kPaStart, 0);
                pos += upto - at;
                at = upto;
                if (blk1 > blk0) return true;
            } else if (rt + 1 < p.row_tiles && blocks > 0) {
                enter(b, rt + 1);
            } else {
                enter(b + 1, 0);                                   // (there is one: the share has units left)
            }
        }
        return false;
    }
    // How many units there are in all, and where this CTA's share begins: each of the first 128 threads counts the row tiles of
    // some items, or some of the row tiles of one, and the one that has found the place makes out the first segment (and
    // whether there is one, which it returns).  All of the CTA's threads call it; `smem` is free again afterwards.
    // per: units of a share.
    __device__ __forceinline__ bool locate(uint8_t *smem, long long &per)
    {
        struct Found {
            long long pos, end, per;
            PagedItem it;
            int at, b, rt, blk0, blk1, blocks, some;
        };
        long long *warp_sum = reinterpret_cast<long long *>(smem);
        Found &found = *reinterpret_cast<Found *>(warp_sum + kPaWarps);
        const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, each = p.count_items, tiles = p.count_tiles;
        const int b0 = (tid >> p.count_shift) * each, rt0 = (tid & ((1 << p.count_shift) - 1)) * tiles;
        long long sum = 0, upto = 0;
        b = -1;
        if (tid < kPaThreads) {
            for (int i = b0; i < min(b0 + each, p.batch); ++i)
                for (int r = rt0; r < min(rt0 + tiles, p.row_tiles); ++r) {
                    enter(i, r);
                    if (blocks == 0) break;
                    sum += units(blocks);
                }
            upto = sum;                                            // units of all threads up to this one
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const long long v = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += v;
            }
            if (lane == 31) warp_sum[warp] = upto;
        }
        if (tid == 0) {
            found.some = 0;                                        // (unless one of the threads finds its place)
            p.desc[blockIdx.x * kPaDesc] = 0;
        }
        __syncthreads();
        if (tid < kPaThreads) {
            long long total = 0;
#pragma unroll
            for (int w = 0; w < kPaWarps; ++w) {
                if (w < warp) upto += warp_sum[w];
                total += warp_sum[w];
            }
            per = max(divide(total + p.shares - 1, p.shares), 1LL);
            pos = (blockIdx.x / (unsigned)p.kv_heads) * per;
            end = min(total, pos + per);
            long long rem = pos - (upto - sum);
            if (pos < end && rem >= 0 && rem < sum) {
                if (each > 1 || tiles > 1)                         // (else it has entered its only one)
                    for (enter(b0, rt0); rem >= units(blocks);) {
                        rem -= units(blocks);
                        if (rt + 1 < min(rt0 + tiles, p.row_tiles) && blocks > 0) enter(b, rt + 1);
                        else enter(b + 1, rt0);
                    }
                at = (int)rem;
                const bool some = next();
                found = Found{pos, end, per, it, at, b, rt, blk0, blk1, blocks, some};
            }
        }
        __syncthreads();
        const Found f = found;
        pos = f.pos;
        end = f.end;
        at = f.at;
        per = f.per;
        it = f.it;
        b = f.b;
        kvh = (int)(blockIdx.x % (unsigned)p.kv_heads);
        rt = f.rt;
        blk0 = f.blk0;
        blk1 = f.blk1;
        blocks = f.blocks;
        __syncthreads();
        return f.some;
    }
    __device__ __forceinline__ int rows() const { return min(it.news * p.group - rt * ROWS, ROWS); }
    __device__ __forceinline__ int key0() const { return blk0 * BLOCK; }
    __device__ __forceinline__ int key_end() const { return min(paged_tile_seen(p, it, ROWS, rt), blk1 * BLOCK); }
    // blocks that hold keys (a row tile that sees nothing has one that holds none)
    __device__ __forceinline__ int live() const { return (int)((unsigned)max(0, key_end() - key0() + BLOCK - 1) / (unsigned)BLOCK); }
    // keys below this are seen by every row
    __device__ __forceinline__ int seen_lo() const { return paged_seen(it, paged_token(p, rt * ROWS)); }
    __device__ __forceinline__ bool whole() const { return blk0 == 0 && blk1 == blocks; }
    // The first of several parts of an item, key head and row tile says how many CTAs share them: every kv_heads-th from here.
    __device__ __forceinline__ void describe(long long per) const
    {
        int *d = p.desc + blockIdx.x * kPaDesc;
        d[0] = ((int)divide(pos - blk1 + blocks - 1, per) - (int)(blockIdx.x / (unsigned)p.kv_heads) + 1) | rows() << 16;
        d[1] = b;
        d[2] = kvh;
        d[3] = rt;
    }
};

// 1 / sum and lse of a row, or of a part of it.
struct PagedNorm { float inv, lse; };
__device__ __forceinline__ PagedNorm paged_norm(float m, float sum, float scale)
{
    if (sum != 0.f) return PagedNorm{1.f / sum, fmaf(m, scale, logf(sum))};
    return PagedNorm{0.f, m == kPaOnlyInf ? kPaOnlyInf : -INFINITY};
}
// ... of a whole row: scores of -inf alone are no number.
__device__ __forceinline__ PagedNorm paged_whole(PagedNorm n)
{
    const float nan = __int_as_float(0x7fc00000);
    return n.lse == kPaOnlyInf ? PagedNorm{nan, nan} : n;
}
// ... of a row joined from parts, of which `mx` is the largest lse and `sum` the sum of their weights.
__device__ __forceinline__ PagedNorm paged_joined(float mx, float sum)
{
    return sum == 0.f ? PagedNorm{0.f, -INFINITY} : paged_whole(PagedNorm{1.f / sum, mx == kPaOnlyInf ? kPaOnlyInf : mx + logf(sum)});
}

// A row's eight columns (c), normalised, as a part of the result: row r of [row][DP] fp32 and, behind them, lse.
template <int DP, int ROWS>
__device__ __forceinline__ void paged_store_part(float *slot, int r, int c, const float (&v)[8], float lse)
{
    float4 *dst = reinterpret_cast<float4 *>(slot + r * DP + c * 8);
    dst[0] = make_float4(v[0], v[1], v[2], v[3]);
    dst[1] = make_float4(v[4], v[5], v[6], v[7]);
    if (c == 0) slot[ROWS * DP + r] = lse;
}
// The segment of a CTA of a cluster: an equal share of the blocks of the cluster's item, key head and row tile.  false: there is
// nothing to do (for the whole cluster).
template <int ROWS, int BLOCK>
__device__ __forceinline__ bool paged_cluster_segment(const PagedParams &p, PagedSegments<ROWS, BLOCK> &seg, int rank)
{
    int x = blockIdx.x / p.cluster;
    seg.rt = x % p.row_tiles;
    x /= p.row_tiles;
    seg.kvh = x % p.kv_heads;
    seg.b = x / p.kv_heads;
    seg.it = paged_item(p, seg.b);
    seg.blocks = paged_blocks(p, seg.it, ROWS, seg.rt, BLOCK);
    seg.blk0 = (int)((long long)seg.blocks * rank / p.cluster);
    seg.blk1 = (int)((long long)seg.blocks * (rank + 1) / p.cluster);
    return seg.blocks > 0;
}
// The cluster's CTAs each write a share of the rows' pieces, from the parts that all of them hold at `at` in shared memory.
template <int DP, typename T, int ROWS, int BLOCK>
__device__ __forceinline__ void paged_join_cluster(const PagedParams &p, const PagedSegments<ROWS, BLOCK> &seg, uint32_t at, int rank)
{
    constexpr int kChunks = DP / 8;
    cluster_sync_all();
    const int rows = seg.rows();
    for (int i = rank * kPaThreads + threadIdx.x; i < rows * kChunks; i += p.cluster * kPaThreads) {
        const int r = i / kChunks, c = i % kChunks;
        float part[kPaCluster], mx = -INFINITY, sum = 0.f, acc[8] = {};
#pragma unroll
        for (int s = 0; s < kPaCluster; ++s) {
            part[s] = s < p.cluster ? cluster_ld(cluster_map(at + (ROWS * DP + r) * 4, s)) : -INFINITY;
            mx = fmaxf(mx, part[s]);
        }
#pragma unroll
        for (int s = 0; s < kPaCluster; ++s) {
            if (part[s] == -INFINITY) continue;                    // no keys there (a NaN goes on)
            const float w = expf(part[s] - mx);
            sum += w;
            const uint32_t src = cluster_map(at + (r * DP + c * 8) * 4, s);
            const float4 a = cluster_ld4(src), b4 = cluster_ld4(src + 16);
            acc[0] = fmaf(w, a.x, acc[0]); acc[1] = fmaf(w, a.y, acc[1]); acc[2] = fmaf(w, a.z, acc[2]); acc[3] = fmaf(w, a.w, acc[3]);
            acc[4] = fmaf(w, b4.x, acc[4]); acc[5] = fmaf(w, b4.y, acc[5]); acc[6] = fmaf(w, b4.z, acc[6]); acc[7] = fmaf(w, b4.w, acc[7]);
        }
        const PagedNorm norm = paged_joined(mx, sum);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= norm.inv;
        const int row = seg.rt * ROWS + r, t = paged_token(p, row), h = seg.kvh * p.group + row - t * p.group;
        paged_store<T>(p, seg.b, t, h, c, acc);
        if (c == 0) paged_store_lse(p, seg.b, t, h, norm.lse);
    }
    cluster_sync_all();                                            // nobody's shared memory goes while it is read
}

template <int DP, int MT, typename T>
__global__ void __launch_bounds__(kPaThreads, 2)
paged_wide_kernel(const PagedParams p)
{
    using L = PagedSmem<DP, MT>;
    constexpr int kChunks = DP / 8, kRows = L::kRows;
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x;
    grid_launch_dependents();
    grid_dependency_wait();

    PagedSegments<kRows, L::kBlock> seg(p);
    long long per = 1;
    const int cta = blockIdx.x, rank = p.cluster ? cta % p.cluster : 0;
    if (!(p.cluster ? paged_cluster_segment(p, seg, rank) : seg.locate(smem, per))) return;
    for (;;) {
        paged_walk_wide<DP, MT, T>(p, smem, seg.it, seg.b, seg.kvh, seg.rt, seg.blk0, seg.blk1);
        // whole results leave at once, parts go to the cluster's or the call's scratch
        const bool whole = seg.whole() && p.cluster <= 1;
        const int rows = seg.rows();
        const float *o = reinterpret_cast<const float *>(smem), *m = o + kRows * L::kPitch, *l = m + kRows;
        float *slot = p.cluster ? reinterpret_cast<float *>(smem + L::kShare) : p.part + (2LL * cta + (seg.blk0 == 0)) * kRows * (DP + 1);
        for (int i = tid; i < rows * kChunks; i += kPaThreads) {
            const int r = i / kChunks, c = i % kChunks;
            PagedNorm norm = paged_norm(m[r], l[r], p.scale);
            if (whole) norm = paged_whole(norm);
            float acc[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = o[r * L::kPitch + c * 8 + e] * norm.inv;
            if (whole) {
                const int row = seg.rt * kRows + r, t = paged_token(p, row), h = seg.kvh * p.group + row - t * p.group;
                paged_store<T>(p, seg.b, t, h, c, acc);
                if (c == 0) paged_store_lse(p, seg.b, t, h, norm.lse);
            } else {
                paged_store_part<DP, kRows>(slot, r, c, acc, norm.lse);
            }
        }
        if (p.cluster) break;
        if (tid == 0 && seg.blk0 == 0 && !whole) seg.describe(per);
        if (!seg.next()) return;
        __syncthreads();                                           // the result has been read
    }
    if (p.cluster > 1) paged_join_cluster<DP, T>(p, seg, smem_u32(smem) + L::kShare, rank);
}

// The parts of an item's key head and row tile that several CTAs worked on, added up in order: the first lies in slot 1 of
// the CTA that it began in, the others in slot 0 of the next CTAs of the key head.  blockIdx.x: that CTA.  Where an item may
// have many parts (few items over many CTAs), 2^group_shift threads share a row's eight columns, part by part in turn, and join at
// the end (16000 and 64000 states of one key head of 128, some 250 parts: 12.3 and 17.5 us the whole call, 23.1 and 39.7 with one).
constexpr int kPaJoinThreads = 128;
template <int DP, int ROWS, typename T>
__global__ void __launch_bounds__(kPaJoinThreads)
paged_join_kernel(const PagedParams p, const int group_shift)
{
    constexpr int kChunks = DP / 8, kSlot = ROWS * (DP + 1);
    __shared__ float shared[kPaJoinThreads][11];               // of each thread: the maximum, the sum, eight columns
    grid_launch_dependents();
    grid_dependency_wait();
    const int cta = blockIdx.x, groups = 1 << group_shift;
    const int4 d = *reinterpret_cast<const int4 *>(p.desc + cta * kPaDesc);
    if (d.x == 0) return;
    const int parts = d.x & 0xffff, rows = d.x >> 16;
    const int c = threadIdx.x % kChunks, g = threadIdx.x / kChunks & (groups - 1), each = kPaJoinThreads / kChunks >> group_shift;
    const float *first = p.part + (2LL * cta + 1) * kSlot, *next = p.part + 2LL * (cta + p.kv_heads) * kSlot;
    for (int r0 = blockIdx.y * each; r0 < rows; r0 += gridDim.y * each) {
        const int r = r0 + (threadIdx.x / kChunks >> group_shift);
        float mx = -INFINITY, sum = 0.f, acc[8] = {};
        for (int s0 = g; s0 < parts && r < rows; s0 += 8 * groups) {
            float lse[8], top = mx;
            float4 v[8][2];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int s = s0 + k * groups;
                const float *src = s == 0 ? first : next + 2LL * (s - 1) * p.kv_heads * kSlot;
                const bool live = s < parts;
                lse[k] = live ? src[ROWS * DP + r] : -INFINITY;
                if (live) {
                    v[k][0] = *reinterpret_cast<const float4 *>(src + r * DP + c * 8);
                    v[k][1] = *reinterpret_cast<const float4 *>(src + r * DP + c * 8 + 4);
                }
                top = fmaxf(top, lse[k]);
            }
            if (top > mx) {
                const float f = expf(mx - top);                    // (0 at the first; a NaN stays one)
                sum *= f;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] *= f;
                mx = top;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (lse[k] == -INFINITY) continue;                 // no states there (a NaN goes on)
                const float w = expf(lse[k] - mx);
                sum += w;
                acc[0] = fmaf(w, v[k][0].x, acc[0]); acc[1] = fmaf(w, v[k][0].y, acc[1]);
                acc[2] = fmaf(w, v[k][0].z, acc[2]); acc[3] = fmaf(w, v[k][0].w, acc[3]);
                acc[4] = fmaf(w, v[k][1].x, acc[4]); acc[5] = fmaf(w, v[k][1].y, acc[5]);
                acc[6] = fmaf(w, v[k][1].z, acc[6]); acc[7] = fmaf(w, v[k][1].w, acc[7]);
            }
        }
        if (groups > 1) {
            float *mine = shared[threadIdx.x];
            mine[0] = mx;
            mine[1] = sum;
#pragma unroll
            for (int e = 0; e < 8; ++e) mine[2 + e] = acc[e];
            __syncthreads();
            if (g == 0) {
                for (int k = 1; k < groups; ++k) mx = fmaxf(mx, shared[threadIdx.x + k * kChunks][0]);
                sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = 0.f;
                for (int k = 0; k < groups; ++k) {
                    const float *other = shared[threadIdx.x + k * kChunks];
                    if (other[1] == 0.f) continue;                 // (a NaN goes on)
                    const float w = expf(other[0] - mx);
                    sum = fmaf(w, other[1], sum);
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] = fmaf(w, other[2 + e], acc[e]);
                }
            }
            __syncthreads();
        }
        if (g != 0 || r >= rows) continue;
        const PagedNorm norm = paged_joined(mx, sum);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= norm.inv;
        const int row = d.w * ROWS + r, t = paged_token(p, row), h = d.z * p.group + row - t * p.group;
        paged_store<T>(p, d.y, t, h, c, acc);
        if (c == 0) paged_store_lse(p, d.y, t, h, norm.lse);
    }
}

// ------------------------------------------------------------------ append --
struct AppendParams {
    const uint4 *k_new, *v_new;                // in pieces of 16 bytes, as are the strides
    uint4 *k, *v;
    const int *table, *lens, *slot_of, *new_lens;
    XaStrides skn, svn;
    PagedStrides sk, sv;
    long long table_stride;
    FastDiv by_chunks, by_rows, by_page_rows;
    int tokens, pieces, chunks, q_rows, page_rows, pages, slots, cap;      // pieces: of a token's keys; chunks: of a head's
    int lanes;                                 // lanes of a token: a power of two
};
constexpr int kAppendThreads = 256, kAppendPieces = 4;

// `lanes` neighbouring lanes move a token's keys and values, four 16-byte pieces of each side by side.  First where they go:
// slot -> length -> page is what a token waits for, and one that is not there is not read.  Bound: HBM for prompts (8 x 2048 tokens,
// 8 key heads of 128: 134 MB moved in 25.7 us, 5.2 TB/s, the launch and the chain among them), that chain for
// single tokens (64 of them: 3.0 us).
__global__ void __launch_bounds__(kAppendThreads)
cache_append_kernel(const AppendParams p)
{
    grid_launch_dependents();
    grid_dependency_wait();
    const unsigned thread = blockIdx.x * kAppendThreads + threadIdx.x, token = thread / (unsigned)p.lanes;
    if (token >= (unsigned)p.tokens) return;
    const int b = (int)fast_div(token, p.by_rows), t = (int)token - b * p.q_rows;
    const PagedItem it = paged_item(p.table, p.table_stride, p.lens, p.slot_of, p.new_lens, b, p.slots, p.cap, p.q_rows);
    const int pos = it.len - it.news + t;
    if (t >= it.news || pos < 0) return;
    const int col = (int)fast_div((uint32_t)pos, p.by_page_rows), page = it.row[col], in_page = pos - col * p.page_rows;
    if ((unsigned)page >= (unsigned)p.pages) return;
    const uint4 *k_new = p.k_new + b * p.skn.b + t * p.skn.r, *v_new = p.v_new + b * p.svn.b + t * p.svn.r;
    uint4 *k = p.k + page * p.sk.page + in_page * p.sk.row, *v = p.v + page * p.sv.page + in_page * p.sv.row;
    for (int first = (int)(thread % (unsigned)p.lanes); first < p.pieces; first += kAppendPieces * p.lanes) {
        uint4 key[kAppendPieces], value[kAppendPieces];
        int h[kAppendPieces], c[kAppendPieces];
#pragma unroll
        for (int n = 0; n < kAppendPieces; ++n) {
            const int i = first + n * p.lanes;
            h[n] = (int)fast_div((uint32_t)i, p.by_chunks);
            c[n] = i - h[n] * p.chunks;
            if (i < p.pieces) {
                key[n] = k_new[h[n] * p.skn.h + c[n]];
                value[n] = v_new[h[n] * p.svn.h + c[n]];
            }
        }
#pragma unroll
        for (int n = 0; n < kAppendPieces; ++n)
            if (first + n * p.lanes < p.pieces) {
                k[h[n] * p.sk.head + c[n]] = key[n];
                v[h[n] * p.sv.head + c[n]] = value[n];
            }
    }
}

}  // namespace cudallm
