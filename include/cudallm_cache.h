/*
 * cudallm_cache.h -- C ABI of the operators that answer from a cache of keys and
 * values kept in pages:
 *
 *   cudallm_cache_append     keys and values of new tokens into the pages
 *   cudallm_paged_attn       attention of the newest tokens over their sequence's pages
 *   cudallm_pages_copy       whole pages, in every layer's pools
 *   cudallm_pages_fork       sequences that continue others, sharing their pages
 *   cudallm_pages_resize     sequences grow (pages are taken), shrink or end (given back)
 *   cudallm_pages_compact    the pages in use moved down to the lowest numbers
 *   cudallm_draft_verify     drafted tokens held against the target's probabilities
 *
 * A step of an answering program: resize (room for the new tokens), append and attend
 * in every layer, verify, resize (back to what was accepted).
 *
 * The conventions of cudallm_layers.h hold: device pointers unless "host" is said,
 * owned by the caller and on the current device, strides in ELEMENTS, calls enqueue on
 * `stream` and return without synchronising, argument errors are found before any CUDA
 * call, scratch comes from the caller (16-byte aligned, its contents before the call do
 * not matter), calls with different scratch, results and books may run at the same time
 * on several streams, all can be captured into CUDA graphs, and the same inputs give the
 * same bits.  Lengths, tables and lists are read on the device, so that a captured
 * step stays right while sequences grow.
 */
#ifndef CUDALLM_CACHE_H
#define CUDALLM_CACHE_H

#include <stddef.h>
#include <stdint.h>

#include "cudallm_layers.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * One layer's cache, and the new tokens of a batch.  A sequence lies in a slot: row s
 * of the table holds the numbers of its pages, state j being row j % page_rows of page
 * table[s][j / page_rows].  Filled in once for a layer.
 *   batch, q_rows : items of a call, and new tokens of an item at most
 *   q_heads, kv_heads, head_dim : kv_heads divides q_heads; head_dim a multiple of 8, at most 128
 *   pages, page_rows : of the pools; any page_rows >= 1
 *   slots, table_cols, table_stride : rows of the table (and of lens), page numbers in a row, pitch
 *   q_stride, o_stride, kn_stride, vn_stride : (item, token, head) of queries, results, new keys, new values
 *   k_stride, v_stride : (page, row, head) of the pools; rows x heads and heads x rows
 *              layouts, and keys and values side by side, are all taken as they lie
 *   strides  : multiples of 8 for dimensions larger than 1, no two elements in one place
 *              (kn_stride and vn_stride count for append only, q_stride and o_stride for attention only)
 *   dtype    : CUDALLM_BF16 or CUDALLM_F16, of everything but lse
 *   scale    : 0 to 2e38 (usually 1 / sqrt(head_dim))
 */
typedef struct cudallm_paged_shape {
    int64_t batch, q_rows, q_heads, kv_heads, head_dim;
    int64_t pages, page_rows;
    int64_t slots, table_cols, table_stride;
    int64_t q_stride[3], o_stride[3], kn_stride[3], vn_stride[3];
    int64_t k_stride[3], v_stride[3];
    int32_t dtype;
    float scale;
} cudallm_paged_shape;

/*
 * What both calls take:
 *   table    : int32, as above; a number outside 0..pages-1 is a page that is not there
 *   lens     : int32, `slots` elements: states of each sequence, the new tokens among
 *              them (values outside 0..table_cols * page_rows: the nearer end)
 *   slot_of  : int32, `batch` elements, the slot of each item, or NULL: item b lies in slot
 *              b.  An item whose slot is outside 0..slots-1 (padding of a batch) is not
 *              there: nothing is read or written for it.
 *   new_lens : int32, `batch` elements, new tokens n of each item (values outside
 *              0..q_rows: the nearer end), or NULL: q_rows.  Token t < n stands at position
 *              lens - n + t of its sequence.  Tokens from n on are not there.
 *
 * Append: row lens - n + t of the sequence becomes k_new[b][t], v_new[b][t].  Rows whose
 * page is not there, or whose position is negative, are not written.  Two items must
 * not write to the same row (of a page that two sequences share, see cudallm_pages_resize).
 * k_new, v_new, k, v: 16-byte aligned; the pools must not overlap the new tokens.
 * batch, q_rows, kv_heads, head_dim, slots, pages or table_cols == 0: success, nothing written.
 * Errors: INVALID_POINTER, INVALID_DTYPE, INVALID_DIM, INVALID_LD (strides),
 * UNSUPPORTED_SHAPE (head_dim; strides or pointers off 16 bytes), MISALIGNED,
 * UNSUPPORTED_DEVICE, CUDA.
 */
int cudallm_cache_append(const cudallm_paged_shape *shape, const void *k_new, const void *v_new, void *k, void *v,
                         const int32_t *table, const int32_t *lens, const int32_t *slot_of, const int32_t *new_lens,
                         void *stream);

/*
 * Attention of the new tokens (already appended) over their sequence, each seeing the states up
 * to its own position.  For query head h and key head g = h / (q_heads / kv_heads):
 *     S_tj = scale * Q[b, t, h] . K_j[g]  for j <= lens - n + t,   P = softmax(S)
 *     O[b, t, h] = sum_j P_tj V_j[g],   lse[b][h][t] = log(sum_j exp(S_tj))
 *   q, o     : 16-byte aligned; o must not overlap what is read
 *   lse      : fp32, contiguous [batch][q_heads][q_rows], or NULL
 * Rows of o and lse of tokens from n on, and of items that are not there, stay as they
 * are.  States on pages that are not there are left out, as if masked.  A token that sees no state
 * gives O = 0, lse = -inf.  What is not finite reaches the tokens that see it, as the formulas
 * say, and no others: a score of NaN or +inf makes its row (O and lse) NaN, one of -inf is a weight of zero unless the
 * row has no other (then NaN), a value that is not finite makes its column of O not finite.  What lies in
 * pages behind a sequence's end does not matter, whatever it is.
 * Products on the tensor cores with fp32 accumulation; maxima and sums in fp32; the
 * probabilities, relative to a maximum, are rounded to dtype for the second product
 * (2^-8 or 2^-11 of themselves; fp16 also 2^-25 of the maximum); O is rounded once.
 * K and V are read once for every 128 rows (query heads of a key head x tokens) where page_rows is 8,
 * 16, 32, 64 or a multiple of 128, else for every 64: single tokens, drafts and prompts (whole, or in pieces) alike.
 * The work is dealt out by the lengths on the device, so that unequal lengths cost no time (small shapes, in
 * which every SM has room for the longest sequence's share, are split by table_cols * page_rows).
 * Where K and V come in tiles of 128 rows the kernel's waits have a limit in time; if one runs out, it gives up
 * (o and lse are then not valid) and cudallm_device_status reports it, as for cudallm_xattn_fwd.
 * Empty sizes: as append (q_heads too); with no pages, slots or columns every token that is there has no
 * states, or its item is not there (slots == 0).
 * Errors: as append; WORKSPACE.
 */
int cudallm_paged_attn(const cudallm_paged_shape *shape, const void *q, const void *k, const void *v, const int32_t *table,
                       const int32_t *lens, const int32_t *slot_of, const int32_t *new_lens, void *o, float *lse,
                       void *scratch, size_t scratch_bytes, void *stream);
/* 0 where no scratch is needed (it may be NULL then), and for shapes that the call refuses */
size_t cudallm_paged_attn_scratch_bytes(const cudallm_paged_shape *shape);

/* Pages of one tensor: page i is `bytes` bytes at data + i * stride (bytes; multiples of
 * 16, stride >= bytes unless there is only one page, data 16-byte aligned).  A layer's keys, its values, or
 * both side by side. */
typedef struct cudallm_page_pool {
    void *data;
    int64_t stride, bytes;
} cudallm_page_pool;

/*
 * Copies page src[i] to page dst[i], i < n, in each of `count` pools (HOST array, read
 * during the call only) of `pages` pages.
 *   src, dst : int32, n elements on the device.  Pairs with a number outside 0..pages-1,
 *              and pairs of one page, are left out.  No page may be the dst of two pairs,
 *              nor the src of one and the dst of another.
 * n, count or pages == 0: success, nothing copied.
 * Errors: INVALID_POINTER, INVALID_DIM (negative; n > 2^31 - 1024, pages > 2^31 - 1024,
 * count > 65536, a page of more than 2^35 bytes, a pool of more than 2^46), INVALID_LD (stride < bytes), UNSUPPORTED_SHAPE (off 16 bytes),
 * MISALIGNED (src, dst), UNSUPPORTED_DEVICE, CUDA.
 */
int cudallm_pages_copy(const cudallm_page_pool *pools, int64_t count, int64_t pages, const int32_t *src, const int32_t *dst,
                       int64_t n, void *stream);

/*
 * Whose pages are whose.  A page is free if refs[page] == 0, else as many sequences hold it.
 *   refs  : int32, `pages` elements, 16-byte aligned
 *   lens  : int32, `slots` elements: states of the sequence in each slot, 0 for none
 *   table : int32, slots rows of table_cols page numbers, pitch table_stride; a sequence
 *           holds the first ceil(lens / page_rows) entries of its row, the others mean nothing
 * A new book is all zeros.  The book is the caller's: it can be copied and put back as a whole (all three
 * arrays), and lens and table go into the calls above as they are.  Calls that change
 * one book must not overlap.  A book that contradicts itself gives wrong page
 * numbers, never an access outside the arrays; page numbers outside 0..pages-1 are passed over,
 * lengths outside 0..table_cols * page_rows taken as the nearer end.
 */
typedef struct cudallm_page_book {
    int32_t *refs, *lens, *table;
    int64_t pages, page_rows, slots, table_cols, table_stride;
} cudallm_page_book;

/*
 * Sequence dst[i] becomes what sequence src[i] was before the call, i < n, all at once (src
 * may hold slots that are overwritten: a reordering, or several continuations of one).  Its
 * length and page numbers are copied, no data is: the pages are shared, and what dst held is
 * given back.  Entries with a slot outside 0..slots-1 are passed over; of several with the same
 * dst the first counts; dst == src changes nothing.
 *   src, dst : int32, n elements on the device
 * Errors: INVALID_POINTER, INVALID_DIM (also pages > 2^20, n > 16384, table_cols * page_rows > 2^31 - 1024),
 * INVALID_LD (table_stride < table_cols), MISALIGNED, WORKSPACE, UNSUPPORTED_DEVICE, CUDA.
 */
int cudallm_pages_fork(const cudallm_page_book *book, const int32_t *src, const int32_t *dst, int64_t n,
                       void *scratch, size_t scratch_bytes, void *stream);
size_t cudallm_pages_fork_scratch_bytes(const cudallm_page_book *book, int64_t n);

/*
 * The sequence in slot_of[i] gets the length new_lens[i], i < n.
 *  - A shorter one gives back the pages behind its new end (length 0: it ends); a page
 *    that nobody holds any more is free.
 *  - A longer one takes the pages it lacks.  If its last page so far is not full and
 *    shared, the new tokens would be written into another sequence's page: it gets a copy
 *    of its own instead, in all pools, unless all that share it grow in this call, in which case the first
 *    of them keeps it.
 * With pools the copies are a launch of their own behind the book's, also where none turn out to be needed (only the
 * device knows).  A step in which no sequence that grows shares its last page may pass count == 0 and save it.
 * New pages are the lowest free ones (those given back in this call among them), dealt out in the order
 * of the list, a sequence's copy first.
 * All or nothing: where there are not enough pages, or a length exceeds table_cols *
 * page_rows, nothing changes at all.
 *   slot_of  : int32, n elements, or NULL: slots 0..n-1.  Slots outside 0..slots-1 and
 *              negative lengths are passed over; of several entries with the same slot the first of the others counts.
 *   new_lens : int32, n elements
 *   pools    : HOST array of `count` pools that the copies are made in (0: a book without data)
 *   result   : int32, one word, or NULL: 0 done; > 0: so many pages are missing (at most 2^31 - 1 is said);
 *              -1: a length beyond the table
 * Errors: as cudallm_pages_fork and cudallm_pages_copy.
 */
int cudallm_pages_resize(const cudallm_page_book *book, const cudallm_page_pool *pools, int64_t count, const int32_t *slot_of,
                         const int32_t *new_lens, int64_t n, int32_t *result, void *scratch, size_t scratch_bytes,
                         void *stream);
size_t cudallm_pages_resize_scratch_bytes(const cudallm_page_book *book, int64_t n);

/*
 * Moves the pages in use into the lowest numbers: with m of them, the k-th page in use
 * from m on moves to the k-th free page below m, in all pools; refs and table follow.  Afterwards pages
 * m.. are free.
 *   used : int32, one word, or NULL: m
 * Errors: as cudallm_pages_resize.
 */
int cudallm_pages_compact(const cudallm_page_book *book, const cudallm_page_pool *pools, int64_t count, int32_t *used,
                          void *scratch, size_t scratch_bytes, void *stream);
size_t cudallm_pages_compact_scratch_bytes(const cudallm_page_book *book);

/*
 * Drafted tokens of `batch` sequences against the target's probabilities, so that what is
 * kept is distributed as the target's own tokens.  For sequence b with drafts x_0 .. x_{m-1}:
 *     x_t is accepted if all before it are and u_t * q_t(x_t) < p_t(x_t);
 *     with a = the number accepted, one more token is drawn: the first v with
 *     sum_{w <= v} r(w) > u_n * sum_w r(w), where r = max(p_a - q_a, 0) if a < m, and r = p_a if
 *     a = m or where the former is zero everywhere.
 *   p          : dtype, batch * (n + 1) rows of `vocab` probabilities, pitch ldp: row b (n + 1) + t is p_t
 *   q          : dtype, batch * n rows, pitch ldq; or NULL: the drafts were certain, q_t(x_t) = 1
 *                and 0 elsewhere
 *   drafts     : int32, batch x n;  a token outside 0..vocab-1 is never accepted (its q is taken as zero)
 *   draft_lens : int32, `batch` elements, m of each (values outside 0..n: the nearer end), or NULL: n
 *   u          : fp32, batch x (n + 1) random numbers in [0, 1)
 *   tokens     : int32, batch x (n + 1): the accepted drafts, the token drawn, then -1
 *   accepted   : int32, `batch` elements: a
 *   dtype      : CUDALLM_F32, _BF16 or _F16
 * Comparisons and sums are in 64 bits (the product and the difference are exact).  Probabilities need not add up
 * to one; values of r that are not positive and finite, as fp32 has them, count as zero.  Where p_a has no mass
 * either, the token drawn is -1.  n may be 0 (a token is drawn from p_0).  Drafts behind m, and their
 * probabilities, are read but change nothing.  tokens and accepted must not overlap what is read.
 * Errors: INVALID_DTYPE, INVALID_DIM (negative; vocab 0; batch * (n + 1) or vocab > 2^31 - 1024), INVALID_LD,
 * INVALID_POINTER, MISALIGNED, UNSUPPORTED_DEVICE, CUDA.
 */
int cudallm_draft_verify(const void *p, const void *q, const int32_t *drafts, const int32_t *draft_lens, const float *u,
                         int32_t *tokens, int32_t *accepted, int64_t batch, int64_t n, int64_t vocab, int64_t ldp, int64_t ldq,
                         int dtype, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* CUDALLM_CACHE_H */
