/*
 * cudallm_layers.h -- C ABI of the operators around the matrix products of a
 * transformer block, for its training step and for single tokens:
 *
 *   cudallm_layernorm_rows       LayerNorm over the rows of a matrix, with the rows'
 *   cudallm_layernorm_rows_bwd   statistics, and its gradient
 *   cudallm_grad_norm            the norm of all gradients of a model together,
 *   cudallm_grad_clip            and scaling them down to a limit
 *   cudallm_grad_clip_norm
 *   cudallm_xattn_fwd            attention of one sequence's queries to the states of
 *   cudallm_xattn_bwd            another, of another length, and its gradient
 *
 * The general conventions of cudallm_gemm.h hold (device pointers owned by the
 * caller, pitches in elements, calls enqueue on `stream` and return without
 * synchronising, negative CUDALLM_ERR_* status codes, argument errors found
 * before any CUDA call, compute capability 10.0 only, no CPU fallback).  All
 * pointers must belong to the device that is current at the call, and `stream`
 * to that device.
 *
 * What a call needs beside its operands it takes as `scratch` from the caller
 * (16-byte aligned, at least what the matching _scratch_bytes function says; its
 * contents before the call do not matter and are not kept).  Nothing else is
 * shared between calls: calls with different scratch and outputs may run at the
 * same time on several streams, and every call can be captured into a CUDA graph
 * (a graph keeps using the scratch of the captured call).  Given the same inputs
 * on the same kind of device, a call returns the same bits each time.
 */
#ifndef CUDALLM_LAYERS_H
#define CUDALLM_LAYERS_H

#include <stddef.h>
#include <stdint.h>

#include "cudallm_gemm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of these operators: CUDALLM_F32, CUDALLM_BF16 and */
#define CUDALLM_F16 2

/*
 * LayerNorm of every row of a matrix.
 *     mean_r = (1/n) sum_i x[r][i]
 *     var_r  = (1/n) sum_i (x[r][i] - mean_r)^2              (biased estimate)
 *     rstd_r = 1 / sqrt(var_r + eps)
 *     y[r][i] = (x[r][i] - mean_r) * rstd_r * gamma[i] + beta[i]
 *   x, y        : dtype, rows x n, row pitches ldx, ldy >= n; padding columns of y
 *                 are left untouched; y may be x itself (with ldy == ldx), else the
 *                 two must not overlap
 *   gamma, beta : param_dtype, n elements each, or NULL for all ones / all zeros
 *   mean, rstd  : fp32, rows elements each, written; either may be NULL
 *   dtype       : CUDALLM_F32, _BF16 or _F16; param_dtype: dtype or CUDALLM_F32
 * Statistics and arithmetic are in fp32 (mean and variance from differences to a
 * first mean, so a mean far above the spread costs no accuracy of y); y is
 * rounded once.  A row that holds an infinity or a NaN gives NaN in that row only; so
 * does a finite row whose sum leaves fp32's range, and one whose squared differences
 * do (differences of 1e19 and more) has rstd = 0 and y = beta.
 * rows == 0 or n == 0: success, nothing written.
 * Errors: INVALID_DIM (negative, rows or n > 2^31 - 1024, eps negative or not
 * finite), INVALID_LD (also for y == x with another pitch), INVALID_DTYPE, INVALID_POINTER (x or y NULL), MISALIGNED
 * (a pointer off its element size), UNSUPPORTED_DEVICE, CUDA.
 */
int cudallm_layernorm_rows(const void *x, const void *gamma, const void *beta, void *y, float *mean, float *rstd,
                           int64_t rows, int64_t n, int64_t ldx, int64_t ldy, int dtype, int param_dtype,
                           float eps, void *stream);

/*
 * Gradient of cudallm_layernorm_rows.  With xhat = (x - mean) * rstd, g = dy * gamma:
 *     dx     = rstd * (g - (1/n) sum_i g_i - xhat * (1/n) sum_i g_i xhat_i)
 *     dgamma = sum_rows dy * xhat,   dbeta = sum_rows dy
 *   dy, x, dx     : dtype, rows x n, pitches lddy, ldx, lddx >= n; dx may be dy or x
 *                   itself (with the same pitch), else must not overlap them
 *   gamma         : param_dtype, or NULL for all ones
 *   mean, rstd    : fp32, rows elements, as the forward call wrote them
 *   dgamma, dbeta : param_dtype, n elements each, overwritten (no accumulation)
 * Any of dx, dgamma and dbeta may be NULL: that gradient is not computed.
 * Sums are in fp32 in a fixed order; every result is rounded once.  rows == 0
 * gives dgamma = dbeta = 0; n == 0 is a no-op.
 * Errors: as the forward call; WORKSPACE (scratch NULL, misaligned or smaller than
 * cudallm_layernorm_rows_bwd_scratch_bytes; not needed when dgamma and dbeta are NULL).
 */
int cudallm_layernorm_rows_bwd(const void *dy, const void *x, const void *gamma, const float *mean, const float *rstd,
                               void *dx, void *dgamma, void *dbeta, int64_t rows, int64_t n,
                               int64_t lddy, int64_t ldx, int64_t lddx, int dtype, int param_dtype,
                               void *scratch, size_t scratch_bytes, void *stream);
/* 0 for sizes that the call refuses */
size_t cudallm_layernorm_rows_bwd_scratch_bytes(int64_t rows, int64_t n);

/* One gradient of a model: n contiguous elements of `dtype` at `data` (device).
 * `out` is where the scaled gradient goes: `data` itself (in place) or a buffer of
 * the same size and type that overlaps no `data` of the list.  No two `out` overlap,
 * and one in place overlaps no other entry's `data` (one call would read it while
 * it is scaled). */
typedef struct cudallm_tensor {
    void *data;
    void *out;
    int64_t n;
    int32_t dtype;
    int32_t reserved;     /* 0 */
} cudallm_tensor;

/*
 * norm[0] = sqrt(sum over all tensors and elements of g^2), fp32 on the DEVICE.
 *   tensors : HOST array of `count` entries, read during the call only (the
 *             entries travel in the kernels' parameters); `out` is not used
 * Squares are summed in fp32 in groups of eight and from there in double; a group
 * whose sum leaves the middle of the fp32 range is summed in double, so the norm is
 * right for gradients of any size as long as it fits into fp32 itself.  An infinity
 * gives inf, a NaN gives NaN.  No tensors, or only empty ones, give 0.  Entries with
 * n == 0 are skipped (their pointers may be NULL).
 * Errors: INVALID_DIM (count or an n negative, count > 2^24, n > 2^40, more than 2^44
 * elements), INVALID_POINTER, INVALID_DTYPE, MISALIGNED, WORKSPACE,
 * UNSUPPORTED_DEVICE, CUDA.
 */
int cudallm_grad_norm(const cudallm_tensor *tensors, int64_t count, float *norm, void *scratch, size_t scratch_bytes,
                      void *stream);
/*
 * out = g * c for every tensor, with c = min(1, max_norm / (norm[0] + eps)) (1 where
 * max_norm >= norm[0] + eps, both zero or both infinite too), the product rounded once.  `norm` is on the device, from cudallm_grad_norm or, for
 * gradients spread over several devices, combined by the caller.  A NaN norm makes
 * all gradients NaN, an infinite one makes the finite ones zero.  Tensors that are
 * scaled in place stay untouched (no bit changes) where c is 1.
 * Errors: as cudallm_grad_norm; INVALID_DIM also for max_norm or eps negative or NaN.
 */
int cudallm_grad_clip(const cudallm_tensor *tensors, int64_t count, const float *norm, float max_norm, float eps,
                      void *stream);
/* Both, in fewer launches: norm[0] is written, then the gradients are scaled. */
int cudallm_grad_clip_norm(const cudallm_tensor *tensors, int64_t count, float max_norm, float eps, float *norm,
                           void *scratch, size_t scratch_bytes, void *stream);
/* Scratch of cudallm_grad_norm and cudallm_grad_clip_norm for lists of up to `count` tensors. */
size_t cudallm_grad_norm_scratch_bytes(int64_t count);

/*
 * Cross attention: batch items of q_rows queries attend to kv_rows states of their
 * own.  For batch item b, query head h and key head g = h / (q_heads / kv_heads):
 *     S = scale * Q[b, :, h] K[b, :, g]^T,  P = softmax(S) over the keys < kv_lens[b]
 *     O[b, :, h] = P V[b, :, g],   lse[b][h][i] = log(sum_j exp(S_ij))
 * Sizes, strides (ELEMENTS; order: batch item, row, head; the head_dim values of a
 * row and head are contiguous) and scale come in a struct, which a program fills in
 * once for a layer.  Q and O (and their gradients) use q_stride and o_stride; K, V
 * and their gradients k_stride and v_stride, so rows x heads and heads x rows
 * layouts, and keys and values side by side in one tensor, are all taken as they lie.
 *   dtype    : CUDALLM_BF16 or CUDALLM_F16, of all operands and results but lse (fp32,
 *              contiguous [batch][q_heads][q_rows])
 *   head_dim : a multiple of 8, at most 128; kv_heads divides q_heads
 *   strides  : multiples of 8 for dimensions larger than 1, and such that no two
 *              elements share a place (the stride of a dimension of size 1 is not used)
 *   scale    : finite, >= 0 (usually 1 / sqrt(head_dim))
 */
typedef struct cudallm_xattn_shape {
    int64_t batch, q_rows, kv_rows, q_heads, kv_heads, head_dim;
    int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];
    int32_t dtype;
    float scale;
} cudallm_xattn_shape;

/*
 * Forward.
 *   q, k, v : read only, 16-byte aligned;  o : written, must not overlap them
 *   kv_lens : int32, `batch` elements on the device, the states of each item that
 *             exist (values outside 0..kv_rows are taken as the nearer end), or NULL:
 *             all.  States from kv_lens[b] on are never used, whatever they hold
 *             (NaN and infinities too).
 *   lse     : written unless NULL (the backward call needs it)
 * An item without states (kv_lens[b] == 0, or kv_rows == 0) gives O = 0 and
 * lse = -inf.  A query, key or value that is not finite makes the rows that see it
 * not finite, and no others.
 * Products are taken on the tensor cores with fp32 accumulation; maxima and sums in
 * fp32; the probabilities, relative to a maximum, are rounded to dtype for the second
 * product: by at most 2^-8 (bf16) or 2^-11 (fp16) of themselves each, and in fp16 by
 * up to 2^-25 (of the maximum) where they are below 2^-14.  O is rounded once.
 * Kernels: (q_heads / kv_heads) * q_rows <= 16 rows per key head (single tokens) take
 * a kernel that reads every K and V once and splits the keys over the GPU; longer
 * queries one that owns 256 query rows of a head per CTA, split over the keys where
 * there are too few of those.  Up to eight splits of single tokens join inside the
 * launch (a cluster of CTAs, no scratch); all other split calls in a second one.
 * batch, q_rows or q_heads == 0 or head_dim == 0: success, nothing written.
 * Errors: INVALID_POINTER (shape, q or o NULL; k or v NULL with kv_rows > 0),
 * INVALID_DTYPE, INVALID_DIM (negative or too large sizes, kv_heads not a divisor of
 * q_heads, scale), INVALID_LD (strides), UNSUPPORTED_SHAPE (head_dim, strides or
 * pointers off 16 bytes), MISALIGNED (kv_lens, lse), WORKSPACE, UNSUPPORTED_DEVICE,
 * CUDA.
 */
int cudallm_xattn_fwd(const cudallm_xattn_shape *shape, const void *q, const void *k, const void *v,
                      const int32_t *kv_lens, void *o, float *lse, void *scratch, size_t scratch_bytes, void *stream);
/* 0 where no scratch is needed (it may be NULL then), and for shapes that the call refuses */
size_t cudallm_xattn_fwd_scratch_bytes(const cudallm_xattn_shape *shape);

/*
 * Gradient of cudallm_xattn_fwd.  With P = exp(S - lse), delta_i = sum_c dO_ic O_ic:
 *     dV = P^T dO,  dS = P * (dO V^T - delta),  dQ = scale * dS K,  dK = scale * dS^T Q
 * with dK and dV summed over the query heads that share a key head.
 *   o, lse      : as the forward call wrote them;  d_o : laid out like o (o_stride)
 *   dq          : written, q_stride;  dk, dv : written, k_stride and v_stride; both or
 *                 neither may be NULL (the states' gradients are not computed then)
 * Results must not overlap any operand.  States from kv_lens[b] on get zero
 * gradients; an item without states gives dQ = 0; q_rows == 0 gives dK = dV = 0.
 * P and dS are rounded to dtype for the tensor cores (as P is in the forward call);
 * sums are in fp32, without atomics.  For fp16 that means that a dS below 2^-14 loses
 * relative precision and one beyond 65504 overflows: scale the loss accordingly.
 * Errors: as the forward call.
 */
int cudallm_xattn_bwd(const cudallm_xattn_shape *shape, const void *q, const void *k, const void *v,
                      const int32_t *kv_lens, const void *o, const float *lse, const void *d_o,
                      void *dq, void *dk, void *dv, void *scratch, size_t scratch_bytes, void *stream);
size_t cudallm_xattn_bwd_scratch_bytes(const cudallm_xattn_shape *shape);

#ifdef __cplusplus
}
#endif

#endif /* CUDALLM_LAYERS_H */
