/*
 * C ABI of linear layers in 8-bit integers: the layers of a network that are not kept in ternary-SVD form, with the
 * activations, layouts, bias and output types of tsvd_forward_io.
 *
 * Weights: codes w [M][N] in int8 and one fp32 scale t [M] for each row (output channel).  Activations: codes q [B][N] and one
 * fp32 scale s [B] for each token, made from x when the layer is called (or by the norm before it, tsvd_norm.h):
 *   a_b = max(max_n |x_bn|, 2^-100),  s_b = fl(a_b / 127),  r_b = fl(127 / a_b),  q_bn = the whole number nearest to x_bn r_b
 *   y_bm = (sum_n q_bn w_mn) s_b t_m + bias_m
 * fl rounds to fp32; the product x r is not rounded before the whole number is taken, ties go to the even one, and |q| <= 127.
 * The sum is an exact whole number (N below 2^17); the rest is fp32 arithmetic, ((sum) t) s + bias in this order: where (sum) t is zero
 * or a normal number, y is within 2^-22 of |(sum) s t| + |bias| of what the formula gives, then rounded to nearest even where y is bf16.  A token's result does not depend on the tokens beside it.
 * A token that holds an infinity or NaN gets the scale NaN: its outputs are NaN, those of other tokens are as ever.  (All of the
 * 2^-100 floor: smaller tokens keep fewer bits, and a token of zeros has codes 0.)
 *
 * Status codes, streams and ownership are those of tsvd.h: calls enqueue on `stream` (hipStream_t as void*, NULL = default
 * stream) and return without synchronising unless stated otherwise; on failure outputs are left untouched.  The current HIP
 * device has to be the one that the pointers and the stream belong to.  Nothing is kept between calls but the handle, which is
 * only read: calls on one handle may overlap in time if their workspaces and outputs differ.
 */
#ifndef TSVD_INT8_H
#define TSVD_INT8_H

#include <stddef.h>
#include <stdint.h>

#include "tsvd.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tsvd_int8_handle tsvd_int8_handle; /* opaque; owns or borrows the packed device blob */

/* ---- codes of activations -------------------------------------------------------------------
 *
 * Codes are token-major, [B][ldq] bytes, codes_dev 16-byte aligned and ldq >= N a multiple of 16.  What stands between N and ldq
 * is not used, and calls that write codes may write there up to the next multiple of 16.
 * tsvd_int8_row_bytes(N) is the pitch that suits the products (N rounded up to 128; 0 if N <= 0). */
size_t tsvd_int8_row_bytes(int64_t N);

/* q and s of x, as above.
 *   x_dev : device, [B][N] with row stride ldx >= N (TSVD_TOKEN_MAJOR) or [N][B] with ldx >= B (TSVD_FEATURE_MAJOR) elements of
 *           x_dtype, at any stride and element alignment.
 *   scales_dev : device fp32 [B].
 *   workspace : device, at least tsvd_int8_quantize_workspace_bytes(B, N, x_layout) bytes, 256-byte aligned (NULL with workspace_bytes 0 where that is 0, as it is for
 *               TSVD_TOKEN_MAJOR); its contents are undefined afterwards.
 * Also what makes the codes and scales of weights from W [M][N] (a row is a token then).
 * TSVD_EINVAL: null pointers, sizes below 1, strides that are too small, codes that are not aligned, a workspace that is too small.  TSVD_EUNSUPPORTED: N >= 2^17, B > 2^24. */
size_t tsvd_int8_quantize_workspace_bytes(int64_t B, int64_t N, tsvd_layout x_layout);
tsvd_status tsvd_int8_quantize(const void* x_dev, tsvd_dtype x_dtype, tsvd_layout x_layout, int64_t B, int64_t N, int64_t ldx,
                               int8_t* codes_dev, int64_t ldq, float* scales_dev, void* workspace, size_t workspace_bytes, void* stream);

/* ---- weights --------------------------------------------------------------------------------
 *
 * tsvd_int8_packed_bytes(M, N): size of the packed weights (0 if a dimension is <= 0 or N >= 2^17).
 * tsvd_int8_pack: reorders codes w_dev [M][ldw] (ldw >= N, any alignment, all 256 values allowed) and scales t_dev [M], both device memory,
 * into the layout of the matrix instruction.
 *   dev_buf == NULL : the library allocates it and tsvd_int8_free releases it.
 *   dev_buf != NULL : caller-owned device memory of dev_buf_bytes >= tsvd_int8_packed_bytes(M, N), 256-byte aligned; it must outlive
 *                     the handle and is not freed.
 * Enqueues on `stream` and WAITS for it: the handle is ready for any stream.  A stream that is being captured is refused
 * (TSVD_EDEVICE) with nothing enqueued.  *out is written only on success.  TSVD_EUNSUPPORTED: N >= 2^17 or M > 2^24. */
size_t tsvd_int8_packed_bytes(int64_t M, int64_t N);
tsvd_status tsvd_int8_pack(const int8_t* w_dev, int64_t ldw, const float* t_dev, int64_t M, int64_t N, void* dev_buf, size_t dev_buf_bytes,
                           void* stream, tsvd_int8_handle** out);
/* Dimensions; any output may be NULL. */
tsvd_status tsvd_int8_info(const tsvd_int8_handle* h, int64_t* M, int64_t* N);
/* Releases the handle and whatever device memory it owns.  NULL is allowed. */
void tsvd_int8_free(tsvd_int8_handle* h);

/* ---- the layer ------------------------------------------------------------------------------
 *
 * y from codes that are there (several layers that read the same activations share them):
 *   y_dev : [M][B] with ldy >= B (TSVD_FEATURE_MAJOR) or [B][M] with ldy >= M (TSVD_TOKEN_MAJOR), of y_dtype, at any stride and element
 *           alignment.   bias_dev : device fp32 [M] or NULL.
 * TSVD_EINVAL as above, and where the current device is not the one of the handle; TSVD_EUNSUPPORTED: B > 2^24, ldq > 2^22, or
 * more than 2^23 tiles of 64 x 64 results or larger ones (M B above 2^35). */
tsvd_status tsvd_int8_product(const tsvd_int8_handle* h, const int8_t* codes_dev, int64_t ldq, const float* scales_dev, int64_t B,
                              const float* bias_dev, void* y_dev, tsvd_dtype y_dtype, tsvd_layout y_layout, int64_t ldy, void* stream);

/* y from x: tsvd_int8_quantize and tsvd_int8_product, the same bits, in one launch where tokens are few.
 *   workspace : device, at least tsvd_int8_workspace_bytes(h, B, x_dtype, x_layout) bytes, 256-byte aligned (NULL with
 *               workspace_bytes 0 where that is 0); its contents are undefined afterwards.  x, y and workspace must not alias. */
size_t tsvd_int8_workspace_bytes(const tsvd_int8_handle* h, int64_t B, tsvd_dtype x_dtype, tsvd_layout x_layout);
tsvd_status tsvd_int8_forward(const tsvd_int8_handle* h, const void* x_dev, tsvd_dtype x_dtype, tsvd_layout x_layout, int64_t B, int64_t ldx,
                              const float* bias_dev, void* y_dev, tsvd_dtype y_dtype, tsvd_layout y_layout, int64_t ldy, void* workspace,
                              size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
