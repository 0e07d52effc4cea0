/*
 * C ABI of the group norm with an activation, channels last: what stands between the layers of tsvd.h, tsvd_int8.h and
 * tsvd_conv.h.
 *
 * x is [images][positions][C], a row of C channels for each position (the token-major activations of those headers), C / groups
 * channels in each group.  For every image and group, over its positions and channels:
 *   mu = mean of x,  v = mean of (x - mu)^2,  h = (x - mu) / sqrt(v + eps) gamma_c + beta_c,  y = act(h)
 * groups = 1 and positions = 1 is the layer norm of `images` tokens.
 * Mean and variance are taken in fp32, from deviations: of values from one of the values themselves, of pieces of a group (joined in
 * fp64) from the mean of one of them, so that no square of a mean enters; everything up to act(h) is fp32.  A group that holds an
 * infinity or NaN gives NaN in its own outputs and no others.
 * Deviations have to stay below 2^60, whose squares fp32 still sums.  Results do not depend on what runs beside the call: the sums have
 * a fixed order.
 *
 * Status codes, streams and ownership are those of tsvd.h: calls enqueue on `stream` and return without synchronising; on failure
 * outputs are left untouched.  The current HIP device has to be the one that the pointers and the stream belong to.
 */
#ifndef TSVD_NORM_H
#define TSVD_NORM_H

#include <stddef.h>
#include <stdint.h>

#include "tsvd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* none, max(h, 0), h / (1 + e^-h), h (1 + erf(h / sqrt 2)) / 2
 * in fp32: against the formula at h, SiLU is within (2 |h| + 4) 2^-24 |y| + 2^-116 and GELU within 2^-22 |h|, for negative h also within
 * 2.2 10^-7 (far out, where y is smaller still, that is less than fp32 holds: 2 10^-4 of y at h = -3.5, 2 10^-3 at -5). */
typedef enum { TSVD_ACT_NONE = 0, TSVD_ACT_RELU = 1, TSVD_ACT_SILU = 2, TSVD_ACT_GELU = 3 } tsvd_activation;

/* Scratch that the calls below need (0 on invalid arguments; 256 at least otherwise). */
size_t tsvd_group_norm_workspace_bytes(int64_t images, int64_t positions, int64_t C, int64_t groups);

/* y of x.
 *   x_dev : device, rows of C elements of x_dtype, ldx >= C elements from one position to the next (of the same image or of the next one),
 *           at any stride and element alignment.
 *   gamma_dev, beta_dev : device fp32 [C], or NULL for ones and zeros.   eps : positive and finite.
 *   y_dev : of y_dtype, TSVD_TOKEN_MAJOR: like x with ldy >= C;  TSVD_FEATURE_MAJOR: [C][images * positions] with
 *           ldy >= images * positions (what tsvd_conv2d_forward reads: [C][images][H][W]).
 *   workspace : device, at least tsvd_group_norm_workspace_bytes(...) bytes, 256-byte aligned; contents undefined afterwards.
 * x, y and workspace must not alias.
 * TSVD_EINVAL: null pointers, sizes below 1, groups that do not divide C, strides that are too small, an unknown type, layout or activation.
 * TSVD_EUNSUPPORTED: C > 2^20, groups > 4096, images * positions > 2^31 - 1, work for more than 2^31 - 1 workgroups. */
tsvd_status tsvd_group_norm(const void* x_dev, tsvd_dtype x_dtype, int64_t images, int64_t positions, int64_t C, int64_t ldx, int64_t groups,
                            const float* gamma_dev, const float* beta_dev, float eps, tsvd_activation act, void* y_dev, tsvd_dtype y_dtype,
                            tsvd_layout y_layout, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream);

/* The same with y as the 8-bit codes of tsvd_int8.h, a scale for each position: what tsvd_int8_quantize would make of y in fp32, without y in memory.  (The statistics may be joined in
 * another order than tsvd_group_norm joins them, so that the last bits of y differ: a scale's too then, and of codes those whose value is that near to the border between two.)
 * One scale holds all groups of a position: an infinity or NaN in any of them makes it NaN.
 *   codes_dev : [images * positions][ldq] bytes, 16-byte aligned, ldq >= C a multiple of 16; up to the next multiple of 16 behind C may be written.   scales_dev : fp32 [images * positions].
 * TSVD_EUNSUPPORTED also: C >= 2^17. */
tsvd_status tsvd_group_norm_int8(const void* x_dev, tsvd_dtype x_dtype, int64_t images, int64_t positions, int64_t C, int64_t ldx, int64_t groups,
                                 const float* gamma_dev, const float* beta_dev, float eps, tsvd_activation act, int8_t* codes_dev, int64_t ldq,
                                 float* scales_dev, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
