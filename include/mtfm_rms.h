/*
 * mtfm_rms.h -- C ABI of the root-mean-square normalization with the residual's addition of libmtfm_hta.so,
 * hand-written for AMD gfx950 (MI355X).
 *
 * The operation, per row of `width` features:
 *   h_i    = x_i + residual_i   (rounded to the element type it is stored in; h = x without a residual)
 *   rstd_i = 1 / sqrt(mean_c(h_ic^2) + eps)
 *   y_i    = h_i rstd_i (.) weight
 * or, for products in 8 bits, q_i with y_i = q_i scale_i: scale_i = max_c |y_ic| / top, top = 127 (int8) or 448 (e4m3,
 * the OCP format), q_i = y_i / scale_i rounded to nearest even.  A row of zeros has scale 0 and q = 0 (so has a row whose
 * scale is too small for a float32).  A row whose largest magnitude is infinite or that holds a NaN has that as its scale.
 * Backward, for the gradients dy of y and dh of h (what arrives through the residual stream; optional):
 *   xhat_i = h_i rstd_i     w_i = dy_i (.) weight
 *   dx_i = dh_i + rstd_i (w_i - xhat_i mean_c(w_i (.) xhat_i))     dweight = sum_i dy_i (.) xhat_i
 * dx is the gradient of x and of residual alike.
 *
 * Layout.  Rows of `dtype` (MTFM_HTA_BF16 or MTFM_HTA_FP32).  x, residual, dy, dh and the backward pass's h may have a row
 * stride (in elements, >= width); outputs are contiguous, [n_rows][width].  weight, dweight: [width] float32.  rstd, scale:
 * [n_rows] float32.  width 1 to 8192.  Pointers are aligned to their element; where all of a call's are to 16 bytes and width
 * and strides are multiples of 8 (bf16) or 4 (float32), rows move in 16-byte words, and by single elements otherwise.  An output
 * may be the very memory of an input of the same element type and of stride `width`; otherwise outputs overlap nothing.
 * All arithmetic is float32.
 *
 * Pointers are DEVICE pointers owned by the caller; `stream` is a hipStream_t passed as void* (NULL = the default stream).  The
 * calls validate their scalar arguments on the host, enqueue kernels and return; they never allocate, copy to the host or
 * synchronise, and may be captured.  Status codes and mtfm_hta_last_error() are those of mtfm_hta.h; on a non-zero status
 * other than MTFM_HTA_ERR_LAUNCH nothing has been enqueued.  n_rows = 0 is valid; per-row arrays may be NULL then.
 */
#ifndef MTFM_RMS_H
#define MTFM_RMS_H

#include "mtfm_hta.h"

#ifdef __cplusplus
extern "C" {
#endif

/* 8-bit types of mtfm_rms_fwd_q8() */
enum { MTFM_RMS_INT8 = 0, MTFM_RMS_E4M3 = 1 };

/* kernel kinds of this header for mtfm_hta_timing_read() */
enum { MTFM_RMS_KERNEL_FWD = 7,        /* forward, either form */
       MTFM_RMS_KERNEL_BWD = 8,        /* backward: dx and each workgroup's share of dweight */
       MTFM_RMS_KERNEL_BWD_REDUCE = 9  /* sum of the shares */ };

/*
 * Forward.  residual NULL: h must be NULL too (h is x).  With a residual, h receives the sum.  rstd: what the backward
 * pass reads, or NULL.
 */
MTFM_HTA_API int mtfm_rms_fwd(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                 const float* weight, void* h, void* y, float* rstd, int64_t n_rows, int32_t width, float eps, int dtype,
                 void* stream);

/* Forward with an output in 8 bits: q [n_rows][width] of the type `kind`, scale [n_rows]. */
MTFM_HTA_API int mtfm_rms_fwd_q8(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                 const float* weight, void* h, void* q, float* scale, int64_t n_rows, int32_t width, float eps, int dtype,
                 int kind, void* stream);

/* Bytes of device workspace mtfm_rms_bwd() needs (0 if the width is invalid): room for the shares of dweight of 512
 * workgroups, which is what the backward kernel's grid stays within. */
MTFM_HTA_API size_t mtfm_rms_bwd_workspace_bytes(int32_t width);

/*
 * Backward.  h and rstd: the forward pass's (x itself without a residual).  dh may be NULL.  dweight is overwritten
 * (n_rows = 0 zeroes it); its sums are formed in float32 in an order that depends on the sizes alone.  `workspace`: 256-byte
 * aligned, at least mtfm_rms_bwd_workspace_bytes(); contents need not be initialised and are not preserved.
 */
MTFM_HTA_API int mtfm_rms_bwd(const void* dy, int64_t dy_stride, const void* h, int64_t h_stride, const float* weight,
                 const float* rstd, const void* dh, int64_t dh_stride, void* dx, float* dweight, int64_t n_rows,
                 int32_t width, int dtype, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MTFM_RMS_H */
