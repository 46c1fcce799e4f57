/*
 * layer_norm.h -- C ABI of the B200 layer norm of a residual stream, forward and backward.
 *
 * What stands between the layers of a sequence policy (ssm.h, gated_recurrence.h, gated_ffn.h): each adds its
 * result to a stream and reads the stream normalised.  Both are one pass over memory here:
 *
 *     s = x + residual                       rounded to the type: the stream as it goes on (s = x without residual)
 *     m = mean s     v = mean (s - m)^2      over the row's `width` elements
 *     q = 1 / sqrt(v + eps)
 *     y = (s - m) q w + b                    w: ones where absent, b: zeros where absent
 *
 * Backward, for dy and, where the stream's own gradient arrives from behind, dsum:
 *
 *     z = (s - m) q     c = dy w
 *     dx = dsum + q (c - mean c - z mean(c z))     the gradient of x and of the residual alike
 *     dw = sum over rows of dy z     db = sum over rows of dy
 *
 * Types.  x, residual, s, y, dy, dsum, dx are of the handle's type (binary32, bfloat16, binary16).  w, b, the saved
 * statistics and dw, db are binary32, as is all arithmetic; a result is rounded once when it is stored.  The variance
 * is summed from differences to the mean, which are formed first.  Every sum has a fixed order: the same call gives the
 * same bits (on arrays of the same strides and alignment).  A row with a NaN or an infinity in it gives NaN in that row
 * (and in dw, db), and in no other.  Where the variance is beyond binary32 (differences of 1e19), q is zero and y is b.
 *
 * Rows are contiguous, `width` elements, with a row stride in elements (inputs: >= 0, so that one row can serve for all;
 * outputs: >= width).  Any width and alignment to the element is taken; rows of whole 16-byte pieces are faster.
 * Pointers are DEVICE pointers owned by the caller.  Outputs must overlap neither one another nor inputs, except in place,
 * with the same pointer and stride: sum may be x or residual, y may be x where there is no residual, dx may be dy or dsum.
 *
 * Calls enqueue on the handle's stream, on the device that was current when the handle was created (whichever is
 * current now stays so), and return; nothing is allocated but the handle.  A handle is not thread-safe (its stream is
 * set by one call and used by the next): use one handle per host thread or lock.  Return 0 or a negative
 * LAYER_NORM_E* code; no exceptions, aborts, traps or printing; no CPU fallback.
 */
#ifndef LAYER_NORM_H_
#define LAYER_NORM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LAYER_NORM_OK       0
#define LAYER_NORM_EINVAL (-1)  /* bad size, stride, eps or type */
#define LAYER_NORM_ENULL  (-2)  /* required pointer is NULL */
#define LAYER_NORM_EALIGN (-3)  /* a pointer is not aligned to its element (saved: 8 bytes, workspace: 16) */
#define LAYER_NORM_ECUDA  (-4)  /* a CUDA runtime call or launch failed */
#define LAYER_NORM_ENOMEM (-5)  /* allocation failed, or the workspace is too small */

#define LAYER_NORM_F32  0
#define LAYER_NORM_BF16 1
#define LAYER_NORM_F16  2

#define LAYER_NORM_MAX_WIDTH 8192

typedef struct layer_norm layer_norm;

/* width: 1..LAYER_NORM_MAX_WIDTH; eps: positive and finite. */
int layer_norm_create(layer_norm **out, int width, float eps, int type);
int layer_norm_destroy(layer_norm *p);
int layer_norm_set_stream(layer_norm *p, void *cuda_stream);

/* residual and sum: both or neither.  w, b may be NULL.  saved: float [n][2] (m and q of each row), or NULL if there
 * will be no backward pass.  n >= 1. */
int layer_norm_forward(layer_norm *p, const void *x, int64_t x_stride, const void *residual, int64_t residual_stride,
                       const float *w, const float *b, void *sum, int64_t sum_stride, void *y, int64_t y_stride,
                       float *saved, int64_t n);

/* Scratch of a backward call on n rows (0 where neither dw nor db is wanted). */
size_t layer_norm_workspace_bytes(const layer_norm *p, int64_t n);

/* s: the rows that were normalised (the forward call's sum, or its x).  dsum may be NULL: zeros.  dw and db: both or
 * neither. */
int layer_norm_backward(layer_norm *p, const void *dy, int64_t dy_stride, const void *s, int64_t s_stride,
                        const float *w, const float *saved, const void *dsum, int64_t dsum_stride, void *dx,
                        int64_t dx_stride, float *dw, float *db, void *workspace, size_t workspace_bytes, int64_t n);

/* kernels launched through this handle so far */
int64_t layer_norm_launch_count(const layer_norm *p);
const char *layer_norm_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* LAYER_NORM_H_ */
