/*
 * gated_ffn.h -- C ABI of the B200 gated feed-forward block, forward and backward.
 *
 * The other half of a sequence-policy layer beside the recurrence of ssm.h:
 *
 *     [g | u] = x W_in^T            both projections in one product
 *     hidden  = act(g) * u          formed where the accumulators are
 *     y       = hidden W_out^T
 *
 * x[n][model], W_in[2 * hidden][model] (the gate's rows, then the other projection's),
 * W_out[model][hidden].  act is silu, v sigmoid(v), or gelu in its tanh form,
 * 0.5 v (1 + tanh(sqrt(2 / pi) (v + 0.044715 v^3))).  Backward, for dy[n][model]:
 *
 *     dhidden = dy W_out      dg = dhidden u act'(g)      du = dhidden act(g)
 *     dx = [dg | du] W_in     dW_in = [dg | du]^T x       dW_out = dy^T hidden
 *
 * Types.  Everything the caller passes is bfloat16 or binary16, one type per handle.
 * Products run on the tensor cores and accumulate in binary32.  Rounded to the type:
 * results; hidden, dg and du, which are operands of further products (in binary16 they are
 * infinite beyond 65,504).  g and u are kept for the backward pass (`pre`) with the upper 24
 * bits of their binary32 values, cut off: within 2^-15, always towards zero (adding half a unit
 * first could carry a NaN over into a number), which the rounding of dg and du exceeds by far.  The
 * activation and its slope are binary32; hidden comes from the unrounded g and u.  The
 * accumulation order inside the tensor cores is not specified; the same call gives the
 * same bits.
 *
 * model and hidden are multiples of 8 (16-byte rows); n is any.  Weights and saved
 * buffers are contiguous; x, y, dy, dx have a row stride in elements (multiple of 8).
 * Pointers are DEVICE pointers owned by the caller, 16-byte aligned; inputs must not
 * overlap outputs.  Calls enqueue on the handle's stream, on the device that was current when
 * the handle was created (whichever is current now stays so), and return
 * (gated_ffn_status synchronises).  A handle is not thread-safe (its stream is set by one call
 * and used by the next): use one handle per host thread or lock.  The library allocates only in
 * gated_ffn_create.
 * Return 0 or a negative GATED_FFN_E* code; no exceptions, aborts, traps or printing;
 * no CPU fallback.
 */
#ifndef GATED_FFN_H_
#define GATED_FFN_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define GATED_FFN_OK        0
#define GATED_FFN_EINVAL   (-1)  /* bad size, stride, type or activation */
#define GATED_FFN_ENULL    (-2)  /* required pointer is NULL */
#define GATED_FFN_EALIGN   (-3)  /* pointer not 16-byte aligned */
#define GATED_FFN_ECUDA    (-4)  /* a CUDA call or launch failed */
#define GATED_FFN_ENOMEM   (-5)  /* allocation failed, or the workspace is too small */
#define GATED_FFN_ETIMEOUT (-6)  /* a kernel gave up a bounded wait; its output is invalid */

#define GATED_FFN_BF16 0
#define GATED_FFN_F16  1
#define GATED_FFN_SILU 0
#define GATED_FFN_GELU 1

#define GATED_FFN_MAX_WIDTH 65536   /* largest model and hidden */

typedef struct gated_ffn gated_ffn;

int gated_ffn_create(gated_ffn **out, int model, int hidden, int activation, int type);
int gated_ffn_destroy(gated_ffn *p);
int gated_ffn_set_stream(gated_ffn *p, void *cuda_stream);

/* Scratch of a forward (backward = 0) or backward (backward = 1) call on n rows. */
size_t gated_ffn_workspace_bytes(const gated_ffn *p, int64_t n, int backward);

/* Bytes of `pre` for n rows: g and u in a layout of the library's own. */
size_t gated_ffn_pre_bytes(const gated_ffn *p, int64_t n);

/* hidden[n][hidden] and, if there will be a backward pass, pre (else NULL) are written: the backward
 * call reads both, with the same n.  n >= 1. */
int gated_ffn_forward(gated_ffn *p, const void *x, int64_t x_stride, const void *w_in, const void *w_out,
                      void *pre, void *hidden, void *y, int64_t y_stride, void *workspace,
                      size_t workspace_bytes, int64_t n);

/* dw_in[2 * hidden][model], dw_out[model][hidden]; dx may be NULL (the first layer). */
int gated_ffn_backward(gated_ffn *p, const void *dy, int64_t dy_stride, const void *x, int64_t x_stride,
                       const void *w_in, const void *w_out, const void *pre, const void *hidden, void *dx,
                       int64_t dx_stride, void *dw_in, void *dw_out, void *workspace,
                       size_t workspace_bytes, int64_t n);

/* Synchronises the stream; GATED_FFN_ETIMEOUT if any kernel since the last call gave up
 * a wait (clears the flag), GATED_FFN_ECUDA on a CUDA error, else 0. */
int gated_ffn_status(gated_ffn *p);

/* kernels launched through this handle so far */
int64_t gated_ffn_launch_count(const gated_ffn *p);
const char *gated_ffn_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* GATED_FFN_H_ */
