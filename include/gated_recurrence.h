/*
 * gated_recurrence.h -- C ABI of the B200 gated linear recurrence: a recurrent layer of one state per channel that is
 * trained on whole rollouts and stepped one token at a time in the policy loop.
 *
 * Beside the selective scan of ssm.h, which mixes `states` states per channel, this is the light mixer: both gates come
 * from projections, the decay is the channel's own rate scaled by its gate, and the input's gain keeps the state's
 * variance what the input's is.  Per channel c:
 *
 *     L_t = a[c] sigmoid(r_t)                        a <= 0: the logarithm of the strongest decay
 *     h_t = e^(L_t) h_{t-1} + sqrt(1 - e^(2 L_t)) sigmoid(i_t) x_t          y_t = h_t
 *
 * Where reset_t is set, h_{t-1} is taken as zero (h may hold anything there, also NaN).
 * Backward, with g_t the gradient of h_t, u_t = sigmoid(i_t) x_t and k_t = sqrt(1 - e^(2 L_t)):
 *
 *     g_t = dy_t + e^(L_{t+1}) g_{t+1}  (0 across a reset at t + 1; dstate_out behind the last step)
 *     dx = g k sigmoid(i)     di = g k x sigmoid(i) (1 - sigmoid(i))
 *     dL = g (e^L h_{t-1} - u e^(2 L) / k)     dr = dL L (1 - sigmoid(r))     da = sum of dL sigmoid(r)
 *     dstate = e^(L_0) g_0
 *
 * a = 0 (and a gate that vanishes in binary32) means no decay and no input; the derivative by the rate has no limit there
 * and counts as zero.  A positive a gives NaN.  A state that has become infinite stays so until a reset; gradients of
 * steps that meet one are not finite.
 *
 * Types.  x, r, i, y, dy and their gradients are of the handle's type (binary32, bfloat16, binary16).  a, the states and
 * their gradients are binary32, as is all arithmetic; a result is rounded once when it is stored.  The decay enters as
 * h + (e^L - 1) h with e^L - 1 to full relative precision, so that slow channels gather no bias; of a fast one e^L is off by
 * 2^-25 of one.  The gates' sigmoids are exact to some units of 2^-24 relative in binary32, in the 16-bit types
 * to the rounding of their argument.  Every sum has a fixed order: the same call gives the same bits.  Single tokens go
 * through the states of the sequence bit for bit where it is taken in one piece (a forward workspace of 0 bytes); a row whose time is
 * cut starts its pieces from chained values, which agree but for roundings.
 *
 * Sequences are described by gated_recurrence_seq: element (n, t, c) of a [batch][time][channels] array is
 * ptr[n * stride_b + t * stride_t + c], strides in elements; batch and time are at least 1.  A time-major rollout
 * [time][batch][channels] is the same array with the strides exchanged; a column range of a wider projection is one with a
 * larger stride_t.  Pointers are DEVICE pointers owned by the caller, aligned to their element.  Outputs must overlap neither
 * inputs nor one another, except that a step may update its state in place.  Outputs whose rows would share memory are
 * refused.
 *
 * Calls enqueue on the handle's stream, on the device that was current when the handle was created (whichever is
 * current now stays so), and return; nothing is allocated but the handle.  A handle is not thread-safe (its stream is
 * set by one call and used by the next): use one handle per host thread or lock.  Return 0 or a negative
 * GATED_RECURRENCE_E* code; no exceptions, aborts, traps or printing; no CPU fallback.
 */
#ifndef GATED_RECURRENCE_H_
#define GATED_RECURRENCE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define GATED_RECURRENCE_OK       0
#define GATED_RECURRENCE_EINVAL (-1)  /* bad size, stride or type */
#define GATED_RECURRENCE_ENULL  (-2)  /* required pointer is NULL */
#define GATED_RECURRENCE_EALIGN (-3)  /* a pointer is not aligned to its element (workspace: 16 bytes) */
#define GATED_RECURRENCE_ECUDA  (-4)  /* a CUDA runtime call or launch failed */
#define GATED_RECURRENCE_ENOMEM (-5)  /* allocation failed, or the workspace is too small */

#define GATED_RECURRENCE_F32  0
#define GATED_RECURRENCE_BF16 1
#define GATED_RECURRENCE_F16  2

#define GATED_RECURRENCE_MAX_CHANNELS 65536

typedef struct gated_recurrence gated_recurrence;

typedef struct gated_recurrence_seq {
    void *ptr;
    int64_t stride_b, stride_t;   /* elements; >= 0 */
} gated_recurrence_seq;

typedef struct gated_recurrence_args {
    int64_t batch, time;
    gated_recurrence_seq x, r, i;     /* in  [batch][time][channels] */
    gated_recurrence_seq reset;       /* in  uint8 [batch][time][1], or ptr NULL: no resets */
    const float *a;                   /* in  [channels] */
    const float *state;               /* in  (forward) [batch][channels] or NULL: zeros */
    float *state_out;                 /* out (forward) [batch][channels] or NULL; not `state` */
    gated_recurrence_seq y;           /* out (forward) */
    float *saved;                     /* forward: out, or NULL if there will be no backward; backward: in */
    gated_recurrence_seq dy;          /* in  (backward) */
    const float *dstate_out;          /* in  (backward): gradient of state_out, or NULL: zeros */
    gated_recurrence_seq dx, dr, di;  /* out (backward) */
    float *da;                        /* out (backward) [channels] */
    float *dstate;                    /* out (backward): gradient of state, or NULL */
    void *workspace;                  /* gated_recurrence_workspace_bytes; forward and backward */
    size_t workspace_bytes;
} gated_recurrence_args;

/* channels: 1..GATED_RECURRENCE_MAX_CHANNELS. */
int gated_recurrence_create(gated_recurrence **out, int channels, int type);
int gated_recurrence_destroy(gated_recurrence *p);
int gated_recurrence_set_stream(gated_recurrence *p, void *cuda_stream);

/* Bytes of `saved`: the state at the start of every block of steps. */
size_t gated_recurrence_saved_bytes(const gated_recurrence *p, int64_t batch, int64_t time);
/* Scratch of a forward (backward = 0) or backward (backward = 1) call; may be 0. */
size_t gated_recurrence_workspace_bytes(const gated_recurrence *p, int64_t batch, int64_t time, int backward);
int gated_recurrence_forward(gated_recurrence *p, const gated_recurrence_args *a);
int gated_recurrence_backward(gated_recurrence *p, const gated_recurrence_args *a);

/* One token of n rows.  x, r, i and y have a row stride in elements; done uint8[n] (stride done_stride) or NULL: where
 * set, the row's state is taken as zeros.  state_out may be state. */
int gated_recurrence_step(gated_recurrence *p, const void *x, int64_t x_stride, const void *r, int64_t r_stride,
                          const void *i, int64_t i_stride, const uint8_t *done, int64_t done_stride, const float *a,
                          const float *state, float *state_out, void *y, int64_t y_stride, int64_t n);

/* kernels launched through this handle so far */
int64_t gated_recurrence_launch_count(const gated_recurrence *p);
const char *gated_recurrence_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* GATED_RECURRENCE_H_ */
