/*
 * ssm.h -- C ABI of the B200 state-space sequence library: the short causal
 * convolution and the selective state space scan of a recurrent policy that is
 * trained on whole rollouts and stepped one token at a time in the policy loop.
 *
 * The GRU of gru_policy.h steps; it has no form for a whole sequence.  The
 * operators here have three: a sequence (a prompt, or a rollout with episode ends
 * inside), its gradients, and a single token, all of the same recurrence.
 *
 * Convolution, per channel, `width` taps, oldest first:
 *
 *     u_t = bias + sum_k w[k] x[t - width + 1 + k]          y_t = u_t sigmoid(u_t)
 *
 * Taps before the sequence come from `history` (the last width - 1 inputs, oldest
 * first) or are zero; taps before the episode that t belongs to are dropped.
 *
 * Scan, per channel d of group g, with `states` states n:
 *
 *     delta_t = softplus(dt_t + dt_bias)
 *     h_t[n]  = exp(delta_t a[n]) h_{t-1}[n] + delta_t x_t b_t[g][n]
 *     y_t     = (sum_n c_t[g][n] h_t[n] + d x_t) * z_t sigmoid(z_t)
 *
 * Where reset_t is set, h_{t-1} is taken as zero (h may hold anything there, also
 * NaN).  d, dt_bias and z may be absent: no skip term, no bias, no gate.
 *
 * Types.  x, dt, z, b, c, y, their gradients and the history are of the handle's
 * type (binary32, bfloat16, binary16).  Parameters (w, bias, a, d, dt_bias),
 * recurrent states and all their gradients are binary32, as is all arithmetic; a
 * result is rounded once when it is stored.  Every sum has a fixed order: the same
 * call gives the same bits.
 *
 * Sequences are described by ssm_seq: element (i, t, f) of a [batch][time][features]
 * array is ptr[i * stride_b + t * stride_t + f], strides in elements.  A time-major
 * rollout [time][batch][features] is the same array with the strides exchanged; a
 * column range of a wider projection is one with a larger stride_t.  Pointers are
 * DEVICE pointers owned by the caller, aligned to their element.  Inputs must not
 * overlap outputs, except that a step may update its state or history in place.
 *
 * Calls enqueue on the handle's stream, on the device that was current when the handle was
 * created (whichever is current now stays so), and return; nothing is allocated but the
 * handle.  A handle is not thread-safe (its stream is set by one call and used by the next): use one
 * handle per host thread or lock.  Return 0 or a negative SSM_E* code; no exceptions, aborts, traps or
 * printing; no CPU fallback.
 */
#ifndef SSM_H_
#define SSM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SSM_OK       0
#define SSM_EINVAL (-1)  /* bad size, stride or type */
#define SSM_ENULL  (-2)  /* required pointer is NULL */
#define SSM_EALIGN (-3)  /* a pointer is not aligned to its element (state, saved, workspace: 16 bytes) */
#define SSM_ECUDA  (-4)  /* a CUDA runtime call or launch failed */
#define SSM_ENOMEM (-5)  /* allocation failed, or the workspace is too small */

#define SSM_F32  0
#define SSM_BF16 1
#define SSM_F16  2

#define SSM_MAX_CHANNELS 65536
#define SSM_MAX_STATES   64
#define SSM_MAX_WIDTH    4

typedef struct ssm ssm;

typedef struct ssm_seq {
    void *ptr;
    int64_t stride_b, stride_t;   /* elements; >= 0 */
} ssm_seq;

/* channels: 1..SSM_MAX_CHANNELS, a multiple of groups; states: 1..SSM_MAX_STATES;
 * width: 2..SSM_MAX_WIDTH; type: SSM_F32, SSM_BF16 or SSM_F16. */
int ssm_create(ssm **out, int channels, int states, int groups, int width, int type);
int ssm_destroy(ssm *p);
int ssm_set_stream(ssm *p, void *cuda_stream);

/* ---- convolution.  w[channels][width] and bias[channels] are binary32. ---- */

typedef struct ssm_conv_args {
    int64_t batch, time;
    ssm_seq x;              /* in  [batch][time][channels] */
    ssm_seq reset;          /* in  uint8 [batch][time][1], or ptr NULL: no resets */
    const float *w, *bias;  /* bias may be NULL */
    const void *history;    /* in  [batch][width - 1][channels], contiguous, or NULL: zeros */
    ssm_seq y;              /* out (forward) */
    void *history_out;      /* out (forward) [batch][width - 1][channels] or NULL; not `history` */
    ssm_seq dy;             /* in  (backward) */
    ssm_seq dx;             /* out (backward); the history is taken as a constant */
    float *dw, *dbias;      /* out (backward) [channels][width], [channels]; dbias may be NULL */
    void *workspace;        /* backward: ssm_conv_workspace_bytes */
    size_t workspace_bytes;
} ssm_conv_args;

size_t ssm_conv_workspace_bytes(const ssm *p, int64_t batch, int64_t time);
int ssm_conv_forward(ssm *p, const ssm_conv_args *a);
int ssm_conv_backward(ssm *p, const ssm_conv_args *a);
/* One token of n rows.  x and y have a row stride in elements; done uint8[n] (stride done_stride)
 * or NULL: where set, the row's history is taken as zeros.  history_out may be history. */
int ssm_conv_step(ssm *p, const void *x, int64_t x_stride, const uint8_t *done, int64_t done_stride,
                  const float *w, const float *bias, const void *history, void *history_out, void *y,
                  int64_t y_stride, int64_t n);

/* ---- scan.  a[channels][states], d[channels], dt_bias[channels] are binary32. ---- */

typedef struct ssm_scan_args {
    int64_t batch, time;
    ssm_seq x, dt;          /* in  [batch][time][channels] */
    ssm_seq z;              /* in  [batch][time][channels] or ptr NULL */
    ssm_seq b, c;           /* in  [batch][time][groups * states] */
    ssm_seq reset;          /* in  uint8 [batch][time][1] or ptr NULL */
    const float *a, *d, *dt_bias;   /* d, dt_bias may be NULL */
    const float *state;     /* in  (forward) [batch][channels][states] or NULL: zeros */
    float *state_out;       /* out (forward) [batch][channels][states] or NULL; not `state` */
    ssm_seq y;              /* out (forward) */
    float *saved;           /* forward: out, or NULL if there will be no backward; backward: in */
    ssm_seq dy;             /* in  (backward) */
    const float *dstate_out;   /* in  (backward): gradient of state_out, or NULL: zeros */
    ssm_seq dx, ddt, dz, db, dc;   /* out (backward); dz.ptr NULL exactly where z.ptr is */
    float *da, *dd, *ddt_bias;     /* out (backward); dd, ddt_bias may be NULL */
    float *dstate;          /* out (backward): gradient of state, or NULL */
    void *workspace;        /* ssm_scan_workspace_bytes; forward and backward */
    size_t workspace_bytes;
} ssm_scan_args;

/* Bytes of `saved`: the recurrent state at the start of every block of steps. */
size_t ssm_scan_saved_bytes(const ssm *p, int64_t batch, int64_t time);
/* Scratch of a forward (backward = 0) or backward (backward = 1) call; may be 0. */
size_t ssm_scan_workspace_bytes(const ssm *p, int64_t batch, int64_t time, int backward);
int ssm_scan_forward(ssm *p, const ssm_scan_args *a);
int ssm_scan_backward(ssm *p, const ssm_scan_args *a);

/* One token of n rows: the recurrence above with t a single step.  state_out may be state. */
int ssm_scan_step(ssm *p, const void *x, int64_t x_stride, const void *dt, int64_t dt_stride,
                  const void *z, int64_t z_stride, const void *b, int64_t b_stride, const void *c,
                  int64_t c_stride, const uint8_t *done, int64_t done_stride, const float *a,
                  const float *d, const float *dt_bias, const float *state, float *state_out, void *y,
                  int64_t y_stride, int64_t n);

/* kernels launched through this handle so far */
int64_t ssm_launch_count(const ssm *p);
const char *ssm_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* SSM_H_ */
