/*
 * orthogonal.h -- C ABI of the B200 orthogonalised update: the step that an optimiser takes for a weight matrix when it
 * gives every direction of the momentum the same size.
 *
 * For G [rows][cols], with k = min(rows, cols):
 *
 *     X = G / (|G| + eps)                           |G|: square root of the sum of squares
 *     `steps` times:   A = X X^T  (X^T X if rows > cols)      B = b A + c A A      X = a X + B X  (a X + X B)
 *     update = X
 *
 * The singular vectors stay; each singular value s goes through p(s) = a s + b s^3 + c s^5.  With the usual coefficients
 * (3.4445, -4.7750, 2.0315) five steps bring everything above about 0.002 |G| to between 0.7 and 1.2.
 *
 * Types.  G is binary32, bfloat16 or binary16, one type per handle; the update is bfloat16 whatever G is (the polynomial
 * itself leaves the singular values a third apart).  |G| is summed in binary64.  The products run on the tensor cores with
 * binary16 operands and binary32 accumulation.  What a rounding of operands would cost is kept out of them: X is held as
 * the sum of two binary16 numbers (22 bits) wherever it is not an operand, and the diagonals of A and B, which are of the
 * size of the whole result late in the iteration, are binary32 and enter the products as exact row or column factors.
 * Against binary64 the update is off by its own rounding (1.7e-3 relative, root mean square) and 2e-4 to 8e-4 more; an
 * exactly rank-deficient G by up to 2e-3 more (the directions that are not there take up rounding errors).  So an evaluation
 * in binary32 differs from it by 1.2e-3 (root mean square), whatever the type of G.  X is held
 * times 2^13 and stays finite as long as none of its elements exceeds 7 in magnitude, which the usual coefficients
 * keep; other ones are the caller's choice.  The same call gives the same bits.  An infinity or NaN in a
 * matrix gives NaN in its update, and in no other matrix's.
 *
 * G and update are [batch][rows][cols] with contiguous rows, strides in elements.  Pointers are DEVICE pointers owned by
 * the caller, aligned to their element; the update must not overlap G.
 *
 * Calls enqueue on the handle's stream, on the device that was current when the handle was created (whichever is
 * current now stays so), and return (orthogonal_status synchronises).  A handle is not thread-safe (its stream is set by
 * one call and used by the next): use one handle per host thread or lock.  The library allocates only in
 * orthogonal_create.  Return 0 or a negative ORTHOGONAL_E* code; no exceptions, aborts, traps or printing; no CPU
 * fallback.
 */
#ifndef ORTHOGONAL_H_
#define ORTHOGONAL_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ORTHOGONAL_OK        0
#define ORTHOGONAL_EINVAL   (-1)  /* bad size, stride, type, steps, coefficient or eps */
#define ORTHOGONAL_ENULL    (-2)  /* required pointer is NULL */
#define ORTHOGONAL_EALIGN   (-3)  /* a pointer is not aligned to its element (workspace: 256 bytes) */
#define ORTHOGONAL_ECUDA    (-4)  /* a CUDA call or launch failed */
#define ORTHOGONAL_ENOMEM   (-5)  /* allocation failed, or the workspace is too small */
#define ORTHOGONAL_ETIMEOUT (-6)  /* a kernel gave up a bounded wait; its output is invalid */

#define ORTHOGONAL_F32  0
#define ORTHOGONAL_BF16 1
#define ORTHOGONAL_F16  2

#define ORTHOGONAL_MAX_SIDE  65536
#define ORTHOGONAL_MAX_STEPS 32

typedef struct orthogonal orthogonal;

/* rows, cols: 1..ORTHOGONAL_MAX_SIDE; steps: 1..ORTHOGONAL_MAX_STEPS; a, b, c finite; eps: positive and finite. */
int orthogonal_create(orthogonal **out, int rows, int cols, int steps, float a, float b, float c, float eps, int type);
int orthogonal_destroy(orthogonal *p);
int orthogonal_set_stream(orthogonal *p, void *cuda_stream);

/* Scratch of a call on `batch` matrices; may be 0. */
size_t orthogonal_workspace_bytes(const orthogonal *p, int64_t batch);

/* batch >= 1 matrices, each by itself. */
int orthogonal_update(orthogonal *p, const void *g, int64_t g_stride_batch, int64_t g_stride_row, void *update,
                      int64_t update_stride_batch, int64_t update_stride_row, void *workspace, size_t workspace_bytes,
                      int64_t batch);

/* Synchronises the stream; ORTHOGONAL_ETIMEOUT if any kernel since the last call gave up a wait (clears the flag),
 * ORTHOGONAL_ECUDA on a CUDA error, else 0. */
int orthogonal_status(orthogonal *p);

/* kernels launched through this handle so far */
int64_t orthogonal_launch_count(const orthogonal *p);
const char *orthogonal_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* ORTHOGONAL_H_ */
