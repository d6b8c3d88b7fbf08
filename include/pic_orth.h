/*
 * pic_orth.h -- C ABI of orthogonalised updates: for every matrix G of a list,
 * a matrix of the same shape whose singular values are drawn towards one by
 * Newton-Schulz products, as the Muon optimiser takes its steps.
 *
 *   X = G / (|G| + eps)            |G| the Frobenius norm
 *   `steps` times:
 *     A = X X^T                    (with more rows than columns: A = X^T X, and
 *     X = a X + (b A + c A^2) X     X = a X + X (b A + c A^2), which is the same)
 *   out = X
 *
 * With the usual coefficients, 3.4445, -4.7750 and 2.0315, five steps take
 * singular values above 0.01 of the largest to between 0.7 and 1.2.
 *
 * The norm is summed as pic_clip.h's, sums are fp32, and out is rounded once, to
 * nearest.  Matrices of fp32 and fp16: between products X, A and b A + c A^2 are
 * held in two IEEE halves each (22 bits, scaled by 4096), of whose four products
 * three are formed; the fourth is below 2^-22 of a product.  Matrices of
 * bfloat16 do so too where they are small, all of up to 64 on the smaller side
 * among them; of others products take halves of 11 bits, and X has a second one,
 * which is added to a X, but before the last two steps.  Elements of X below 2^-37
 * are lost.  Measured for full matrices, root mean square error of out's own:
 * fp32 1e-6 (64 x 64), 3e-6 (1024 x 1024), 9e-6 (512 x 20000, 2048 x 8192), 2e-5 (4000 x
 * 12000), where elementary fp32 operations have 1.3e-6, 3e-6, 3e-6 and 5e-6, and 8e-6 (a
 * tensor core truncates what it adds); bfloat16 1.7e-3
 * to 2.3e-3, of which its rounding is 1.7e-3.  An infinite or
 * NaN element makes all of its matrix's out NaN (steps > 0), and no other's.
 *
 * Conventions as in pic_decode.h: device pointers owned by the caller,
 * asynchronous on `stream`, pic_status codes, no traps.  Results do not vary
 * from call to call.
 */
#ifndef PIC_ORTH_H
#define PIC_ORTH_H

#include <stddef.h>
#include <stdint.h>

#include "pic_linear.h"

#ifdef __cplusplus
extern "C" {
#endif

/* One matrix: `rows` x `cols` (>= 0 each, below 2^31 - 256) of `dtype`, rows
 * `ld_grad` (>= cols) elements apart, orthogonalised to `out` (ld_out), which
 * is `grad` itself (ld_out = ld_grad) or overlaps no grad and no other out. */
typedef struct {
  const void *grad;
  void *out;
  int64_t rows, cols;
  int64_t ld_grad, ld_out;
  int dtype; /* pic_dtype */
} pic_orth_matrix;

typedef struct pic_orthogonalizer pic_orthogonalizer; /* opaque: the list, and room for X, A and b A + c A^2 */

/* Bytes of device memory that a handle for these matrices holds between calls for X, A and
 * b A + c A^2, of those that are not taken by one CTA each: 8 for every element, each row
 * rounded up to 64 columns, and 4 (bfloat16 above 64 on the smaller side) or 8 for every
 * element of a square matrix of the smaller side.  (Its lists of work and the parts of
 * products take more beside that.)  At most 2^50 or a little above; -1 for a list that
 * pic_orth_create refuses. */
int64_t pic_orth_room_bytes(const pic_orth_matrix *matrices, int n);

/*
 * Creates a handle for n (>= 0) matrices on the current device.  The list is
 * copied; the matrices stay the caller's, and the handle is to be destroyed
 * before they are freed.  Synchronises.
 * Errors: PIC_ERR_INVALID_ARG (NULL or misaligned pointers, sizes or strides
 * out of range, an unknown type, outputs that overlap), PIC_ERR_UNSUPPORTED (a
 * device that is not sm_103), PIC_ERR_ALLOC (the matrices' room does not fit
 * the device, among others), PIC_ERR_CUDA.
 */
int pic_orth_create(const pic_orth_matrix *matrices, int n, pic_orthogonalizer **out);

/*
 * Orthogonalises the handle's matrices as they are when the kernels run.
 * steps in [0, 64], eps >= 0 and finite.  a, b and c are refused where a
 * singular value in [0, 1] would leave [-2, 2] in one of the steps, or
 * |b s^2| + |c s^4| would be above 12 for one it meets.  Calls with one handle
 * must not overlap on the GPU.
 * Errors: PIC_ERR_INVALID_ARG (also for a current device other than the
 * handle's), PIC_ERR_CUDA.
 */
int pic_orth(pic_orthogonalizer *h, int steps, float a, float b, float c, float eps, void *stream);

/* Synchronises `stream`; PIC_OK if no bounded device-side wait of this handle's
 * calls gave up since the last check, PIC_ERR_TIMEOUT if one did (the outs of
 * that call are unspecified), PIC_ERR_CUDA. */
int pic_orth_check(pic_orthogonalizer *h, void *stream);

void pic_orth_destroy(pic_orthogonalizer *h);

#ifdef __cplusplus
}
#endif

#endif /* PIC_ORTH_H */
