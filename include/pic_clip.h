/*
 * pic_clip.h -- C ABI of the global gradient norm over many tensors, and of
 * clipping by it:
 *
 *   norm = sqrt(sum of the squares of all elements of all tensors)
 *   coef = min(1, max_norm / (norm + 1e-6)),   out = coef * grad
 *
 * The squares are summed in fp32 within short runs and in fp64 across them,
 * and a run whose sum leaves fp32's range is summed again in fp64: finite
 * gradients of any size are clipped as the formula says.  The norm is returned
 * in fp32: one above fp32's largest value is infinite there (coef is then
 * computed from the fp64 sum).  If an element is infinite or NaN, so is the
 * norm, and the outputs are what the formula gives: NaN where coef or the
 * element is NaN, or for an infinite element times coef = 0.  With max_norm
 * infinite coef is 1, whatever the norm.  coef and the products are fp32 (a
 * coef below 2^-126 has fewer bits); a product is rounded once, to nearest, to
 * the tensor's type.
 *
 * Conventions as in pic_decode.h: device pointers owned by the caller,
 * asynchronous on `stream`, pic_status codes, no traps.
 */
#ifndef PIC_CLIP_H
#define PIC_CLIP_H

#include <stddef.h>
#include <stdint.h>

#include "pic_linear.h"

#ifdef __cplusplus
extern "C" {
#endif

/* One gradient tensor: `count` (>= 0) consecutive elements of `dtype`, clipped
 * to `out`, which is `grad` itself or overlaps no gradient and no other out. */
typedef struct {
  const void *grad;
  void *out;
  int64_t count;
  int dtype; /* pic_dtype */
} pic_clip_tensor;

typedef struct pic_clipper pic_clipper; /* opaque: the list of tensors, and room for partial sums */

/*
 * Creates a handle for n (>= 0) tensors on the current device.  The list is
 * copied; the tensors stay the caller's, and the handle is to be destroyed
 * before they are freed.  Synchronises.
 * Errors: PIC_ERR_INVALID_ARG (NULL or misaligned pointers, a negative count,
 * an unknown type, outputs that overlap), PIC_ERR_UNSUPPORTED (a device that
 * is not sm_103), PIC_ERR_ALLOC, PIC_ERR_CUDA.
 */
int pic_clip_create(const pic_clip_tensor *tensors, int n, pic_clipper **out);

/*
 * Computes the norm of the handle's tensors as they are when the launch runs,
 * writes it to norm (float, device, [1]) and the clipped tensors to their
 * outs.  max_norm >= 0; infinity clips nothing (tensors clipped in place are
 * then only read).  Calls with one handle must not overlap on the GPU.
 * Errors: PIC_ERR_INVALID_ARG (NULL or misaligned pointers, max_norm negative
 * or NaN, a current device other than the handle's), PIC_ERR_CUDA.  The launch
 * is cooperative: all its blocks are on the GPU at once.
 */
int pic_clip(pic_clipper *c, float max_norm, float *norm, void *stream);

/* Synchronises `stream`; PIC_OK if the blocks of every launch of this handle
 * since the last check met in time, PIC_ERR_TIMEOUT if those of one did not (its
 * outs are not all written then, and its norm is unspecified: it may look right,
 * so a program that must know asks here), PIC_ERR_CUDA. */
int pic_clip_check(pic_clipper *c, void *stream);

void pic_clip_destroy(pic_clipper *c);

#ifdef __cplusplus
}
#endif

#endif /* PIC_CLIP_H */
