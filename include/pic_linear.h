/*
 * pic_linear.h -- C ABI of one linear layer and its gradient: the building
 * block with which the nets that pic_decode runs (MLP^s, MLP^i, arxiv
 * 2609.09020 Sec. 3.1) and the nets around them are trained and evaluated
 * outside the fused decode.
 *
 *   forward   z = x w^T + b,  y = act(z) + residual
 *   backward  dz = dy * act'(z),  dx = dz w,  dw = dz^T x,  db = sum_rows dz
 *             (the residual's gradient is dy itself)
 *   act       none, ReLU (max(z, 0), derivative 1 where z > 0, else 0, at NaN
 *             too) or GELU in its erf form (z Phi(z), derivative Phi(z) + z
 *             phi(z)); dz is 0 where the derivative is, whatever dy is
 *
 * Matrices are row-major with unit stride inside a row and `ld` elements from
 * row to row: x [rows][in], w [out][in] (the layout of pic_decode.h's blobs),
 * y, residual, pre and dy [rows][out].  All tensors of a call have one type:
 * fp32 (PIC_DTYPE_F32), IEEE half (PIC_DTYPE_F16) or bfloat16
 * (PIC_DTYPE_BF16).  Sums are held in fp32; outputs are rounded once, to
 * nearest.  In the backward pass of a 16-bit type, dz is rounded to that type
 * before the products (but for db, and for dw of up to 15 rows).
 *
 * Products run on the tensor cores, which truncate when they add to a sum:
 * after at most 1024 additions of 16 terms (fp32: 48) a sum is taken over and
 * added to nearest, so that less than 2^-13 of a 16-bit type's sum of terms of
 * one sign is lost, below the rounding of the output.  fp32 operands (but
 * for a few rows, which the FP32 cores take) are cut into three bfloat16 pieces,
 * which hold 24 bits, or fewer of values below 2^-110 in size; of a product of
 * two values less than 2^-23 is left out.  Measured, root mean square, of sums of 1024: 6e-7, as much as fp32
 * FMAs in order.
 *
 * Conventions as in pic_decode.h: device pointers owned by the caller and
 * aligned to their element, asynchronous on `stream`, pic_status codes, no
 * traps.  Nothing is allocated; calls that overlap on the GPU need workspaces
 * of their own.  Results do not vary from call to call.
 */
#ifndef PIC_LINEAR_H
#define PIC_LINEAR_H

#include <stddef.h>
#include <stdint.h>

#include "pic_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { PIC_DTYPE_F32 = 0, PIC_DTYPE_F16 = 1, PIC_DTYPE_BF16 = 2 } pic_dtype;

/* A linear layer without activation; the others are pic_act's. */
#define PIC_ACT_NONE 2

/* rows >= 0, in_features >= 1, out_features >= 1, each below 2^31 - 256. */
typedef struct {
  int64_t rows, in_features, out_features;
  int dtype; /* pic_dtype */
  int act;   /* PIC_ACT_NONE, PIC_ACT_RELU or PIC_ACT_GELU */
  const void *x;
  int64_t ldx; /* >= in_features */
  const void *w;
  int64_t ldw;      /* >= in_features */
  const void *bias; /* [out_features], or NULL */
  const void *residual; /* [rows][out_features], or NULL; may be y itself (ldr = ldy) */
  int64_t ldr;      /* >= out_features, or 0: one row for all */
  void *y;
  int64_t ldy; /* >= out_features */
  void *pre;   /* receives z for the backward pass, or NULL */
  int64_t ldpre;
} pic_linear_args;

/* Bytes of device workspace that pic_linear needs for these sizes, types,
 * strides and pointers (it may be 0), or -1 for arguments it would refuse. */
int64_t pic_linear_workspace_bytes(const pic_linear_args *a);

/*
 * The forward layer.  With rows = 0 nothing is launched.  Outputs overlap
 * neither inputs nor each other, but for residual == y.
 * Errors: PIC_ERR_INVALID_ARG (NULL or misaligned pointers, sizes, strides,
 * type or activation out of range, workspace too small or not 256-byte
 * aligned) with nothing launched; PIC_ERR_UNSUPPORTED (a device that is not
 * sm_103); PIC_ERR_CUDA.
 */
int pic_linear(const pic_linear_args *a, void *workspace, size_t workspace_bytes, void *stream);

typedef struct {
  int64_t rows, in_features, out_features;
  int dtype;
  int act;
  const void *dy;
  int64_t lddy;
  const void *x; /* read for dw; may be NULL without dw */
  int64_t ldx;
  const void *w; /* read for dx; may be NULL without dx */
  int64_t ldw;
  const void *pre; /* z of the forward pass (ReLU without residual: y will do, it
                      has z's sign); may be NULL with PIC_ACT_NONE */
  int64_t ldpre;
  void *dx; /* [rows][in_features], or NULL: not computed */
  int64_t lddx;
  void *dw; /* [out_features][in_features], or NULL */
  int64_t lddw;
  void *db; /* [out_features], or NULL */
} pic_linear_grad_args;

int64_t pic_linear_backward_workspace_bytes(const pic_linear_grad_args *a);

/* The gradients that are asked for (at least one).  With rows = 0, dw and db
 * are set to zero.  Errors as for pic_linear. */
int pic_linear_backward(const pic_linear_grad_args *a, void *workspace, size_t workspace_bytes,
                        void *stream);

/* Synchronises `stream`; PIC_OK if no bounded device-side wait of these calls
 * on the current device gave up since the last check, PIC_ERR_TIMEOUT if one
 * did (its outputs are unspecified), PIC_ERR_CUDA. */
int pic_linear_check(void *stream);

/*
 * Test hook of the bounded device-side waits, as pic_decode_test_wait_fault:
 * while withhold_arrival = 1, one warp of the first tile of every tensor-memory
 * kernel skips one mbarrier arrival, so that a later wait of that CTA runs out
 * (after spin_limit polls, where that is not 0) and the kernel takes its abort
 * path.  pic_linear_test_wait_fault(0, 0) restores production behaviour.
 * Errors: PIC_ERR_INVALID_ARG (withhold_arrival not 0 or 1).
 */
int pic_linear_test_wait_fault(int withhold_arrival, unsigned spin_limit);

#ifdef __cplusplus
}
#endif

#endif /* PIC_LINEAR_H */
