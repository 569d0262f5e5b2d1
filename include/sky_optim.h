/*
 * sky_optim.h -- parameter updates of tensors that no slice owns.
 *
 * sky_slice_optimizer_step (sky_slice.h) updates the layers of a slice.  What stands
 * beside them (experts in the place of a feed-forward block, a router, a decoder's
 * weights) is updated here: one call for any number of tensors, with AdamW's moments in
 * 32 bits or in 8.  The common rules of sky_ops.h hold: pointers are device pointers of
 * the caller's, nothing is allocated, all work is enqueued on `stream`.
 */
#ifndef SKY_OPTIM_H
#define SKY_OPTIM_H

#include <stddef.h>
#include <stdint.h>

#include "sky_slice.h"

#ifdef __cplusplus
extern "C" {
#endif

/* How the two moments of a tensor are held.
 *   FP32: m and v as they are.
 *   8BIT: m and r = sqrt(v) in one byte a value, with a fp32 scale for every
 *         SKY_STATE_BLOCK consecutive values of the tensor (the last block may be
 *         shorter).  m is the e4m3 number of its byte times the block's scale, the scale
 *         being the block's largest |m| / 448.  r's byte c > 0 is
 *         (1 + (c % 16) / 16) 2^(floor(c / 16) - 16) times the block's scale, the scale
 *         being the largest r / 0.96875, and c = 0 is 0; the root is held because its
 *         range is half of v's.  Both are rounded to nearest (ties to even), and no r
 *         above 0 becomes 0, so m never meets a vanished v.  A block whose largest
 *         value is below 1e-30 is all 0.  The update itself uses the moments before they
 *         are rounded.  A change of a moment by less than half a step (1/16 of m, 1/32
 *         of r, at most) beside its block's largest is not kept.
 *         So r does not end at its 32-bit value but near it: over 24576 values and 12000
 *         steps of N(0, 1) gradients, of one size in a block or of sizes up to a
 *         hundredfold apart, it settles at 0.77 to 1.47 times that (5th to 95th percentile;
 *         the median 0.98 to 1.19) with beta2 of 0.99 to 0.9999, and at 0.94 to 1.07 with
 *         0.95.  It follows gradients that shrink together.
 * Tensors of zeros are the moments before the first step, in either form. */
typedef enum { SKY_STATE_FP32 = 0, SKY_STATE_8BIT = 1 } sky_state_type;
#define SKY_STATE_BLOCK 256

/* One tensor of n values. */
typedef struct {
  float* w;           /* master weights, rewritten                                   */
  const void* g;      /* gradients, in the call's grad_dtype                         */
  void* m;            /* first moment: fp32 or bytes, by the call's states           */
  void* v;            /* second moment: v in fp32, or r's bytes                      */
  float* m_scale;     /* 8BIT: [ceil(n / SKY_STATE_BLOCK)] scales; else unused       */
  float* v_scale;
  void* p;            /* bf16 copy of the weights, rewritten (round to nearest); or NULL */
  int64_t n;
  int32_t decay;      /* 1: weight decay applies, 0: not                             */
} sky_adamw_tensor;

typedef struct {
  float lr;             /* finite, >= 0                                              */
  float beta1, beta2;   /* in [0, 1)                                                 */
  float eps;            /* finite, >= 2^-126 (its inverse is taken)                  */
  float weight_decay;   /* finite, >= 0                                              */
  int64_t step;         /* t >= 1, this update's number                              */
  sky_dtype grad_dtype;
  sky_state_type states;
} sky_adamw_config;

/* What changes from step to step, in device memory: for calls captured into a graph,
 * whose values by argument would stay those of the capture. */
typedef struct {
  float lr;           /* in the place of the config's                                */
  float correction1;  /* 1 - beta1^t                                                 */
  float correction2;  /* 1 - beta2^t                                                 */
  float grad_scale;   /* what gradients are multiplied by (clipping, loss scaling)   */
} sky_adamw_now;

/* One AdamW step of every tensor (the rule of sky_slice_optimizer_step):
 *   g <- grad_scale g,  m <- beta1 m + (1 - beta1) g,  v <- beta2 v + (1 - beta2) g^2,
 *   w <- w - lr weight_decay w  (where decay is 1),
 *   w <- w - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps),  p <- bf16(w).
 * `tensors` is host memory, read before the call returns.  d_now: NULL (lr and step of
 * the config, gradients as they are) or a device pointer read when the work runs.
 * Tensors may start anywhere on their types' grids (on 16 bytes they are faster), and may
 * not overlap each other.  A gradient that is not finite leaves its value, and in 8 bits
 * its whole block's moments, not finite; a finite one whose square overflows fp32 does so
 * to its second moment, in 8 bits to both of its whole block.
 * Errors: INVALID_ARG (null, n_tensors < 1, n < 1, the ranges above, a pointer off its
 * type's grid), UNSUPPORTED (more than 2^40 values in a tensor, or 2^41 in all), CUDA. */
sky_status sky_adamw_step(const sky_adamw_config* config, const sky_adamw_tensor* tensors,
                          int32_t n_tensors, const sky_adamw_now* d_now, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SKY_OPTIM_H */
