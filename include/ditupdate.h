/*
 * ditupdate.h -- the end of a policy update, in libditstep.so and under the conventions of ditstep.h: the norm over the
 * gradients of all weights, clipping by it, and the weights' AdamW step. The clip factor stays on the device: an update
 * needs neither a host synchronisation nor a pass over the gradients for it.
 *
 *   grad_norm    the 2-norm over many tensors, and the factor that clips it
 *   grad_clip    gradients times that factor, in place
 *   adamw_step   decoupled-decay Adam over many tensors, with the factor applied by the way
 *
 * Many tensors are given as a host array of descriptors, which is read during the call (a captured call holds what it
 * said). A tensor is `count` elements without gaps, at any address its type allows; count 0 is fine. Tensors that a call
 * writes must not overlap each other or another tensor of the call. At most 2^20 tensors and 2^44 elements in all.
 * Calls have a launch for every 192 (norm, clip) or 64 (AdamW) tensors. Every result is the same from run to run.
 */
#ifndef DITUPDATE_H
#define DITUPDATE_H

#include <stddef.h>
#include <stdint.h>

#include "ditstep.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  void* data;
  int64_t count;
  int32_t dtype;      /* dit_dtype; tensors of a call may have different types */
  int32_t reserved;   /* 0 */
} dit_gradient;

/* Workspace bytes of grad_norm (0 for an invalid list; `data` is not looked at). */
size_t grad_norm_workspace_bytes(const dit_gradient* grads, int32_t n);

/* *norm (device fp64, may be NULL) = sqrt(sum of g^2 over all elements of all tensors), summed in fp64 in a fixed order, and
 * *scale (device fp32, may be NULL) = min(1, max_norm / (norm + 1e-6)), or NaN where the norm is not finite (a gradient is
 * NaN or infinite; finite gradients have a finite norm). max_norm >= 0; infinity: scale is 1 wherever the norm is finite.
 * A list of no elements has norm 0. Errors: DIT_ERR_DOMAIN for max_norm < 0 or NaN; DIT_ERR_WORKSPACE. */
dit_status grad_norm(const dit_gradient* grads, int32_t n, double max_norm, double* norm, float* scale, void* workspace,
                     size_t workspace_bytes, dit_stream stream);

/* g *= *scale for every tensor, in fp32 with one rounding. Nothing is written where *scale is 1; where it is NaN every gradient
 * becomes NaN. */
dit_status grad_clip(const dit_gradient* grads, int32_t n, const float* scale, dit_stream stream);

typedef struct {
  void* param;         /* the weights, in/out */
  const void* grad;
  float* m;            /* running means of the gradient and of its square, in/out */
  float* v;
  void* copy;          /* bf16 weights that are written with the new param (fp32 master weights), or NULL */
  int64_t count;
  int32_t param_dtype; /* dit_dtype of param */
  int32_t grad_dtype;  /* dit_dtype of grad */
} dit_adamw_tensor;

typedef struct {
  double lr;            /* finite in fp32 */
  double beta1, beta2;  /* 0 <= beta < 1, also where it is rounded to fp32 (1 - 2^-25 is not): the means are fp32 numbers */
  double eps;           /* 0 or in the range of normal fp32 numbers */
  double weight_decay;  /* finite in fp32 */
  int64_t step;         /* t >= 1: this step's number (without step_dev) */
} dit_adamw_config;

/* With g' = *scale g (scale NULL: 1),
 *   m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2,
 *   param -= lr ( (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps) + weight_decay param ),
 * in fp32, rounded once to the types of param and copy. The betas count to 2^-24 of 1 - beta; each step rounds the means twice, by 2^-24 of
 * them at most, and squares below 2^-149 vanish in v. Nothing changes where *scale is NaN: a step whose gradients are not finite is left out.
 *   scale     device fp32 (grad_norm's), or NULL
 *   step_dev  device int64 holding t (a captured step, which the caller counts on the device), or NULL: cfg's. Nothing
 *             changes where it is below 1 */
dit_status adamw_step(const dit_adamw_config* cfg, const dit_adamw_tensor* tensors, int32_t n, const float* scale,
                      const int64_t* step_dev, dit_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* DITUPDATE_H */
