/*
 * jacobi_adamw.h -- C ABI of the optimiser step of libjacobi_made.so: AdamW (bias-corrected moments, decoupled weight
 * decay) over many tensors in one call, for the gradients that rnn_param_grads (jacobi_rnn.h), linattn_backward
 * (jacobi_linattn.h) and the caller's own layers give.
 *
 *     m <- beta1 m + (1 - beta1) g,     v <- beta2 v + (1 - beta2) g^2,      g = grad_scale * gradient
 *     p <- p (1 - lr weight_decay) - lr c1 m / (sqrt(c2 v) + eps),           c1 = 1 / (1 - beta1^step), c2 = 1 / (1 - beta2^step)
 *
 * Moments in 8 bits (moment_bits = 8): ADAMW_BLOCK consecutive elements of a tensor share a scale, the block's largest
 * absolute moment rounded to fp32.  m is int8, one of scale * c |c| / 127^2 with c = -127..127; v is uint8, one of
 * scale * (c / 255)^4, c = 0..255: finer steps near zero, where most moments of a block lie.  A moment takes the code with
 * the nearest root (halves up), a second moment that is not zero never code 0, so that a step is not divided by eps alone.  All
 * zero bytes and scales are moments of zero.  m and v are computed in 64 bits from their codes and rounded once, to codes;
 * the step takes them as fp32 before that.  A block with a moment that is not finite has the scale NaN, and reads as NaN.
 * Moments in 32 bits are formed in fp32: the square of a g beyond 2^64 is infinite there, and its weight then only decays.
 *
 * Conventions (as in jacobi_rnn.h): the arrays of pointers and sizes are HOST memory, read during the call; what they
 * point to is DEVICE memory, contiguous, owned by the caller, and no two of the buffers written may overlap.  Calls are
 * enqueued on `stream` and return without waiting; they may be recorded into a graph (which keeps the pointers and, unless
 * they come from `scalars`, the numbers).  No call allocates memory.  The return value is MADE_OK or a negative
 * made_status (jacobi_made.h), made_last_error() has the message.
 */
#ifndef JACOBI_ADAMW_H
#define JACOBI_ADAMW_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { ADAMW_BLOCK = 256 };

typedef struct adamw_config {
  double lr, beta1, beta2, eps, weight_decay;   /* finite; 0 <= beta < 1; eps a normal fp32 number or 0 (NaN where v is 0) */
  double grad_scale;                            /* factor of the gradients (1, or a clipping or loss-scaling factor)  */
  int32_t step;                                 /* 1, 2, ...: steps taken including this one                          */
  int32_t param_dtype, grad_dtype;              /* MADE_F32 or MADE_BF16 (bf16 weights are rounded to nearest)         */
  int32_t moment_bits;                          /* 32 (fp32) or 8                                                     */
} adamw_config;

/*
 * adamw_step -- one step of n tensors.
 *   sizes   : elements of each tensor (0 allowed, at most 2^36 - 2^12);   params, grads, m, v: n device pointers each
 *   m_scale, v_scale: n device pointers to ceil(size / ADAMW_BLOCK) fp32 scales each (8-bit moments, else NULL)
 *   copies  : n device pointers to bf16 tensors that get the new weights rounded, or NULL; with fp32 weights only
 *   scalars : DEVICE double[4] {lr, c1, c2, grad_scale} read when the step runs, in place of cfg's lr, step and grad_scale
 *             (a recorded step then follows the schedule), or NULL
 */
int adamw_step(const adamw_config* cfg, int32_t n, const int64_t* sizes, void* const* params, const void* const* grads,
               void* const* m, void* const* v, float* const* m_scale, float* const* v_scale, void* const* copies,
               const double* scalars, void* stream);

/*
 * adamw_unpack -- the fp32 values that 8-bit moments stand for (to look at them, or to go on with 32-bit moments).
 */
int adamw_unpack(int32_t n, const int64_t* sizes, const void* const* m, const void* const* v, const float* const* m_scale,
                 const float* const* v_scale, float* const* m_out, float* const* v_out, void* stream);

#ifdef __cplusplus
}
#endif
#endif
