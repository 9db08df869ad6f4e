/*
 * cocod_adamw.h -- AdamW over many tensors at once (part of libcocod.so), beside the engine's momentum SGD.
 *
 * Step t of a tensor with parameters p, gradient g (times *grad_scale where that is given), moments m and v:
 *     m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
 *     p = p (1 - lr decay) - lr m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps).
 * All tensors are updated by one launch (by one for every 1024 of them where they are given one by one).  t is the number of the handle's steps, also for a tensor
 * that had no gradient in some of them: its moments stay as they were, their correction goes on.  The number of steps, the powers of the betas and lr live on the device, so that a step captured into a CUDA graph counts its replays and follows cocod_adamw_set_lr.
 *
 * State.  The moments lie in the caller's memory, tensors one behind the other, each starting at a multiple of 128 values; L = the sum
 * of the sizes, each rounded up to 128 (cocod_adamw_values).  What lies behind a tensor's values stays 0.
 *   COCOD_ADAMW_32   m, v: L fp32 each
 *   COCOD_ADAMW_8    m: L int8 c, v: L uint8 d, m_units, v_units: L / 128 fp32 each, one for a block of 128 values:
 *                        m = c |c| m_unit,   sqrt v = d^2 v_unit,   m_unit = max |m| / 127^2,   v_unit = max sqrt v / 255^2
 *     c and d are the nearest whole numbers (half to even), d at least 1 where v > 0, so that a step never divides by a root that was
 *     rounded to 0.  A block whose largest value is below 2^-100 reads as 0, one that met a value that is not finite as NaN.  Between the old
 *     moments and the new ones every product, sum, root and quotient is rounded to fp32 once, in the order of the formulas above.
 * All zero bytes are the state before the first step.
 *
 * Conventions are cocod.h's: int return codes, device pointers on the device current at create, asynchronous on the given stream, one host
 * thread per handle, and the steps of one handle in order.
 */
#ifndef COCOD_ADAMW_H
#define COCOD_ADAMW_H

#include <stdint.h>

#include "cocod.h"
#include "cocod_lm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cocod_adamw cocod_adamw_handle;

enum { COCOD_ADAMW_8 = 8, COCOD_ADAMW_32 = 32 };
#define COCOD_ADAMW_MAX_TENSORS (1 << 20)

/* L, or COCOD_ERR_INVALID (n < 1, a size < 1, or L >= 2^40). */
int64_t cocod_adamw_values(int n, const int64_t *sizes);

/* sizes, decay (NULL: 0), starts: host, n values; the arrays are copied.  starts: where the tensors lie in one flat buffer (cocod_adamw_flat_step,
 * cocod_adamw_local_step), or NULL if every step gives their addresses (cocod_adamw_step).  Allocates its tables (about 40 bytes a tensor and 4 for each
 * chunk of 1024 to 16384 values, at least one a tensor).  m_units, v_units: NULL with 32 bits.  The state is not touched.  Errors: INVALID (0 <= beta < 1, eps >= 0, lr and decay finite), OOM, CUDA. */
int cocod_adamw_create(cocod_adamw_handle **out, int n, const int64_t *sizes, const float *decay, const int64_t *starts, int state_bits, void *m, void *v,
                       float *m_units, float *v_units, float lr, double beta1, double beta2, float eps);
int cocod_adamw_destroy(cocod_adamw_handle *h);
/* The n sizes given at creation (the handle's memory), or NULL without a handle. */
const int64_t *cocod_adamw_sizes(const cocod_adamw_handle *h, int *n);

/* One step.  params, grads, copies: host arrays of n device addresses (the arrays are read before the call returns), tensor i of sizes[i] values; a tensor whose
 * gradient is NULL keeps its parameters and moments.  copies (or NULL): bf16 copies of fp32 parameters, written with them; single ones may be NULL.
 * param_type, grad_type: COCOD_BF16 or COCOD_F32; any alignment of whole values (16 bytes are faster).  bf16 parameters are rounded to nearest.
 * grad_scale: device, one fp32 value, or NULL. */
int cocod_adamw_step(cocod_adamw_handle *h, void *const *params, int param_type, const void *const *grads, int grad_type, void *const *copies,
                     const float *grad_scale, cocod_stream_t stream);

/* The same for tensors in flat buffers: tensor i at params + starts[i] and so on.  params_out may be params_in; copies: bf16 or NULL. */
int cocod_adamw_flat_step(cocod_adamw_handle *h, const void *params_in, void *params_out, int param_type, const void *grads, int grad_type, void *copies,
                          const float *grad_scale, cocod_stream_t stream);

/* The local step of Algorithm 1 (Step II) for every worker of an engine with AdamW in place of momentum SGD: what cocod_local_step does to the
 * engine's models, its bf16 copy, its step count and its state of communication.  The tensors have to cover the K x P values one behind the other.
 * Runs on the engine's compute stream; both handles are of the same device.  grads: device, K x P fp32.  The engine's momentum, lr, mu and wd take no part. */
int cocod_adamw_local_step(cocod_adamw_handle *h, cocod_handle *engine, const float *grads, const float *grad_scale);

/* Ordered on the stream. */
int cocod_adamw_set_lr(cocod_adamw_handle *h, float lr, cocod_stream_t stream);
int cocod_adamw_set_step(cocod_adamw_handle *h, int64_t steps, cocod_stream_t stream);
/* Synchronises the stream. */
int cocod_adamw_get_step(cocod_adamw_handle *h, int64_t *steps, cocod_stream_t stream);

/* The moments in fp32, L values each in the state's order: read, or put in their place (with 8 bits: coded). */
int cocod_adamw_moments(cocod_adamw_handle *h, float *m, float *v, cocod_stream_t stream);
int cocod_adamw_load(cocod_adamw_handle *h, const float *m, const float *v, cocod_stream_t stream);

int64_t cocod_adamw_launch_count(const cocod_adamw_handle *h);

#ifdef __cplusplus
}
#endif
#endif /* COCOD_ADAMW_H */
