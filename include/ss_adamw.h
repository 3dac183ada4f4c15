/*
 * ss_adamw.h -- C ABI of a step of AdamW over many tensors at once, with moments in float32 or in 8 bits.
 *
 * The optimiser of the training recipes of arXiv 2312.00752 (Appendix E.2: AdamW, decoupled weight decay).  For every element of every
 * tensor, in step t = count[0] + 1:
 *
 *     g      = grad (* grad_scale)
 *     m      = beta1 m + (1 - beta1) g
 *     v      = beta2 v + (1 - beta2) g^2
 *     param  = param (1 - lr weight_decay) - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 *
 * in float32.  A bfloat16 param may have a float32 `master`, which is then what is updated, and param its rounding; without one the sum is
 * rounded to param.  The call counts the step itself, in device memory, so a captured call that is replayed takes further steps.
 *
 * state_bits 8: m and sqrt(v) are held in blocks of SS_ADAMW_BLOCK elements (the last of a tensor may be shorter) by a scale a, their
 * largest magnitude, and codes q of 8 bits:
 *
 *     m       = sign(q) (q / 127)^2 a          int8
 *     sqrt(v) = (q / 255)^2 a                  uint8
 *
 * whose steps grow with the value, as the error that a moment tolerates does.  Between two codes the upper one is taken when
 *     (y - q^2) / (2 q + 1) > u,    y = |m| (127^2 (1 / a))   (sqrt(v) (255^2 (1 / a))),  q = floor(sqrt(y)),
 *     u = ((i c0 + t c1) mod 2^32) / 2^32 cut to 24 bits
 * for element i of its tensor: over the steps, u goes evenly through [0, 1) (a Weyl sequence: c0 and c1 are the fractional parts of sqrt(2) and
 * sqrt(3), for v of sqrt(5) and sqrt(7), in units of 2^-32), so a rounding is right in the mean, of values too that move by less than a code's distance;
 * rounded to the nearest, v would not move at all at beta2 = 0.999.  m stays right in the mean over any number of steps.  v, the square of what is rounded, gathers the
 * rounding's variance: with normal gradients and beta2 = 0.999 it comes to be too large by about 1 / q, that is by 0.9, 4, 12 and 58 % for elements at 1/10, 1/100, 1/1000 and
 * 1/10000 of their block's largest, sqrt(v) by 0.2, 0.9, 2.5 and 13 %, by which their steps are shorter.  sqrt(v) > 0 has a code of 1 at least, so a parameter's step stays bounded.  The
 * parameter's step takes the moments as they are before they are rounded.  A block whose largest magnitude is below 2^-100 counts as zero (scale 0);
 * one that holds an infinity or NaN has the scale NaN and comes out as NaN.
 *
 * Rules as in ss_scan.h (device pointers owned by the caller, host-side validation before any device call, SS_OK or a
 * negative SS_ERR_* code, nothing allocated), but pointers need be aligned to their element only.  The list and the tensors' descriptions are
 * host memory and read before the call returns.  Tensors must not overlap.  Zero tensors, and tensors of no elements, are valid: the step is
 * counted.
 */
#ifndef SS_ADAMW_H
#define SS_ADAMW_H

#include "ss_scan.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SS_ADAMW_BLOCK 256

typedef struct {
    int64_t n;                       /* elements                                            */
    int32_t param_dtype, grad_dtype; /* ss_dtype each                                       */
    void *param;                     /* written; read where there is no master              */
    const void *grad;
    float *master;                   /* or NULL; only with a bfloat16 param                 */
    void *m, *v;                     /* float32, or int8 and uint8                          */
    float *m_scale, *v_scale;        /* (ceil(n / SS_ADAMW_BLOCK)) with state_bits 8        */
} ss_adamw_tensor;

typedef struct {
    int32_t tensors;
    int32_t state_bits;              /* 32 or 8                                             */
    const ss_adamw_tensor *list;
    int32_t *count;                  /* (2), device: steps taken; 0, the call's own while it runs */
    double lr, beta1, beta2;         /* 0 <= beta < 1                                       */
    double eps, weight_decay;        /* >= 0, finite in float32; eps 0, or 2^-126 and more  */
    const float *lr_device;          /* or NULL; else lr is read there (lr is not)          */
    const float *grad_scale;         /* or NULL: 1                                          */
} ss_adamw_params;

/* Deterministic.  Calls with the same count must not run at once. */
int ss_adamw_step(const ss_adamw_params *p, void *stream);

typedef struct {
    int64_t n;
    int32_t with_sign;               /* 1: codes of m; 0: of v                              */
    int32_t out_dtype;               /* ss_dtype                                            */
    const void *codes;
    const float *scale;
    void *out;                       /* (n): m, or sqrt(v)                                  */
} ss_adamw_values_params;

/* What a moment's 8-bit codes stand for. */
int ss_adamw_values(const ss_adamw_values_params *p, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SS_ADAMW_H */
