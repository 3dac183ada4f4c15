/*
 * ss_norm.h -- C ABI of layer norm and root-mean-square norm with the residual sum that stands before them.
 *
 * The block of arXiv 2312.00752 (Section 3.4, Figure 3) is interleaved with residual connections and an
 * optional normalisation layer.  A call takes both steps for `rows` tokens of `width` channels:
 *
 *     s    = x + residual             (x without SS_NORM_HAS_RESIDUAL), held in the residual's type
 *     out  = (s - mean) / sqrt(var + eps) * weight + bias       mean, var over the width, of s as held
 *     out  = s / sqrt(mean(s^2) + eps) * weight + bias          with SS_NORM_RMS
 *
 * Rules as in ss_scan.h (device pointers owned by the caller, dense row-major layouts, outputs
 * overwritten, host-side validation before any device call, SS_OK or a negative SS_ERR_* code, nothing
 * allocated), but io pointers need be aligned to their element only.  Statistics and sums are float32
 * whatever io_dtype is.  rows == 0 is valid.
 *      x, out, dout, dx                       : (rows, width)  io_dtype
 *      residual, summed, dsummed, dresidual   : (rows, width)  io_dtype, or float32 with SS_NORM_RESIDUAL_F32
 *      weight, bias, dweight, dbias           : (width)        float32
 *      stats                                  : (2, rows)      float32: means, then 1 / sqrt(var + eps);
 *                                               (rows) with SS_NORM_RMS: 1 / sqrt(mean(s^2) + eps)
 */
#ifndef SS_NORM_H
#define SS_NORM_H

#include "ss_scan.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    SS_NORM_HAS_WEIGHT   = 1u, /* weight is given (else 1)                                  */
    SS_NORM_HAS_BIAS     = 2u, /* bias is given (else 0)                                    */
    SS_NORM_HAS_RESIDUAL = 4u, /* residual and summed are given                             */
    SS_NORM_RESIDUAL_F32 = 8u, /* they are float32 whatever io_dtype is                     */
    SS_NORM_SAVE_STATS   = 16u,/* stats is written                                          */
    SS_NORM_RMS          = 64u /* no mean is taken off                                      */
};

typedef struct {
    int32_t rows, width;
    int32_t io_dtype;          /* ss_dtype                                                  */
    uint32_t flags;            /* OR of SS_NORM_* bits                                      */
    float eps;                 /* >= 0, finite                                              */
    const void *x, *residual;
    const float *weight, *bias;
    void *out;
    void *summed;              /* may be `residual` itself: the stream is updated in place  */
    float *stats;
} ss_norm_params;

int ss_norm_fwd(const ss_norm_params *p, void *stream);

typedef struct {
    ss_norm_params fwd;        /* as for ss_norm_fwd, without SS_NORM_SAVE_STATS; out is not written */
    int8_t *q;                 /* (rows, ss_quant_pitch(width)), 16-byte aligned; bytes behind width are 0 */
    float *scale;              /* (rows) */
} ss_norm_quant_params;

/* The forward pass with its result in 8 bits (ss_quant.h), as ss_qlinear takes it: what ss_quant_rows makes of ss_norm_fwd's out, to the
 * bit, of which nothing is stored.  width <= SS_QUANT_MAX_DIM. */
int ss_norm_quant(const ss_norm_quant_params *p, void *stream);

typedef struct {
    ss_norm_params fwd;        /* the forward call's sizes, flags, eps and weight; what was normalised (summed, or x
                                  without a residual) and stats are read, the rest is not   */
    const void *dout;
    const void *dsummed;       /* gradient that reaches s from behind, in s's type; or NULL */
    void *dx;                  /* gradient of x, and of a residual in io_dtype              */
    void *dresidual;           /* the same in float32: iff SS_NORM_HAS_RESIDUAL and SS_NORM_RESIDUAL_F32 and io_dtype is not float32 */
    float *dweight, *dbias;    /* iff SS_NORM_HAS_WEIGHT / SS_NORM_HAS_BIAS                 */
    void *workspace;           /* ss_norm_workspace_bytes(), 256-byte aligned               */
    size_t workspace_bytes;
} ss_norm_bwd_params;

/* Bytes of scratch of the backward call (partial sums of the weights' gradients); rows and width are read. */
size_t ss_norm_workspace_bytes(const ss_norm_params *p);

/* Gradient of <out, dout> + <s, dsummed>.  Deterministic. */
int ss_norm_bwd(const ss_norm_bwd_params *p, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SS_NORM_H */
