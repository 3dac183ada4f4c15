/*
 * ss_quant.h -- C ABI of products in 8-bit integers with a scale for each token and each output channel.
 *
 * The wide projections of the block of arXiv 2312.00752 (Section 3.4: 3 E D^2 of its parameters) at
 * serving time, with weights held in 8 bits and tokens brought to 8 bits as they come.  Rows (tokens, or
 * a weight's output channels) are quantised symmetrically:
 *
 *     scale = max_k |x_k| / 127,     q_k = round(x_k * (127 * (1 / max_k |x_k|)))    ties to even; float32 arithmetic
 *
 * and a product is summed exactly in 32-bit integers:
 *
 *     out[t, n] = (sum_k q[t,k] w[n,k]) * (scale_t * scale_n) (+ bias[n])
 *
 * A row whose largest magnitude is below 2^-120 counts as zero (scale 0); one that holds an infinity or
 * NaN has the scale NaN and comes out as NaN.
 *
 * Quantised rows lie ss_quant_pitch(dim) bytes apart (dim rounded up to 128), the bytes behind dim
 * being 0.  Rules as in ss_scan.h (device pointers owned by the caller, outputs overwritten, host-side
 * validation before any device call, SS_OK or a negative SS_ERR_* code, nothing allocated), but io
 * pointers need be aligned to their element only.  1 <= dim <= SS_QUANT_MAX_DIM; batch or seqlen 0 is valid.
 * SS_ERR_UNSUPPORTED: batch seqlen or features of 2^31 - 65536 and more; more than 65535 batch entries where a
 * sequence axis comes last; results of 2^31 and more tiles of 64 x 64.
 *      x                : (batch, seqlen, dim)  io_dtype;  (batch, dim, seqlen) with SS_Q_X_SEQ_LAST;
 *                         with SS_Q_X_QUANTISED (batch seqlen, pitch) int8, 16-byte aligned
 *      q, x_scale       : (batch seqlen, pitch) int8, 16-byte aligned; (batch seqlen) float32
 *      weight, scale    : (features, pitch) int8, 16-byte aligned; (features) float32
 *      bias             : (features) float32
 *      out              : (batch, seqlen, features) io_dtype; (batch, features, seqlen) with SS_Q_OUT_SEQ_LAST
 */
#ifndef SS_QUANT_H
#define SS_QUANT_H

#include "ss_scan.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SS_QUANT_MAX_DIM 131072 /* 127^2 times as many stay below 2^31 */

enum {
    SS_Q_X_SEQ_LAST   = 1u,
    SS_Q_OUT_SEQ_LAST = 2u,
    SS_Q_HAS_BIAS     = 4u,
    SS_Q_X_QUANTISED  = 8u  /* x and x_scale come from ss_quant_rows; not together with SS_Q_X_SEQ_LAST */
};

/* Bytes from one quantised row to the next; 0 for dim < 1. */
size_t ss_quant_pitch(int32_t dim);

typedef struct {
    int32_t batch, seqlen, dim;
    int32_t io_dtype;            /* ss_dtype of x                                           */
    uint32_t flags;              /* 0 or SS_Q_X_SEQ_LAST                                    */
    const void *x;
    void *q;
    float *scale;
    void *scratch;               /* ss_quant_rows_scratch_bytes(), 256-byte aligned; may be NULL where that is 0 */
    size_t scratch_bytes;
} ss_quant_params;

size_t ss_quant_rows_scratch_bytes(const ss_quant_params *p);
int ss_quant_rows(const ss_quant_params *p, void *stream);

typedef struct {
    int32_t batch, seqlen, dim, features;
    int32_t io_dtype;            /* ss_dtype of x and out                                   */
    uint32_t flags;              /* OR of SS_Q_* bits                                       */
    const void *x;
    const float *x_scale;        /* with SS_Q_X_QUANTISED                                   */
    const void *weight;
    const float *scale, *bias;
    void *out;
    void *scratch;               /* ss_qlinear_scratch_bytes(), 256-byte aligned            */
    size_t scratch_bytes;
} ss_qlinear_params;

size_t ss_qlinear_scratch_bytes(const ss_qlinear_params *p);

/* Tokens brought to 8 bits (but with SS_Q_X_QUANTISED), times the weight.  Deterministic. */
int ss_qlinear(const ss_qlinear_params *p, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SS_QUANT_H */
