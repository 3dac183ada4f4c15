/*
 * ss_gate.h -- C ABI of the gated linear recurrence.
 *
 * Theorem 1 of arXiv 2312.00752 (Section 3.5.1) shows what the selective scan is for one state: a
 * recurrence h <- (1 - g) h + g x whose gate comes from the input.  Here the gate is an
 * operator of its own: a decay that is a power of a learned rate, an input gate that need not be
 * tied to it, and a normalisation that keeps the state's variance.  For every batch b and channel d:
 *
 *     s_t   = sigmoid(f[b,d,t] (+ f_bias[d]))
 *     a_t   = exp(-rate[d] * s_t)                     rate >= 0
 *     m_t   = sqrt(1 - a_t^2)
 *     g_t   = sigmoid(i[b,d,t] (+ i_bias[d]))         1 without SS_GATE_HAS_I
 *     h_t   = a_t h_{t-1} + m_t g_t x[b,d,t]
 *     out_t = h_t * z_t * sigmoid(z_t) if SS_GATE_HAS_Z, else h_t      (Section 3.4 gate)
 *
 * with h_{-1} = h0[b,d] (SS_GATE_HAS_H0) or 0, and h_last = h_{L-1} (whose memory may be that of h0, and dh0's that of
 * dh_last: a state that is carried on in place).  With SS_GATE_HAS_RESET, where
 * reset[b,t] is not 0, a_t = 0 and m_t = 1: a sequence begins at t (documents packed into one
 * row; the boundary resetting of Section 3.5.2), and nothing of what stands before t, an infinity
 * or NaN included, reaches t or anything behind it, forward or backward.
 *
 * Rules as in ss_scan.h (device pointers owned by the caller, outputs overwritten, host-side
 * validation before any device call, SS_OK or a negative SS_ERR_* code, nothing allocated), with
 * these differences: the io tensors may be slices of wider ones -- the distance between batch
 * entries is given in elements, a batch entry itself is dense (D, L) -- and io pointers need be
 * aligned to their element only.
 *      x, f, i, z, dx, df, di, dz : (B, D, L)  io_dtype, batch stride as given (>= D L)
 *      out, dout                  : (B, D, L)  io_dtype, dense
 *      rate, f_bias, i_bias and their gradients : (D)     float32
 *      reset                      : (B, L)     uint8
 *      h0, h_last, dh_last, dh0   : (B, D)     float32
 * Rows (B D) are limited by the threads of a launch: fewer than 2^26 of more than 128 steps, 2^28 of more
 * than 32, 2^30 else; more, and rows of 2^31 - 2048 steps and more, are SS_ERR_UNSUPPORTED.
 * seqlen == 0 is valid: h_last receives h0 or 0, and the backward call returns zero parameter
 * gradients and dh0 = dh_last.
 */
#ifndef SS_GATE_H
#define SS_GATE_H

#include "ss_scan.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    SS_GATE_HAS_I        = 1u,  /* i is given                                               */
    SS_GATE_HAS_Z        = 2u,  /* z is given                                               */
    SS_GATE_HAS_F_BIAS   = 4u,
    SS_GATE_HAS_I_BIAS   = 8u,  /* only together with SS_GATE_HAS_I                         */
    SS_GATE_HAS_RESET    = 16u,
    SS_GATE_HAS_H0       = 32u,
    SS_GATE_WRITE_H_LAST = 64u,
    SS_GATE_SAVE_FOR_BWD = 128u /* leave state checkpoints in `workspace`                   */
};

typedef struct {
    int32_t batch, dim, seqlen;                 /* B, D, L                                  */
    int32_t io_dtype;                           /* ss_dtype                                 */
    uint32_t flags;                             /* OR of SS_GATE_* bits                     */
    const void *x, *f, *i, *z;
    int64_t x_batch, f_batch, i_batch, z_batch; /* elements between batch entries           */
    const float *rate, *f_bias, *i_bias;
    const uint8_t *reset;
    const float *h0;
    void *out;
    float *h_last;
    void *workspace;                            /* 256-byte aligned                         */
    size_t workspace_bytes;
} ss_gate_params;

/* Bytes of workspace: for_backward == 0 what lets a plain forward call split long sequences of few
 * rows across workgroups (optional: without it the call is correct and one wave walks each
 * row); 1 what a forward call with SS_GATE_SAVE_FOR_BWD and its backward call need (the backward call gets the same,
 * untouched buffer).  Only batch, dim and seqlen are read. */
size_t ss_gate_workspace_bytes(const ss_gate_params *p, int for_backward);

int ss_gate_fwd(const ss_gate_params *p, void *stream);

typedef struct {
    ss_gate_params fwd;       /* the forward call's inputs, flags and filled workspace; out and h_last are not read */
    const void *dout;
    const float *dh_last;     /* or NULL                                                    */
    void *dx, *df, *di, *dz;  /* di, dz iff SS_GATE_HAS_I / SS_GATE_HAS_Z                   */
    int64_t dx_batch, df_batch, di_batch, dz_batch;
    float *drate, *df_bias, *di_bias; /* biases iff SS_GATE_HAS_F_BIAS / SS_GATE_HAS_I_BIAS */
    float *dh0;               /* or NULL                                                    */
} ss_gate_bwd_params;

/* Gradient of <out, dout> + <h_last, dh_last>.  The states are recomputed from the checkpoints.
 * Where m_t is 0 (rate or s_t is 0) its derivative, which has no finite value, counts as 0.  m_t counts as 0,
 * forward and backward, where 1 - a_t^2 is below the least normal number, 2^-126.
 * Deterministic. */
int ss_gate_bwd(const ss_gate_bwd_params *p, void *stream);

typedef struct {
    int32_t batch, dim;
    int32_t io_dtype;
    uint32_t flags;                 /* SS_GATE_HAS_I, _Z, _F_BIAS, _I_BIAS, _RESET           */
    float *h;                       /* (B,D), updated IN PLACE                              */
    const void *x_t, *f_t, *i_t, *z_t;          /* (B,D), rows of a batch entry dense       */
    int64_t x_batch, f_batch, i_batch, z_batch;
    const float *rate, *f_bias, *i_bias;
    const uint8_t *reset_t;         /* (B)                                                  */
    void *out_t;                    /* (B,D) dense                                          */
} ss_gate_step_params;

/* One token. */
int ss_gate_step(const ss_gate_step_params *p, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SS_GATE_H */
