/*
 * ss_logprob.h -- C ABI of the log probabilities of given tokens, with the entropy and the most probable alternatives, and of their gradient.
 *
 * What stands behind the blocks of a language model of arXiv 2312.00752 (Section 4.2): its loss in training, and what is said about
 * a token in generation.  For every row x of `vocab` logits and its target t:
 *
 *     lse      = log sum_j exp(x_j)
 *     logp     = x_t - lse                        0 where t is not in [0, vocab): no token is asked for
 *     entropy  = lse - sum_j p_j x_j              p_j = exp(x_j - lse), and p_j x_j = 0 where p_j is
 *     top_ids  : the `top` columns with the largest logits, the largest first, of equal ones the lowest first
 *     top_logp = x at them - lse
 *     dlogits_j = dlogp ([j = t] - p_j) - dentropy p_j (log p_j + entropy)
 *
 * Logits of -infinity have probability 0 and the gradient 0 (dlogp, if they are the target); exp(x_j - max) below 2^-126 counts as 0.  A row of
 * nothing else has no distribution: the log probabilities in it are -infinity, its entropy and its gradients are 0.  A row that holds +infinity or
 * NaN has the results NaN (top_ids: the columns that are not NaN in the same order, -1 where there are no more).  Without a target (t outside) dlogp
 * is not read into the row's gradient; a row whose dlogp is 0 or not asked for, and whose dentropy is 0 or not given, has the gradient 0 whatever it
 * holds.
 *
 * What is asked for beside them does not change the bits of logp, entropy and stats.
 *
 * Rules as in ss_scan.h (device pointers owned by the caller, outputs overwritten, host-side validation before any device
 * call, SS_OK or a negative SS_ERR_* code, nothing allocated), but pointers need be aligned to their element only.  Sums
 * are float32 whatever io_dtype is.  rows == 0 is valid.  SS_ERR_UNSUPPORTED: rows ceil(vocab / 8192) of 2^24 and more (of 2^26 up to
 * 2048 columns), vocab of 2^31 - 65536 and more.
 *      logits                         : (rows, vocab)  io_dtype, rows `row_stride` elements apart (>= vocab)
 *      dlogits                        : (rows, vocab)  io_dtype, dense; not the logits' own memory
 *      targets                        : (rows)         int64, or int32 with SS_LOGPROB_TARGETS_32; NULL: no row has one
 *      logp, entropy, dlogp, dentropy : (rows)         float32
 *      stats                          : (2, rows)      float32: the largest logit, 1 / sum_j exp(x_j - it) (0, 0 without a distribution)
 *      top_logp, top_ids              : (rows, top)    float32, int64
 */
#ifndef SS_LOGPROB_H
#define SS_LOGPROB_H

#include "ss_scan.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SS_LOGPROB_MAX_TOP 64

enum { SS_LOGPROB_TARGETS_32 = 1u };

typedef struct {
    int32_t rows, vocab, top;        /* 0 <= top <= min(vocab, SS_LOGPROB_MAX_TOP)          */
    int32_t io_dtype;                /* ss_dtype                                            */
    uint32_t flags;                  /* 0 or SS_LOGPROB_TARGETS_32                          */
    int64_t row_stride;
    const void *logits;
    const void *targets;
    float *logp;                     /* may be NULL without targets                         */
    float *entropy;
    float *stats;
    float *top_logp;                 /* iff top > 0                                         */
    int64_t *top_ids;
    void *workspace;                 /* ss_logprob_workspace_bytes(), 256-byte aligned; may be NULL where that is 0 */
    size_t workspace_bytes;
} ss_logprob_params;

/* Bytes of scratch of the forward call (rows that several workgroups share); rows, vocab and top are read. */
size_t ss_logprob_workspace_bytes(const ss_logprob_params *p);

int ss_logprob_fwd(const ss_logprob_params *p, void *stream);

typedef struct {
    ss_logprob_params fwd;           /* the forward call's sizes, logits and targets; entropy (with dentropy) and stats are read, the rest is not */
    const float *dlogp;              /* or NULL: 0 */
    const float *dentropy;           /* or NULL: 0 */
    void *dlogits;
} ss_logprob_bwd_params;

/* Gradient of <logp, dlogp> + <entropy, dentropy>.  Deterministic. */
int ss_logprob_bwd(const ss_logprob_bwd_params *p, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SS_LOGPROB_H */
