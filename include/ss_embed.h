/*
 * ss_embed.h -- C ABI of the embedding of token ids and of its gradient.
 *
 * What stands before the blocks of a language model of arXiv 2312.00752 (Section 4.2): a row of a table for every token.
 *
 *     out[t, :]    = scale * table[ids[t], :]                          0 where ids[t] is not in [0, vocab)
 *     dtable[v, :] = scale * sum over t with ids[t] = v of dout[t, :]  0 where there is none
 *
 * The sums are float32, their terms in an order that the sizes and ids alone decide, so the same call gives the same bits; they are rounded once.
 * Tokens whose id is outside the table have no gradient, whatever their dout holds.
 *
 * Rules as in ss_scan.h (device pointers owned by the caller, dense row-major layouts, outputs overwritten, host-side validation before any device
 * call, SS_OK or a negative SS_ERR_* code, nothing allocated), but pointers need be aligned to their element only.  No output may overlap an input.
 * tokens == 0 is valid (dtable is then 0).  SS_ERR_UNSUPPORTED: tokens or vocab of 2^31 - 65536 and more, dim of more than 512 x 65535.
 *      ids            : (tokens)         int64, or int32 with SS_EMBED_IDS_32
 *      table, dtable  : (vocab, dim)     table_dtype
 *      out, dout      : (tokens, dim)    io_dtype
 */
#ifndef SS_EMBED_H
#define SS_EMBED_H

#include "ss_scan.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { SS_EMBED_IDS_32 = 1u };

typedef struct {
    int32_t tokens, vocab, dim;
    int32_t table_dtype, io_dtype;   /* ss_dtype each                                       */
    uint32_t flags;                  /* 0 or SS_EMBED_IDS_32                                */
    float scale;
    const void *ids;
    const void *table;
    void *out;
} ss_embed_params;

int ss_embed_fwd(const ss_embed_params *p, void *stream);

typedef struct {
    ss_embed_params fwd;             /* the forward call's; table and out are not read      */
    const void *dout;
    void *dtable;
    void *workspace;                 /* ss_embed_workspace_bytes(), 256-byte aligned        */
    size_t workspace_bytes;
} ss_embed_bwd_params;

/* Bytes of scratch of the backward call (sorted ids, sums of pieces); tokens, vocab and dim are read. */
size_t ss_embed_workspace_bytes(const ss_embed_params *p);

/* Gradient of <out, dout> with respect to the table.  Deterministic. */
int ss_embed_bwd(const ss_embed_bwd_params *p, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SS_EMBED_H */
