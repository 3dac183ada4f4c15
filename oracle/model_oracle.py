"""Float64 oracles of root-mean-square norm, embedding, log probabilities of tokens and AdamW, written from the definitions in
include/ss_norm.h, ss_embed.h, ss_logprob.h and ss_adamw.h: plain numpy.

Sums over many terms are returned with the sum of the terms' magnitudes under ``name + "_size"``, which is what a float32
sum's error is relative to.
"""
import numpy as np

f64 = np.float64


# ---- RMS norm -------------------------------------------------------------------------------------
def rms_fwd(s, weight=None, bias=None, eps=1e-5):
    """s (rows, width), as held.  Returns out, xhat, rstd."""
    s = np.asarray(s, f64)
    rstd = 1.0 / np.sqrt((s ** 2).mean(1, keepdims=True) + eps)
    xhat = s * rstd
    out = xhat * (1.0 if weight is None else np.asarray(weight, f64)) + (0.0 if bias is None else np.asarray(bias, f64))
    return out, xhat, rstd


def rms_bwd(dout, s, weight=None, dsummed=None, eps=1e-5):
    dout = np.asarray(dout, f64)
    _, xhat, rstd = rms_fwd(s, eps=eps)
    g = dout * (1.0 if weight is None else np.asarray(weight, f64))
    ds = rstd * (g - xhat * (g * xhat).mean(1, keepdims=True))
    if dsummed is not None:
        ds = ds + np.asarray(dsummed, f64)
    return {"ds": ds, "dweight": (dout * xhat).sum(0), "dweight_size": np.abs(dout * xhat).sum(0),
            "dbias": dout.sum(0), "dbias_size": np.abs(dout).sum(0)}


# ---- embedding ------------------------------------------------------------------------------------
def embed_fwd(ids, table, scale=1.0):
    """ids of any shape, table (vocab, dim)."""
    table = np.asarray(table, f64)
    out = np.zeros(np.shape(ids) + table.shape[1:])
    for k in np.ndindex(*np.shape(ids)):
        if 0 <= ids[k] < len(table):
            out[k] = scale * table[ids[k]]
    return out


def embed_bwd(dout, ids, vocab, scale=1.0):
    grad, size = np.zeros((vocab, dout.shape[-1])), np.zeros((vocab, dout.shape[-1]))
    for k in np.ndindex(*np.shape(ids)):
        if 0 <= ids[k] < vocab:
            grad[ids[k]] += scale * np.asarray(dout[k], f64)
            size[ids[k]] += np.abs(scale * np.asarray(dout[k], f64))
    return {"dtable": grad, "dtable_size": size}
