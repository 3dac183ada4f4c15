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


# ---- log probabilities of tokens --------------------------------------------------------------------
def logprob_fwd(logits, targets=None, top=0):
    """logits (rows, vocab), targets (rows) or None.  Returns a dict with logp, entropy, max, total (sum of exp(x - max)), p, top_logp, top_ids, and
    sizes that float32 errors are relative to: logp_size, entropy_size, top_size."""
    x = np.asarray(logits, f64)
    rows, vocab = x.shape
    r = {k: np.zeros(rows) for k in ("logp", "entropy", "max", "total", "logp_size", "entropy_size")}
    r["p"], r["d"] = np.zeros((rows, vocab)), np.zeros((rows, vocab))
    r["top_logp"], r["top_size"], r["top_ids"] = np.zeros((rows, top)), np.zeros((rows, top)), np.zeros((rows, top), np.int64)
    for k in range(rows):
        t = -1 if targets is None else int(targets[k])
        asked = 0 <= t < vocab
        v = x[k]
        real = np.where(np.isnan(v), -np.inf, v)
        order = np.lexsort((np.arange(vocab), -real, np.isnan(v)))[:top]   # numbers first, then by value, then by column
        r["top_ids"][k] = np.where(np.isnan(v[order]), -1, order)
        if np.isnan(v).any() or (v == np.inf).any():
            for name in ("entropy", "max", "total"):
                r[name][k] = np.nan
            r["logp"][k] = np.nan if asked else 0.0
            r["top_logp"][k] = r["p"][k] = np.nan
            continue
        if (v == -np.inf).all():
            r["logp"][k] = -np.inf if asked else 0.0
            r["top_logp"][k] = -np.inf
            continue
        m = v.max()
        d = v - m
        e = np.exp(d)
        total = e.sum()
        d = np.where(e == 0, 0.0, d)
        p = e / total
        ls = np.log(total)
        r["max"][k], r["total"][k], r["p"][k], r["d"][k] = m, total, p, d
        r["entropy"][k] = ls - (p * d).sum()
        r["entropy_size"][k] = 1 + ls + (p * (d * d - d)).sum()
        if asked:
            r["logp"][k] = v[t] - m - ls
            r["logp_size"][k] = 1 + ls + (0.0 if np.isinf(v[t]) else m - v[t])
        r["top_logp"][k] = v[order] - m - ls
        r["top_size"][k] = 1 + ls + np.where(np.isinf(v[order]), 0.0, m - v[order])
    return r


def logprob_bwd(f, targets=None, dlogp=None, dentropy=None):
    """Gradient of the logits from ``f``, the forward pass's dict; and the sizes of its terms."""
    rows, vocab = f["p"].shape
    grad, size = np.zeros((rows, vocab)), np.zeros((rows, vocab))
    for k in range(rows):
        t = -1 if targets is None else int(targets[k])
        asked = 0 <= t < vocab
        dl = 0.0 if dlogp is None or not asked else float(dlogp[k])
        dh = 0.0 if dentropy is None else float(dentropy[k])
        if f["total"][k] == 0.0 or (dl == 0.0 and dh == 0.0):
            continue
        p, d = f["p"][k], f["d"][k]
        logp = d - np.log(f["total"][k])
        grad[k] = -p * (dl + dh * (logp + f["entropy"][k]))
        size[k] = p * (1 - d) * (abs(dl) + abs(dh) * (f["entropy_size"][k] + np.abs(logp)))
        if asked:
            grad[k, t] += dl
            size[k, t] += abs(dl)
    return {"dlogits": grad, "dlogits_size": size}


# ---- AdamW ------------------------------------------------------------------------------------------
def adamw(param, grad, m, v, step, lr, beta1, beta2, eps, weight_decay):
    """One step on float64 arrays, the moments' factors as float32 holds them.  Returns param, m, v, and what the error of the parameter's step is relative to:
    the step that the magnitudes of m's two terms, which may cancel, would make."""
    f32 = lambda b: f64(np.float32(b))
    size = f32(beta1) * np.abs(m) + f32(1 - beta1) * np.abs(grad)
    m = f32(beta1) * m + f32(1 - beta1) * grad
    v = f32(beta2) * v + f32(1 - beta2) * grad * grad
    rate = lr / (1 - beta1 ** step) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return param * (1 - lr * weight_decay) - rate * m, m, v, rate * size


ADAMW_BLOCK = 256


def adamw_codes(x, step, signed):
    """x (n), m or sqrt(v): (codes, scale) as the moments are held in 8 bits, in exact arithmetic."""
    x = np.asarray(x, f64)
    n, top = len(x), 127 if signed else 255
    c0, c1 = (0x6A09E667, 0xBB67AE85) if signed else (0x3C6EF372, 0xA54FF53A)
    codes, scale = np.zeros(n, np.int64), np.zeros(-(-n // ADAMW_BLOCK))
    for b in range(len(scale)):
        at = slice(b * ADAMW_BLOCK, min(n, (b + 1) * ADAMW_BLOCK))
        a = np.abs(x[at]).max()
        if not np.isfinite(a):
            scale[b] = np.nan
            continue
        if a < 2.0 ** -100:
            continue
        scale[b] = a
        y = top * top * np.abs(x[at]) / a
        q = np.floor(np.sqrt(y))
        u = np.array([((i * c0 + step * c1) % 2 ** 32 >> 8) / 2.0 ** 24 for i in range(at.start, at.stop)])
        q = np.minimum(q + ((y - q * q) / (2 * q + 1) > u), top)
        codes[at] = np.where(x[at] < 0, -q, q) if signed else np.where(x[at] > 0, np.maximum(q, 1), 0)
    return codes, scale


def adamw_values(codes, scale, signed):
    codes = np.asarray(codes, f64)
    top = 127 if signed else 255
    return np.sign(codes) * (codes / top) ** 2 * np.repeat(np.asarray(scale, f64), ADAMW_BLOCK)[: len(codes)]
