"""Float64 oracles of layer norm, the gated linear recurrence and products in 8-bit integers, written from the
definitions in include/ss_norm.h, ss_gate.h and ss_quant.h: plain numpy, one step after another.

Sums over many terms (weights' gradients) are returned with the sum of the terms' magnitudes under ``name + "_size"``, which
is what a float32 sum's error is relative to.
"""
import numpy as np

f64 = np.float64


def _sigmoid(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-v))


# ---- layer norm ---------------------------------------------------------------------------------
def norm_fwd(s, weight=None, bias=None, eps=1e-5):
    """s (rows, width), as held.  Returns out, xhat, rstd."""
    s = np.asarray(s, f64)
    mean = s.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((s - mean) ** 2).mean(1, keepdims=True) + eps)
    xhat = (s - mean) * rstd
    out = xhat * (1.0 if weight is None else np.asarray(weight, f64)) + (0.0 if bias is None else np.asarray(bias, f64))
    return out, xhat, rstd


def norm_bwd(dout, s, weight=None, dsummed=None, eps=1e-5):
    dout = np.asarray(dout, f64)
    _, xhat, rstd = norm_fwd(s, eps=eps)
    g = dout * (1.0 if weight is None else np.asarray(weight, f64))
    ds = rstd * (g - g.mean(1, keepdims=True) - xhat * (g * xhat).mean(1, keepdims=True))
    if dsummed is not None:
        ds = ds + np.asarray(dsummed, f64)
    return {"ds": ds, "dweight": (dout * xhat).sum(0), "dweight_size": np.abs(dout * xhat).sum(0),
            "dbias": dout.sum(0), "dbias_size": np.abs(dout).sum(0)}


# ---- gated linear recurrence ----------------------------------------------------------------------
def _gates(x, f, rate, i, f_bias, i_bias, reset):
    row = lambda v: 0.0 if v is None else np.asarray(v, f64)[None, :, None]
    s = _sigmoid(np.asarray(f, f64) + row(f_bias))
    la = -row(rate) * s
    a, m = np.exp(la), np.sqrt(-np.expm1(2.0 * la))
    g = np.ones_like(a) if i is None else _sigmoid(np.asarray(i, f64) + row(i_bias))
    mark = np.zeros(a.shape, bool) if reset is None else np.broadcast_to(np.asarray(reset, bool)[:, None, :], a.shape)
    return s, la, np.where(mark, 0.0, a), np.where(mark, 1.0, m), g, mark


def gate_fwd(x, f, rate, i=None, z=None, f_bias=None, i_bias=None, reset=None, h0=None):
    """Returns out, the states h (B,D,L) and the last one (B,D)."""
    x = np.asarray(x, f64)
    s, la, a, m, g, mark = _gates(x, f, rate, i, f_bias, i_bias, reset)
    h = np.empty_like(x)
    c = np.zeros(x.shape[:2]) if h0 is None else np.asarray(h0, f64)
    for t in range(x.shape[2]):
        c = np.where(mark[..., t], 0.0, a[..., t] * c) + m[..., t] * g[..., t] * x[..., t]
        h[..., t] = c
    out = h if z is None else h * np.asarray(z, f64) * _sigmoid(np.asarray(z, f64))
    return out, h, c


def gate_bwd(dout, x, f, rate, i=None, z=None, f_bias=None, i_bias=None, reset=None, h0=None, dh_last=None):
    x, dout = np.asarray(x, f64), np.asarray(dout, f64)
    s, la, a, m, g, mark = _gates(x, f, rate, i, f_bias, i_bias, reset)
    _, h, _ = gate_fwd(x, f, rate, i, z, f_bias, i_bias, reset, h0)
    r = {}
    dy = dout
    if z is not None:
        z = np.asarray(z, f64)
        sz = _sigmoid(z)
        r["dz"] = dout * h * (sz + z * sz * (1.0 - sz))
        dy = dout * z * sz
    start = np.zeros(x.shape[:2]) if h0 is None else np.asarray(h0, f64)
    lam = np.empty_like(x)
    c = np.zeros(x.shape[:2]) if dh_last is None else np.asarray(dh_last, f64)
    for t in range(x.shape[2] - 1, -1, -1):
        lam[..., t] = dy[..., t] + c
        c = np.where(mark[..., t], 0.0, a[..., t] * lam[..., t])
    r["dh0"] = c
    before = np.concatenate((start[..., None], h[..., :-1]), -1)[..., : x.shape[2]]
    r["dx"] = lam * m * g
    if i is not None:
        di = lam * m * x * g * (1.0 - g)
        r["di"], r["di_bias"], r["di_bias_size"] = di, di.sum((0, 2)), np.abs(di).sum((0, 2))
    with np.errstate(divide="ignore", invalid="ignore"):
        slope = np.where(m > 0.0, a * a / m, 0.0)   # -dm / d(log a)
        dla = np.where(mark, 0.0, lam * (before * a - g * x * slope))
    with np.errstate(invalid="ignore"):   # at a mark the logit, whatever it is, has no part
        df, dr = np.where(mark, 0.0, dla * la * (1.0 - s)), np.where(mark, 0.0, -dla * s)
    r["df"], r["df_bias"], r["df_bias_size"] = df, df.sum((0, 2)), np.abs(df).sum((0, 2))
    r["drate"], r["drate_size"] = dr.sum((0, 2)), np.abs(dr).sum((0, 2))
    return r


# ---- 8-bit integers ---------------------------------------------------------------------------------
def quant_rows(x):
    """q (rows, K) as integers and scale (rows), both in the float32 arithmetic that the definition gives."""
    x = np.asarray(x, np.float32)
    top = np.abs(x).max(1, initial=0.0)
    some = top >= np.float32(2.0 ** -120)
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        inv = np.where(some, np.float32(127.0) * (np.float32(1.0) / top), np.float32(0.0)).astype(np.float32)
        scale = np.where(np.isfinite(top), np.where(some, top / np.float32(127.0), np.float32(0.0)), np.float32(np.nan)).astype(np.float32)
        p = x * inv[:, None]
    q = np.where(np.isnan(p), np.float32(0.0), np.rint(p)).astype(np.int64)
    return q, scale


def qlinear(q, x_scale, w, w_scale, bias=None):
    """Exact integer sums, the rest in 64 bits."""
    out = (q @ w.T).astype(f64) * x_scale.astype(f64)[:, None] * w_scale.astype(f64)[None, :]
    return out if bias is None else out + np.asarray(bias, f64)
