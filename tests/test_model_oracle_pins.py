"""The float64 oracles of RMS norm, embedding, log probabilities and AdamW against closed forms, torch in float64 and finite differences."""
import numpy as np
import torch

from oracle import model_oracle as mo


def differences(f, x, dout, h=1e-6):
    """Gradient of <f(x), dout> by central differences, coordinate by coordinate."""
    g = np.zeros_like(x)
    for k in np.ndindex(*x.shape):
        at = [x.copy(), x.copy()]
        at[0][k] += h
        at[1][k] -= h
        g[k] = sum(s * (f(a) * dout).sum() for s, a in zip((1, -1), at)) / (2 * h)
    return g


# ---- RMS norm -----------------------------------------------------------------------------------------
def test_rms_norm_closed_forms():
    out, xhat, rstd = mo.rms_fwd([[3.0, 4.0]], eps=0.0)   # mean square 12.5
    assert np.allclose(out, [[3 / 12.5 ** 0.5, 4 / 12.5 ** 0.5]]) and np.allclose(rstd, 12.5 ** -0.5)
    s = np.random.default_rng(0).standard_normal((5, 9))
    assert np.allclose((mo.rms_fwd(s, eps=0.0)[1] ** 2).mean(1), 1.0)
    assert np.allclose(mo.rms_fwd(7.0 * s, eps=0.0)[0], mo.rms_fwd(s, eps=0.0)[0])   # scale does not matter
    assert np.allclose(mo.rms_fwd(np.zeros((1, 4)))[0], 0.0)
    w, b = np.arange(9.0), np.ones(9)
    assert np.allclose(mo.rms_fwd(s, w, b)[0], mo.rms_fwd(s)[0] * w + b)


def test_rms_norm_gradients():
    rng = np.random.default_rng(1)
    s, w, dout, more = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal((3, 7)), rng.standard_normal((3, 7))
    g = mo.rms_bwd(dout, s, w, more)
    assert np.allclose(g["ds"] - more, differences(lambda v: mo.rms_fwd(v, w)[0], s, dout), atol=1e-7)
    assert np.allclose(g["dweight"], differences(lambda v: mo.rms_fwd(s, v)[0], w, dout), atol=1e-7)
    assert np.allclose(g["dbias"], dout.sum(0))
    # a gradient along s itself changes nothing when eps is 0
    assert np.allclose((mo.rms_bwd(dout, s, w, eps=0.0)["ds"] * s).sum(1), 0.0, atol=1e-12)


# ---- embedding ----------------------------------------------------------------------------------------
def test_embedding():
    rng = np.random.default_rng(2)
    ids, table, dout = rng.integers(0, 5, (3, 4)), rng.standard_normal((5, 6)), rng.standard_normal((3, 4, 6))
    w = torch.from_numpy(table).requires_grad_(True)
    out = 0.5 * torch.nn.functional.embedding(torch.from_numpy(ids), w)
    out.backward(torch.from_numpy(dout))
    assert np.allclose(mo.embed_fwd(ids, table, 0.5), out.detach()) and np.allclose(mo.embed_bwd(dout, ids, 5, 0.5)["dtable"], w.grad)
    ids[0, 0], ids[1, 1] = -1, 5   # outside: zeros, and no gradient
    assert (mo.embed_fwd(ids, table)[0, 0] == 0).all() and (mo.embed_fwd(ids, table)[1, 1] == 0).all()
    total = mo.embed_bwd(dout, ids, 5)["dtable"].sum(0)
    assert np.allclose(total, dout.sum((0, 1)) - dout[0, 0] - dout[1, 1])


# ---- log probabilities --------------------------------------------------------------------------------
def test_log_probabilities():
    rng = np.random.default_rng(3)
    x, t, dl, dh = 3 * rng.standard_normal((6, 11)), rng.integers(0, 11, 6), rng.standard_normal(6), rng.standard_normal(6)
    t[4] = -1
    v = torch.from_numpy(x).requires_grad_(True)
    logs = torch.log_softmax(v, -1)
    logp = torch.where(torch.from_numpy(t) < 0, 0.0, logs[torch.arange(6), torch.from_numpy(t).clamp(min=0)])
    entropy = -(logs.exp() * logs).sum(-1)
    grad, = torch.autograd.grad((logp * torch.from_numpy(dl)).sum() + (entropy * torch.from_numpy(dh)).sum(), v)
    f = mo.logprob_fwd(x, t, 4)
    assert np.allclose(f["logp"], logp.detach()) and np.allclose(f["entropy"], entropy.detach()) and np.allclose(f["p"].sum(1), 1.0)
    assert np.allclose(mo.logprob_bwd(f, t, dl, dh)["dlogits"], grad)
    assert np.array_equal(f["top_ids"], torch.topk(v, 4).indices) and np.allclose(f["top_logp"], torch.topk(logs, 4).values.detach())
    assert np.allclose(mo.logprob_bwd(f, t, dl)["dlogits"].sum(1), 0.0)   # a shift of all logits changes nothing


def test_log_probabilities_of_masked_rows():
    inf = np.inf
    x = np.array([[0.0, -inf, 0.0, 0.0], [-inf] * 4, [-inf, 2.0, -inf, -inf], [0.0, np.nan, 1.0, inf]])
    f = mo.logprob_fwd(x, [1, 2, 1, 0], 3)
    assert np.array_equal(f["logp"][:3], [-inf, -inf, 0.0]) and np.allclose(f["entropy"][:3], [np.log(3), 0.0, 0.0]) and np.isnan(f["logp"][3])
    assert f["top_ids"].tolist() == [[0, 2, 3], [0, 1, 2], [1, 0, 2], [3, 2, 0]]
    g = mo.logprob_bwd(f, [1, 2, 1, 0], np.ones(4), np.ones(4))["dlogits"]
    assert np.allclose(g[0], [-1 / 3, 1.0, -1 / 3, -1 / 3]) and (g[1] == 0).all() and (g[2] == 0).all() and np.isnan(g[3]).any()
    assert mo.logprob_fwd(np.array([[np.nan, 1.0]]), None, 2)["top_ids"].tolist() == [[1, -1]]


# ---- AdamW --------------------------------------------------------------------------------------------
def test_adamw_like_torch():
    rng = np.random.default_rng(4)
    p = torch.from_numpy(rng.standard_normal(50)).requires_grad_(True)
    o = torch.optim.AdamW([p], lr=1e-2, betas=(0.75, 0.875), weight_decay=0.1)   # factors that float32 holds
    x, m, v = p.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for step in range(1, 6):
        p.grad = torch.from_numpy(rng.standard_normal(50))
        o.step()
        x, m, v, _ = mo.adamw(x, p.grad.numpy(), m, v, step, 1e-2, 0.75, 0.875, 1e-8, 0.1)
        assert np.allclose(x, p.detach(), rtol=1e-12, atol=1e-14)


def test_adamw_codes():
    rng = np.random.default_rng(5)
    x = rng.standard_normal(700)
    for signed in (True, False):
        w = x if signed else np.abs(x)
        top = 127 if signed else 255
        codes, scale = mo.adamw_codes(w, 3, signed)
        back = mo.adamw_values(codes, scale, signed)
        at = np.repeat(scale, 256)[:700]
        assert (np.abs(back - w) <= (2 * np.abs(codes) + 1) / top ** 2 * at).all() and np.array_equal(scale, [np.abs(w[k:k + 256]).max() for k in (0, 256, 512)])
        assert np.abs(codes).max() == top and (np.sign(back) == np.sign(w))[np.abs(codes) > 0].all()
        # the mean over many steps is the value
        mean = np.mean([mo.adamw_values(*mo.adamw_codes(w[:64], t, signed), signed) for t in range(2000)], 0)
        assert np.abs(mean - w[:64])[np.abs(w[:64]) > 1e-3].max() < 0.02 * (2 * np.abs(codes).max() + 1) / top ** 2 * scale[0]
    codes, scale = mo.adamw_codes([0.0] * 256 + [1.0, np.nan] + [0.0] * 254 + [1e-40], 1, True)
    assert (codes[:256] == 0).all() and scale[0] == 0 and np.isnan(scale[1]) and scale[2] == 0
    assert mo.adamw_codes([1.0, 1e-9, 0.0], 1, False)[0].tolist() == [255, 1, 0]
