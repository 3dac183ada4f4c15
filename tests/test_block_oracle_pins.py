"""The float64 oracles of the block's operators against closed forms, finite differences and each other."""
import numpy as np
import pytest

from oracle import block_oracle as bo


def _gate_inputs(rng, nb=2, nd=3, nl=9, reset=False):
    d = dict(x=rng.standard_normal((nb, nd, nl)), f=rng.standard_normal((nb, nd, nl)), rate=rng.uniform(0.2, 2.0, nd),
             i=rng.standard_normal((nb, nd, nl)), z=rng.standard_normal((nb, nd, nl)), f_bias=rng.standard_normal(nd),
             i_bias=rng.standard_normal(nd), h0=rng.standard_normal((nb, nd)))
    if reset:
        d["reset"] = rng.random((nb, nl)) < 0.3
    return d


def test_gate_is_a_power_of_the_rate():
    """f very large: a = exp(-rate) at every step, so h is a geometric sum."""
    nl, rate = 7, np.array([0.3])
    x = np.ones((1, 1, nl))
    out, h, last = bo.gate_fwd(x, np.full((1, 1, nl), 800.0), rate)
    a = np.exp(-0.3)
    want = np.sqrt(1 - a * a) * (1 - a ** np.arange(1, nl + 1)) / (1 - a)
    np.testing.assert_allclose(h[0, 0], want, rtol=1e-13)
    assert last[0, 0] == h[0, 0, -1] and np.array_equal(out, h)


def test_gate_keeps_variance():
    rng = np.random.default_rng(0)
    x, f = rng.standard_normal((1, 1, 20000)), rng.standard_normal((1, 1, 20000))
    _, h, _ = bo.gate_fwd(x, f, np.array([0.5]))
    assert abs(h[..., 100:].var() - 1.0) < 0.05


def test_gate_pieces_and_resets():
    rng = np.random.default_rng(1)
    d = _gate_inputs(rng)
    out, h, last = bo.gate_fwd(**d)
    seq = ("x", "f", "i", "z")
    first, second = ({**d, **{k: d[k][..., s] for k in seq}} for s in (slice(0, 4), slice(4, None)))
    o1, _, mid = bo.gate_fwd(**first)
    o2, _, end = bo.gate_fwd(**{**second, "h0": mid})
    np.testing.assert_allclose(np.concatenate((o1, o2), -1), out, rtol=1e-13)
    np.testing.assert_allclose(end, last, rtol=1e-13)
    mark = np.zeros((2, 9), bool)
    mark[:, 4] = True
    r = bo.gate_fwd(**{**d, "reset": mark})[0]
    np.testing.assert_allclose(r[..., :4], out[..., :4])
    # at the mark a = 0 and m = 1: the state is the gated input alone
    g = 1 / (1 + np.exp(-(d["i"][..., 4] + d["i_bias"])))
    z = d["z"][..., 4]
    np.testing.assert_allclose(r[..., 4], g * d["x"][..., 4] * z / (1 + np.exp(-z)))
    d["x"][..., 1] = np.nan
    assert np.isfinite(bo.gate_fwd(**{**d, "reset": mark})[0][..., 4:]).all()


@pytest.mark.parametrize("reset", [False, True])
def test_gate_gradients_by_differences(reset):
    rng = np.random.default_rng(2)
    d = _gate_inputs(rng, reset=reset)
    w, wl = rng.standard_normal((2, 3, 9)), rng.standard_normal((2, 3))

    def loss(**k):
        out, _, last = bo.gate_fwd(**{**d, **k})
        return (out * w).sum() + (last * wl).sum()
    g = bo.gate_bwd(w, dh_last=wl, **d)
    for name, grad in (("x", "dx"), ("f", "df"), ("i", "di"), ("z", "dz"), ("rate", "drate"), ("f_bias", "df_bias"),
                       ("i_bias", "di_bias"), ("h0", "dh0")):
        v = rng.standard_normal(d[name].shape)
        e = 1e-5
        num = (loss(**{name: d[name] + e * v}) - loss(**{name: d[name] - e * v})) / (2 * e)
        assert abs(num - (g[grad] * v).sum()) < 1e-7 * (1 + abs(num)), name


def test_norm_gradients_by_differences():
    rng = np.random.default_rng(3)
    s, w, b = rng.standard_normal((4, 7)), rng.standard_normal(7), rng.standard_normal(7)
    dout, more = rng.standard_normal((4, 7)), rng.standard_normal((4, 7))
    g = bo.norm_bwd(dout, s, w, more)

    def loss(s=s, w=w, b=b):
        return (bo.norm_fwd(s, w, b)[0] * dout).sum() + (s * more).sum()
    e = 1e-5
    for name, grad in (("s", "ds"), ("w", "dweight"), ("b", "dbias")):
        base = {"s": s, "w": w, "b": b}[name]
        v = rng.standard_normal(base.shape)
        num = (loss(**{name: base + e * v}) - loss(**{name: base - e * v})) / (2 * e)
        assert abs(num - (g[grad] * v).sum()) < 1e-7 * (1 + abs(num)), name
    out, xhat, _ = bo.norm_fwd(s)
    np.testing.assert_allclose(out.mean(1), 0, atol=1e-14)
    np.testing.assert_allclose((out ** 2).mean(1), 1, rtol=1e-4)


def test_quant_rows():
    x = np.array([[1.0, -0.5, 0.25], [0.0, 0.0, 0.0], [1e-38, 0.0, 0.0], [np.inf, 1.0, 2.0], [np.nan, 1.0, 2.0], [127.0, 2.5, 3.5]])
    q, s = bo.quant_rows(x)
    assert q[0].tolist() == [127, -64, 32] and abs(s[0] - 1 / 127) < 1e-9
    assert not q[1:3].any() and not s[1:3].any()
    assert np.isnan(s[3:5]).all()
    assert q[5].tolist() == [127, 2, 4]   # ties to even
    rng = np.random.default_rng(4)
    v = rng.standard_normal((5, 40)).astype(np.float32)
    q, s = bo.quant_rows(v)
    assert np.abs(q * s[:, None] - v).max() <= 0.5001 * s.max() and np.abs(q).max() == 127
    w, ws = bo.quant_rows(rng.standard_normal((6, 40)))
    np.testing.assert_allclose(bo.qlinear(q, s, w, ws), (q * s[:, None].astype(float)) @ (w * ws[:, None].astype(float)).T, rtol=1e-12)
