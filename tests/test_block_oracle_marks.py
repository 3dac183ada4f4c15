"""The recurrence's oracle at reset marks: the decay has no part there, so its logit may be anything and has no gradient."""
import numpy as np
import pytest

from oracle import block_oracle as bo


@pytest.mark.parametrize("logit", [np.nan, np.inf, -np.inf])
def test_the_decay_logit_at_a_mark(logit):
    rng = np.random.default_rng(1)
    x, f, i, z, dout = rng.standard_normal((5, 2, 3, 20))
    rate = rng.uniform(0.5, 2.0, 3)
    reset = np.zeros((2, 20), bool)
    reset[:, [0, 7, 19]] = True
    bad = np.where(reset[:, None], logit, f)
    kw = dict(i=i, z=z, f_bias=rate, i_bias=rate, reset=reset, h0=x[..., 0])
    for a, b in zip(bo.gate_fwd(x, f, rate, **kw), bo.gate_fwd(x, bad, rate, **kw)):
        assert np.array_equal(a, b)
    want, got = bo.gate_bwd(dout, x, f, rate, **kw), bo.gate_bwd(dout, x, bad, rate, **kw)
    assert set(want) == set(got)
    for name in want:
        assert np.array_equal(want[name], got[name]), name
    assert not got["df"][:, :, [0, 7, 19]].any()
