"""The recurrence's sigmoid against the float64 one, relative to its own value, from 80 below 0 to 80 above.

The exponential's argument -v log2(e) is rounded once and its constant once: (1 + 0.22) 2^-24 |v| of the result; then at most one unit
(2^-23) each of the exponential, the sum and the reciprocal.  Products around it here: three roundings more."""
import numpy as np
import pytest
import torch

from paper_2312_00752_amd import binding as B
from tests import op_util as u

pytestmark = pytest.mark.gpu


def logits():
    v = np.concatenate([np.linspace(-a, -b, 4001) for a, b in ((87.2, 40), (40, 20), (20, 10), (10, 5), (5, 0))])
    return np.concatenate((v, -v)).astype(np.float32)


def bound(v, roundings):
    return (1.25 * np.abs(v) + 6.0 + roundings) * u.EPS


@pytest.mark.parametrize("step", [False, True])
def test_input_gate(step):
    """h = m g x with m = 1 at a mark and x = 1."""
    v = logits().astype(np.float64)
    n = v.size
    x, f, i = torch.ones(1, n, device="cuda"), torch.zeros(1, n, device="cuda"), u.upload(v.reshape(1, n), "f32")
    rate, mark = torch.ones(n, device="cuda"), torch.ones(1, 1, dtype=torch.bool, device="cuda")
    if step:
        got = B.ss_gate_step(torch.zeros(1, n, device="cuda"), x, f, rate, i_t=i, reset_t=mark[:, 0].contiguous())
    else:
        got = B.ss_gate_fwd(x[..., None], f[..., None], rate, i=i[..., None], reset=mark)[0][..., 0]
    got, want = u.host(got).reshape(-1), 1.0 / (1.0 + np.exp(-v))
    off = np.abs(got - want) / want
    assert (off <= bound(v, 2)).all(), (v[np.argmax(off / bound(v, 2))], np.max(off / bound(v, 2)))


def test_output_gate():
    """out = h z sigmoid(z) with h = 1 at a mark."""
    v = logits().astype(np.float64)
    v = v[np.abs(v) > 1e-3]
    n = v.size
    one = torch.ones(1, n, 1, device="cuda")
    out, _ = B.ss_gate_fwd(one, one, torch.ones(n, device="cuda"), z=u.upload(v.reshape(1, n, 1), "f32"), reset=torch.ones(1, 1, dtype=torch.bool, device="cuda"))
    got, want = u.host(out).reshape(-1), v / (1.0 + np.exp(-v))
    off = np.abs(got - want) / np.abs(want)
    assert (off <= bound(v, 4)).all(), (v[np.argmax(off / bound(v, 4))], np.max(off / bound(v, 4)))


def test_below():
    """Under 2^-126, for logits below -87.33, it is 0 or within that of the value."""
    v = np.linspace(-120.0, -87.4, 999).reshape(1, 999, 1)
    one = torch.ones(1, 999, 1, device="cuda")
    out, _ = B.ss_gate_fwd(one, one, torch.ones(999, device="cuda"), i=u.upload(v, "f32"), reset=torch.ones(1, 1, dtype=torch.bool, device="cuda"))
    assert (out >= 0).all() and (out <= 2.0 ** -126).all()
