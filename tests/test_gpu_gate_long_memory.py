"""Decays so near 1 that 1 - a^2 is no normal number: m counts as 0, and so does its derivative, forward and backward.

Against the float64 oracle with m set to 0 in such steps.  Tolerances as in test_gpu_gate.py."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2312_00752_amd import binding as B
from tests import op_util as u
from tests.test_gpu_gate import BWD, FWD, on_gpu

pytestmark = pytest.mark.gpu

# (rate, logit): 2 rate sigmoid(logit) is below 2^-126 = 1.18e-38 ...
BELOW = [(0.1, -86.5), (1e-4, -80.0), (1e-4, -83.0), (5e-39, 0.0), (1e-39, 0.0), (1e-39, -5.0), (0.4, -87.25)]
# ... and above it, by factors that the error of a sigmoid does not bridge
ABOVE = [(1.0, -85.0), (1.0, -79.0), (0.1, -82.0), (1e-4, -75.0), (1e-36, 0.0), (1e-4, -30.0), (2.0, -10.0), (1.0, 1.0)]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("reset", [False, True])
@pytest.mark.parametrize("nl", [1, 24, 100, 700, 2100])
def test_gradients(nl, reset, io, monkeypatch):
    pairs = BELOW + ABOVE
    nb, nd = 2, len(pairs)
    rng = np.random.default_rng(nl)
    big = ("x", "f", "i", "z")
    d = {k: u.rounded(rng.standard_normal((nb, nd, nl)) * (0.02 if k == "f" else 1.0), io) for k in big}
    d["x"][:, :, ::7] = 0.0   # 0 times an infinite m would be NaN
    d["rate"] = np.array([p[0] for p in pairs], np.float32)
    d["f_bias"] = np.array([p[1] for p in pairs], np.float32)
    d["i_bias"] = rng.standard_normal(nd).astype(np.float32)
    d["h0"] = rng.standard_normal((nb, nd)).astype(np.float32)
    if reset:
        d["reset"] = rng.random((nb, nl)) < 0.02
    g = on_gpu(d, big, io)
    dout = u.rounded(rng.standard_normal((nb, nd, nl)), io)
    ws = torch.full((max(256, B.ss_gate_workspace_bytes(nb, nd, nl)),), 0xFF, dtype=torch.uint8, device="cuda")
    out, last = B.ss_gate_fwd(**g, return_last_state=True, workspace=ws, save_for_bwd=True)
    grads = B.ss_gate_bwd(u.upload(dout, io), workspace=ws, want_dh0=True, **g)
    for name, t in {"out": out, "h_last": last, **grads}.items():
        assert torch.isfinite(t).all(), name
    gates = bo._gates

    def counted(*args):
        s, la, a, m, g, mark = gates(*args)
        return s, la, a, np.where(m < 2.0 ** -63, 0.0, m), g, mark
    monkeypatch.setattr(bo, "_gates", counted)
    ref, _, rl = bo.gate_fwd(**d)
    u.close(out, ref, FWD, "out")
    u.close(last, rl, FWD, "h_last")
    r = bo.gate_bwd(dout, **d)
    for name, t in grads.items():
        # the smallest channels' values and sums are themselves near the least normal number
        size = r.get(name + "_size")
        u.close(t, r[name], BWD, name, None if size is None else size + 2.0 ** -110)


def test_steps():
    """One token: m counts as 0 there as well, and the state stays, also at 0."""
    nd = len(BELOW)
    rate, f_bias = (torch.tensor([p[k] for p in BELOW], dtype=torch.float32, device="cuda") for k in (0, 1))
    h = torch.randn(3, nd, device="cuda")
    h[2] = 0.0
    x = torch.randn(3, nd, device="cuda")
    was = h.clone()
    out = B.ss_gate_step(h, x, torch.zeros(3, nd, device="cuda"), rate, f_bias=f_bias)
    assert torch.equal(h, was) and torch.equal(out, was)
    out, _ = B.ss_gate_fwd(x[..., None], torch.zeros(3, nd, 1, device="cuda"), rate, f_bias=f_bias)
    assert not out.any()
