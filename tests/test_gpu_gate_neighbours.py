"""The gated recurrence's gradients where something that has no part in them is NaN: memory behind a row, the next channel, a decay logit
that a mark makes void.  The same calls without the NaN give the same bits."""
import numpy as np
import pytest
import torch

from paper_2312_00752_amd import binding as B
from tests import op_util as u
from tests.test_gpu_gate import make, on_gpu

pytestmark = pytest.mark.gpu
LENGTHS = [5, 21, 37, 133, 1030]   # 4, 16 and 64 lanes a row, teams of waves; no multiple of a lane's eight steps


def gradients(dout, ws, **g):
    out, _ = B.ss_gate_fwd(**g, workspace=ws, save_for_bwd=True)
    return {"out": out, **B.ss_gate_bwd(dout, workspace=ws, want_dh0="h0" in g, **g)}


def workspace(nb, nd, nl):
    return torch.empty(max(256, B.ss_gate_workspace_bytes(nb, nd, nl)), dtype=torch.uint8, device="cuda")


def same(a, b, skip=()):
    for name in a:
        if a[name] is not None and name not in skip:
            assert torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("nl", LENGTHS)
@pytest.mark.parametrize("reset", [0.0, 0.05])
def test_memory_behind_the_rows(nl, io, reset):
    """Each input is a slice of a wider tensor of its own, with NaN before and behind."""
    nb, nd = 3, 10
    d, big = make(nb, nd, nl, io, reset=reset, h0=True)
    g = on_gpu(d, big, io)
    dout = u.upload(np.random.default_rng(1).standard_normal((nb, nd, nl)), io)
    ws = workspace(nb, nd, nl)
    want = gradients(dout, ws, **g)
    for name in big:
        wide = torch.full((nb, nd + 2, nl), float("nan"), dtype=u.TYPES[io], device="cuda")
        wide[:, 1:1 + nd] = g[name]
        got = gradients(dout, ws, **{**g, name: wide[:, 1:1 + nd]})
        same(want, got)
        assert all(torch.isfinite(v).all() for v in got.values() if v is not None), name


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("nl", LENGTHS)
def test_the_next_channel(nl, io):
    """NaN in one channel's inputs and gradient leaves the others' as they are."""
    nb, nd, bad = 2, 20, 7
    d, big = make(nb, nd, nl, io, h0=True)
    g = on_gpu(d, big, io)
    dout = u.upload(np.random.default_rng(2).standard_normal((nb, nd, nl)), io)
    ws = workspace(nb, nd, nl)
    want = gradients(dout, ws, **g)
    rest = [k for k in range(nd) if k != bad]
    for name in big + ("dout",):
        t = (dout if name == "dout" else g[name]).clone()
        t[:, bad] = float("nan")
        got = gradients(t, ws, **g) if name == "dout" else gradients(dout, ws, **{**g, name: t})
        for k, v in want.items():
            axis = 0 if v.dim() == 1 else 1
            at = torch.tensor(rest, device="cuda")
            assert torch.equal(v.index_select(axis, at), got[k].index_select(axis, at)), (name, k)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("nl", LENGTHS)
@pytest.mark.parametrize("logit", [float("nan"), float("inf"), -float("inf")])
def test_the_decay_logit_at_a_mark(nl, io, logit):
    """At a mark the decay has no part, whatever its logit: the forward pass ignores it and its gradient is 0."""
    nb, nd = 2, 9
    d, big = make(nb, nd, nl, io, h0=True)
    d["reset"] = np.zeros((nb, nl), bool)
    d["reset"][:, [0, nl // 2, nl - 1]] = True
    g = on_gpu(d, big, io)
    dout = u.upload(np.random.default_rng(3).standard_normal((nb, nd, nl)), io)
    ws = workspace(nb, nd, nl)
    want = gradients(dout, ws, **g)
    f = torch.where(g["reset"][:, None], torch.tensor(logit, dtype=u.TYPES[io], device="cuda"), g["f"])
    got = gradients(dout, ws, **{**g, "f": f})
    same(want, got)
    assert not got["df"].masked_select(g["reset"][:, None].expand(nb, nd, nl)).any()
