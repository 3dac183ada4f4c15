"""A state that is carried on in place: h_last in h0's memory, and the adjoint dh0 in dh_last's.  Rows that one wave walks, that teams share
and that are cut into segments, whose last one ends while the first may not have begun."""
import pytest
import torch

from paper_2312_00752_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("reset", [False, True])
@pytest.mark.parametrize("nb,nd,nl", [(3, 40, 7), (2, 33, 100), (5, 700, 300), (2, 30, 2100), (1, 4, 50000), (2, 64, 40000), (1, 160, 30000)])
def test_in_place(nb, nd, nl, reset, io):
    x, f, dout = (torch.randn(nb, nd, nl, device="cuda").to(io) for _ in range(3))
    rate = torch.rand(nd, device="cuda") + 0.5
    f_bias = torch.full((nd,), -9.0, device="cuda")   # the first state reaches the last one
    marks = torch.rand(nb, nl, device="cuda") < 1.0 / nl if reset else None
    h0, dh_last = (torch.randn(nb, nd, device="cuda") for _ in range(2))
    ws = [torch.empty(max(256, B.ss_gate_workspace_bytes(nb, nd, nl)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    out, last = B.ss_gate_fwd(x, f, rate, f_bias=f_bias, reset=marks, h0=h0, return_last_state=True, workspace=ws[0], save_for_bwd=True)
    want = B.ss_gate_bwd(dout, x, f, rate, ws[0], f_bias=f_bias, reset=marks, h0=h0, dh_last=dh_last, want_dh0=True)
    for _ in range(3):
        h, adjoint = h0.clone(), dh_last.clone()
        got, same = B.ss_gate_fwd(x, f, rate, f_bias=f_bias, reset=marks, h0=h, h_last=h, workspace=ws[1], save_for_bwd=True)
        assert same is h and torch.equal(got, out) and torch.equal(h, last)
        g = B.ss_gate_bwd(dout, x, f, rate, ws[1], f_bias=f_bias, reset=marks, h0=h, dh_last=adjoint, want_dh0=True, grads={"dh0": adjoint})
        for name, t in want.items():
            assert t is None or torch.equal(g[name], t), name
