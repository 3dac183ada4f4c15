"""The gated recurrence with more channels than the sums of its parameters' gradients have threads for at a time, and with rows of more
than 2^28 steps.  Tolerance as in test_gpu_gate.py."""
import pytest
import torch

from paper_2312_00752_amd import binding as B
from tests import op_util as u
from tests.test_gpu_gate import FWD

pytestmark = pytest.mark.gpu


def test_many_channels():
    """Two entries of one step of 2^28 channels and some: the same bits as the ends by themselves."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB")
    nb, nd = 2, (1 << 28) + 21

    def gradients(x, f, dout, rate, f_bias):
        ws = torch.empty(max(256, B.ss_gate_workspace_bytes(*x.shape)), dtype=torch.uint8, device="cuda")
        out, _ = B.ss_gate_fwd(x, f, rate, f_bias=f_bias, workspace=ws, save_for_bwd=True)
        return {"out": out, **B.ss_gate_bwd(dout, x, f, rate, ws, f_bias=f_bias)}
    x, f, dout = (torch.randn(nb, nd, 1, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    rate = torch.rand(nd, device="cuda")
    whole = gradients(x, f, dout, rate, rate)
    for cut in (slice(0, 100), slice(nd // 2, nd // 2 + 40), slice(nd - 100, nd)):
        part = gradients(*(t[:, cut].contiguous() for t in (x, f, dout)), rate[cut].contiguous(), rate[cut].contiguous())
        for name, t in part.items():
            if t is not None:
                w = whole[name][cut] if t.dim() == 1 else whole[name][:, cut]
                assert torch.equal(t, w), (name, cut)


def test_marks_of_very_long_rows():
    """A row of 2^28 steps and some: marks at its start, within and at its end, against the pieces that begin there."""
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GiB")
    nl = (1 << 28) + 13
    x, f = (torch.randn(1, 1, nl, device="cuda") for _ in range(2))
    rate = torch.ones(1, device="cuda")
    reset = torch.zeros(1, nl, dtype=torch.bool, device="cuda")
    starts = [0, 3, nl // 2 + 1, nl - 700, nl - 5]
    reset[0, starts] = True
    h0 = torch.full((1, 1), 1e30, device="cuda")
    out, last = B.ss_gate_fwd(x, f, rate, reset=reset, h0=h0, return_last_state=True)
    for a, b in zip(starts, starts[1:] + [nl]):
        b = min(b, a + 600)
        part = B.ss_gate_fwd(x[..., a:b].contiguous(), f[..., a:b].contiguous(), rate, reset=reset[:, a:b].contiguous())[0]
        u.close(out[..., a:b], u.host(part), FWD, "from %d" % a)
    assert torch.equal(last, out[..., -1])
