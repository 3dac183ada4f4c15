"""Prompts of one token and a few through the served block: on either side of the line between its two ways to 8 bits, the bits of the operators one by one."""
import pytest
import torch

from paper_2312_00752_amd import binding as B
from paper_2312_00752_amd import block as bk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("batch,length", [(1, 1), (2, 1), (4, 1), (5, 1), (17, 1), (1, 2), (4, 2), (1, 0)])
def test_the_same_bits(batch, length, dtype, norm, monkeypatch):
    torch.manual_seed(0)
    s = bk.GatedBlock(100, 60, dtype=dtype, norm=norm).serving()
    x = torch.randn(batch, length, 100, device="cuda").to(dtype)
    residual = torch.randn_like(x)
    h, summed, _ = B.ss_norm_fwd(x, s.norm_weight, s.norm_bias, residual=residual, eps=s.eps, rms=s.rms)
    xs, f, i, z = B.ss_qlinear(h, s.W_in, s.in_scale, out_seq_last=True).chunk(4, 1)
    y, state = B.ss_gate_fwd(xs, f, s.rate, i=i, z=z, f_bias=s.f_bias, i_bias=s.i_bias, return_last_state=True)
    want = B.ss_qlinear(y, s.W_out, s.out_scale, x_seq_last=True)
    if length == 1 and batch <= 4:   # no launch and no call more than a step's
        monkeypatch.setattr(B, "ss_norm_quant", lambda *a, **k: pytest.fail("a call more"))
    got, kept, last = s.prompt(x, residual)
    assert torch.equal(got, want) and torch.equal(kept, summed) and torch.equal(last, state)
