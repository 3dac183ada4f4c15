"""Sizes that do not fit the library's 32-bit counts are refused by the binding, not cut to their low 32 bits (a call would then work on a few
of its rows and leave the rest of its results as they were allocated).  Tensors without memory."""
import pytest
import torch

from paper_2312_00752_amd import binding as B

MANY = 2 ** 32 + 5


def t(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


W, S = t(8, 128, dtype=torch.int8), t(8, dtype=torch.float32)
CALLS = {
    "norm rows": lambda: B.ss_norm_fwd(t(MANY, 1)),
    "norm width": lambda: B.ss_norm_fwd(t(1, MANY)),
    "norm backward": lambda: B.ss_norm_bwd(t(3, MANY, 2), t(3, MANY, 2), t(2, 3 * MANY, dtype=torch.float32)),
    "norm workspace": lambda: B.ss_norm_workspace_bytes(MANY, 4),
    "recurrence steps": lambda: B.ss_gate_fwd(t(1, 1, MANY), t(1, 1, MANY), t(1, dtype=torch.float32)),
    "recurrence channels": lambda: B.ss_gate_fwd(t(1, MANY, 1), t(1, MANY, 1), t(MANY, dtype=torch.float32)),
    "recurrence backward": lambda: B.ss_gate_bwd(t(MANY, 1, 1), t(MANY, 1, 1), t(MANY, 1, 1), t(1, dtype=torch.float32), t(256, dtype=torch.uint8)),
    "recurrence token": lambda: B.ss_gate_step(t(MANY, 1, dtype=torch.float32), t(MANY, 1), t(MANY, 1), t(1, dtype=torch.float32)),
    "recurrence workspace": lambda: B.ss_gate_workspace_bytes(1, 1, MANY),
    "rows in 8 bits": lambda: B.ss_quant_rows(t(MANY, 1)),
    "a row in 8 bits": lambda: B.ss_quant_rows(t(1, MANY)),
    "tokens in 8 bits, sequence last": lambda: B.ss_quant_rows(t(1, 3, MANY), seq_last=True),
    "pitch": lambda: B.ss_quant_pitch(MANY),
    "product, tokens": lambda: B.ss_qlinear(t(MANY, 8), W, S),
    "product, tokens, sequence last": lambda: B.ss_qlinear(t(1, 8, MANY), W, S, x_seq_last=True),
    "product, features": lambda: B.ss_qlinear(t(4, 8), t(MANY, 128, dtype=torch.int8), t(MANY, dtype=torch.float32)),
    "product, scratch": lambda: B.ss_qlinear_scratch_bytes(1, MANY, 8, 8),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_refused(name):
    with pytest.raises(B.SsError) as e:
        CALLS[name]()
    assert e.value.code == B.SS_ERR_UNSUPPORTED


def test_the_largest_counts():
    """2^31 - 1 goes to the library, which has its own limits."""
    assert B.ss_quant_pitch(2 ** 31 - 1) == 2 ** 31
    assert B.ss_norm_workspace_bytes(2 ** 31 - 1, 16) > 0
    with pytest.raises(B.SsError):
        B.ss_quant_pitch(2 ** 31)
