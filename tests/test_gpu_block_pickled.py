"""A block that was pickled as a whole before its norm could be chosen: it has layer norm."""
import io

import pytest
import torch

from paper_2312_00752_amd import block as bk

pytestmark = pytest.mark.gpu


def test_without_the_choice():
    torch.manual_seed(0)
    block = bk.GatedBlock(40, 24)
    old = bk.GatedBlock(40, 24)
    old.load_state_dict(block.state_dict())
    del old.__dict__["rms"]
    file = io.BytesIO()
    torch.save(old, file)
    file.seek(0)
    old = torch.load(file, weights_only=False)   # of this test's own making
    assert "rms" not in old.__dict__
    x = torch.randn(2, 9, 40, device="cuda")
    assert all(torch.equal(a, b) for a, b in zip(block(x), old(x)))
    served = old.serving()
    del served.__dict__["rms"]
    assert all(torch.equal(a, b) for a, b in zip(block.serving().prompt(x), served.prompt(x)))
