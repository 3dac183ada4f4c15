"""An eps that is no normal float32 is refused, on the host, before any device call: its reciprocal would be infinite, and a step without a gradient NaN."""
import ctypes

import pytest

from paper_2312_00752_amd import binding as B
from tests.test_model_boundary_cpu import adamw, expect


@pytest.mark.parametrize("bits", [8, 32])
def test_refused(bits):
    expect(B.lib().ss_adamw_step, lambda: adamw(bits), [dict(eps=e) for e in (2.0 ** -127, 1e-38, 1e-42, 1e-46, 5e-324)], B.SS_ERR_UNSUPPORTED)


def test_the_least_and_none_are_not():
    """What is looked at behind eps is what refuses these."""
    for eps in (0.0, 2.0 ** -126, 1.2e-38):
        p = adamw()
        p.eps, p.lr = eps, float("inf")
        assert B.lib().ss_adamw_step(ctypes.byref(p), None) == B.SS_ERR_UNSUPPORTED
        p.lr, p.list[1].n = 1e-3, -1
        assert B.lib().ss_adamw_step(ctypes.byref(p), None) == B.SS_ERR_SHAPE
