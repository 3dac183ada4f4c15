"""Gated recurrence where several waves share a row, and where its segments are scanned side by side: the sizes at which the plan
changes, against the float64 oracle (tolerances: test_gpu_gate)."""
import pytest

from tests.test_gpu_gate import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("nb,nd,nl", [(1, 1100, 1025), (1, 1100, 5000), (4, 1024, 1030), (2, 512, 1536), (1, 191, 8200), (1, 192, 9000), (3, 5, 2561), (1, 30, 4096),
                                      (1, 3, 70000), (2, 10, 40001)])
def test_rows_and_lengths(nb, nd, nl, io):
    check(nb, nd, nl, io, seed=nl, h0=True, reset=0.0005)
    check(nb, nd, nl, io, seed=nl + 1, i=nl % 2 == 0, z=nl % 3 == 0, dh_last=False)


def test_one_long_row():
    check(1, 1, 600000, "f32", h0=True)


@pytest.mark.parametrize("reset", [1.0, 0.3])
def test_many_resets(reset):
    check(1, 6, 20000, "f32", reset=reset, h0=True)
    check(1, 1030, 2000, "bf16", reset=reset, h0=True)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 511, 512])
def test_rounds(rows, io):
    """One round of a team's pieces and more, even and odd numbers of them, whole and not: two are requested ahead below 512 rows."""
    for nl in (1025, 2048, 2049, 4095, 4096, 4097, 6144, 8193):
        check(1, rows, nl, io, seed=nl, h0=True, reset=0.001 if nl % 2 else 0.0)
