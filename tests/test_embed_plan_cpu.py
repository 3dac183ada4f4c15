"""The division of the embedding's gradient that the tests' tolerances are counted from is the library's: its scratch memory has the size that follows from it."""
import pytest

from paper_2312_00752_amd import binding as B
from tests import embed_plan


@pytest.mark.parametrize("n", [1, 8, 9, 1024, 1025, 4096, 4097, 5199, 16384, 16385, 40000, 65536, 300000, 2 ** 24 + 1])
@pytest.mark.parametrize("dim", [1, 8, 512, 513, 1021, 2048, 2049, 4099, 16384])
def test_pieces(n, dim):
    for vocab in (2, 257, 51200):
        assert B.ss_embed_workspace_bytes(n, vocab, dim) == embed_plan.workspace_bytes(n, vocab, dim)


def test_roundings():
    assert embed_plan.pieces(40000, 8) == (32, 1250) and embed_plan.roundings(40000, 8) == 32 + 8 + 79 + 5
    assert embed_plan.pieces(16384, 2048) == (32, 512) and embed_plan.roundings(16384, 2048) == 32 + 8 + 32 + 5
    assert embed_plan.pieces(5199, 1021) == (8, 650) and embed_plan.roundings(3, 5) == 3 + 1 + 5
