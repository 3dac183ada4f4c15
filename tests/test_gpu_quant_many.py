"""Products in 8-bit integers with more tiles, or more features, than one launch of small workgroups has threads for: the same bits as
parts of them by themselves."""
import pytest
import torch

from paper_2312_00752_amd import binding as B

pytestmark = pytest.mark.gpu


def _room(gib):
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip("needs %d GiB" % gib)


def test_many_short_sequences():
    """65535 entries of two tokens, sequence last: 16.8 million tiles of 64 x 64."""
    _room(12)
    nb, nl, nk, nf = 65535, 2, 72, 16448
    x = torch.randn(nb, nl, nk, device="cuda").bfloat16()
    w, s = B.ss_quant_rows(torch.randn(nf, nk, device="cuda"))
    out = B.ss_qlinear(x, w, s, out_seq_last=True)
    for at in (0, 1, 32767, 65533):
        part = B.ss_qlinear(x[at:at + 2], w, s, out_seq_last=True)
        assert torch.equal(out[at:at + 2], part), at


@pytest.mark.parametrize("rows", [1, 5])
def test_many_features(rows):
    """A vocabulary of 2^27 and some for few tokens: too many for workgroups of 16 features."""
    _room(40)
    nk, nf = 16, (1 << 27) + 19
    w = torch.zeros(nf, B.ss_quant_pitch(nk), dtype=torch.int8, device="cuda")
    w[:, :nk] = torch.randint(-127, 128, (nf, 1), dtype=torch.int8, device="cuda")
    w[:, 3] = 5
    s = torch.rand(nf, device="cuda")
    x = torch.randn(rows, nk, device="cuda")
    out = B.ss_qlinear(x, w, s)
    for a, b in ((0, 100), (nf // 2, nf // 2 + 77), (nf - 33, nf)):
        assert torch.equal(out[:, a:b], B.ss_qlinear(x, w[a:b], s[a:b])), (a, b)
