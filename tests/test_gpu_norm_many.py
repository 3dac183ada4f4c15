"""Layer norm with more columns, or more wide rows, than one launch has threads for."""
import pytest
import torch

from paper_2312_00752_amd import binding as B

pytestmark = pytest.mark.gpu


def _room(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip("needs %d GiB" % gib)


def test_many_columns():
    """One row of 2^27 columns and some: the weights' gradients are products, of which every one has to be there."""
    _room(12)
    width = (1 << 27) + 40
    x, dout = (torch.randn(1, width, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    w = torch.ones(width, device="cuda")
    _, _, stats = B.ss_norm_fwd(x, w, save_stats=True)
    g = B.ss_norm_bwd(dout, x, stats, w, has_bias=True)
    assert torch.equal(g["dbias"], dout[0].float())
    mean, rstd = stats[:, 0].tolist()
    want = (x[0].float() - mean) * rstd * dout[0].float()
    # three roundings on each side
    assert ((g["dweight"] - want).abs() <= 6 * 2.0 ** -24 * (x[0].float().abs() + abs(mean)) * rstd * dout[0].float().abs()).all()


def test_many_wide_rows():
    """2^22 rows of 16385 columns and some, in place; the ends against the same rows by themselves."""
    _room(150)
    rows, width = (1 << 22) + 5, 16385
    x = torch.zeros(rows, width, device="cuda", dtype=torch.bfloat16)
    ends = torch.randn(10, width, device="cuda", dtype=torch.bfloat16)
    x[:3], x[-7:] = ends[:3], ends[3:]
    want = B.ss_norm_fwd(ends)[0]
    B.ss_norm_fwd(x, out=x)
    assert torch.equal(x[:3], want[:3]) and torch.equal(x[-7:], want[3:])
    assert not x[3:100].any() and not x[-107:-7].any()
    del x
    torch.cuda.empty_cache()
