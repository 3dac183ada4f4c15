"""The quantiser of tokens with the sequence last where registers hold all channels of a tile of tokens: both sides of every change
of its form, ragged tiles, rows without a scale.  The quantiser's arithmetic is fixed to the bit."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2312_00752_amd import binding as B
from tests import op_util as u

pytestmark = pytest.mark.gpu


def check(batch, dim, seqlen, io, change=None, bad=()):
    """``bad``: tokens whose scale must be NaN"""
    rng = np.random.default_rng(dim * 31 + seqlen)
    x = u.rounded(rng.standard_normal((batch, dim, seqlen)) * np.where(rng.random((batch, 1, seqlen)) < 0.1, 50.0, 1.0), io)
    if change:
        change(x)
    q, s = B.ss_quant_rows(u.upload(x, io), seq_last=True)
    rq, rs = bo.quant_rows(np.swapaxes(x, 1, 2).reshape(-1, dim))
    q, s = q.cpu().numpy(), s.cpu().numpy()
    assert not q[:, dim:].any()
    assert np.array_equal(s, rs, equal_nan=True) and set(np.flatnonzero(np.isnan(s))) == set(bad)
    assert np.array_equal(q[:, :dim], rq)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [1, 3, 127, 511, 512, 513, 1000, 1024, 1025, 2048, 2049, 4095, 4096, 4097, 6144, 6145])
def test_widths(dim, io):
    check(2, dim, 37, io)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("dim,tokens", [(300, 9000), (1500, 5999), (1500, 6000), (2047, 6003), (2500, 2999), (2500, 3000), (4096, 3999), (4096, 4001), (4500, 3000), (4500, 3001)])
def test_many_tokens(dim, tokens, io):
    check(1, dim, tokens, io)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("seqlen", [1, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 65])
def test_tiles(seqlen, io):
    check(5, 130, seqlen, io)
    check(2, 2100, seqlen, io)
    check(130, 2100, 33 if seqlen == 33 else seqlen % 30 + 31, io)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [40, 1100, 2100])
def test_rows_without_a_scale(dim, io):
    """Their bytes are 0 as well, also those of a NaN whose bits are not the usual ones."""
    def change(x):
        x[0, :, 3] = 0
        x[0, :, 4] = 1e-37
        x[0, dim // 2, 5] = np.inf
        x[1, 0, 0] = np.nan
        x[1, dim - 1, 18] = -np.inf
    check(2, dim, 19, io, change, bad=(5, 19, 37))
    bits = torch.full((1, dim, 3), 0x7fe500a5, dtype=torch.int32, device="cuda").view(torch.float32)
    x = torch.ones(1, dim, 3, device="cuda")
    x[:, 7::9] = bits[:, 7::9]
    q, s = B.ss_quant_rows(x if io == "f32" else (x.view(torch.int32) >> 16).to(torch.int16).view(torch.bfloat16), seq_last=True)
    assert torch.isnan(s).all() and not q.any()


@pytest.mark.parametrize("dim", [700, 4096, 5000])
def test_bytes_of_elementary_operations(dim):
    """The quantiser rounds as round(x * (127.0 / max |x|)) in torch does, so that products agree to the integer."""
    x = torch.randn(1, 1500, dim, device="cuda") * torch.rand(1, 1500, 1, device="cuda").mul(20).exp()
    want = torch.round(x * (127.0 / x.abs().amax(-1, keepdim=True)))[0].to(torch.int8)
    for t, last in ((x, False), (x.transpose(1, 2).contiguous(), True)):
        assert torch.equal(B.ss_quant_rows(t, seq_last=last)[0][:, :dim], want)


def test_more_rows_than_threads():
    """70 million tokens: offsets past 32 bits, and more threads than one launch may have, in either order."""
    n = 70_000_000
    few = torch.randn(8, 1000, device="cuda").bfloat16()
    last = torch.zeros(1, 8, n, dtype=torch.bfloat16, device="cuda")
    places = torch.cat((torch.arange(500), torch.arange(n - 500, n))).cuda()
    last[0][:, places] = few
    want = B.ss_quant_rows(few[None].contiguous(), seq_last=True)
    assert torch.equal(want[0][:, :8], B.ss_quant_rows(few.t().contiguous())[0][:, :8])
    for x, seq_last in ((last, True), (last[0].t().contiguous(), False)):
        q, s = B.ss_quant_rows(x, seq_last=seq_last)
        assert torch.equal(q[places], want[0]) and torch.equal(s[places], want[1])
        assert not s[500:n - 500].any() and not q[34_000_000:36_000_000].any()
        del q, s


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_rows_off_a_word(io):
    """Tokens' tensors that start one element into their memory."""
    for dim, tokens in ((40, 33), (2100, 100), (4000, 4100)):
        x = torch.randn(1, dim, tokens, device="cuda").to(u.TYPES[io])
        off = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape).copy_(x)
        for a, b in zip(B.ss_quant_rows(x, seq_last=True), B.ss_quant_rows(off, seq_last=True)):
            assert torch.equal(a, b)
