"""Products in 8-bit integers on the GPU against the oracle.

The quantiser's arithmetic is fixed to the bit, and the sums are exact, so what is left is the scaling: the sum's conversion to
float32, the scales' product, one multiply-add: 4 roundings of |product| + |bias| (op_util.close, in multiples of 2^-24)."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2312_00752_amd import binding as B
from tests import op_util as u

pytestmark = pytest.mark.gpu


def tokens(rng, batch, seqlen, dim, io):
    x = rng.standard_normal((batch, seqlen, dim)) * np.where(rng.random(dim) < 0.05, 6.0, 1.0)
    return u.rounded(x, io)


def check_rows(batch, seqlen, dim, io, seq_last, seed=0):
    x = tokens(np.random.default_rng(seed), batch, seqlen, dim, io)
    t = u.upload(np.swapaxes(x, 1, 2) if seq_last else x, io)
    q, s = B.ss_quant_rows(t, seq_last=seq_last)
    rq, rs = bo.quant_rows(x.reshape(-1, dim))
    assert q.shape == (batch * seqlen, -(-dim // 128) * 128)
    got = q.cpu().numpy()
    assert np.array_equal(got[:, :dim], rq) and not got[:, dim:].any()
    assert np.array_equal(s.cpu().numpy(), rs)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [1, 7, 8, 65, 127, 128, 129, 512, 513, 1500, 2048, 2049, 5000, 8193, 16384, 16385, 33000])
def test_rows(dim, io):
    check_rows(1, 3, dim, io, False, seed=dim)
    check_rows(2, 11, dim, io, True, seed=dim)


@pytest.mark.parametrize("seqlen", [1, 2, 7, 8, 9, 63, 64, 65, 255, 256, 257, 1000])
def test_rows_sequence_last(seqlen):
    for io in ("f32", "bf16"):
        check_rows(3, seqlen, 200, io, True, seed=seqlen)


def test_many_rows():
    for dim in (64, 700, 1024, 2000):
        check_rows(1, 3001, dim, "bf16", False)


def test_rows_without_a_scale():
    """Zero and tiny rows count as zero; an infinity or NaN makes its own row's scale NaN and no other's."""
    rng = np.random.default_rng(1)
    for dim in (40, 3000, 20000):
        x = rng.standard_normal((6, dim)).astype(np.float32)
        x[1] = 0
        x[2] = 1e-37
        x[3, dim // 2] = np.inf
        x[4, dim - 1] = np.nan
        rq, rs = bo.quant_rows(x)
        for t, last in ((u.upload(x, "f32"), False), (u.upload(x.T[None], "f32"), True)):
            q, s = B.ss_quant_rows(t, seq_last=last)
            assert np.array_equal(s.cpu().numpy(), rs, equal_nan=True)
            assert np.array_equal(q.cpu().numpy()[[0, 1, 2, 5], :dim], rq[[0, 1, 2, 5]])
        w, ws = B.ss_quant_rows(u.upload(rng.standard_normal((9, dim)), "f32"))
        out = B.ss_qlinear(u.upload(x, "f32"), w, ws, bias=torch.ones(9, device="cuda"))
        assert torch.isnan(out[3:5]).all() and (out[1:3] == 1).all() and torch.isfinite(out[[0, 5]]).all()


def check_linear(batch, seqlen, dim, features, io, x_last=False, out_last=False, bias=False, seed=0):
    rng = np.random.default_rng(seed)
    x = tokens(rng, batch, seqlen, dim, io)
    w = (rng.standard_normal((features, dim)) / np.sqrt(dim)).astype(np.float32)
    b = rng.standard_normal(features).astype(np.float32) if bias else None
    tb = None if b is None else torch.from_numpy(b).cuda()
    qw, sw = B.ss_quant_rows(torch.from_numpy(w).cuda())
    t = u.upload(np.swapaxes(x, 1, 2) if x_last else x, io)
    got = B.ss_qlinear(t, qw, sw, bias=tb, x_seq_last=x_last, out_seq_last=out_last)
    rq, rs = bo.quant_rows(x.reshape(-1, dim))
    rw, rws = bo.quant_rows(w)
    ref = bo.qlinear(rq, rs, rw, rws, b).reshape(batch, seqlen, features)
    size = np.abs(ref) + (0.0 if b is None else np.abs(b))
    if out_last:
        ref, size = np.swapaxes(ref, 1, 2), np.swapaxes(size, 1, 2)
    u.close(got, ref, 4, "out", size=size)
    if not x_last:   # tokens quantised beforehand
        q, s = B.ss_quant_rows(t)
        again = B.ss_qlinear(q.view(batch, seqlen, -1), qw, sw, bias=tb, out_seq_last=out_last, x_scale=s, dim=dim, out_dtype=u.TYPES[io])
        assert torch.equal(got, again)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("count", [1, 2, 3, 4, 5, 8, 15, 16, 17, 31, 32, 33, 48, 64, 65, 96, 127, 128, 129, 250, 300, 513])
def test_token_counts(count, io):
    check_linear(count, 1, 300, 200, io, seed=count)
    check_linear(1, count, 640, 513, io, out_last=True, bias=True, seed=count)


@pytest.mark.parametrize("dim", [1, 16, 100, 128, 129, 1000, 1024, 2048, 4097, 17000])
def test_dims(dim):
    for count in (1, 4, 40, 300):
        check_linear(1, count, dim, 130, "bf16", seed=dim)
    check_linear(2, 45, dim, 70, "f32", x_last=True, out_last=True, seed=dim)


@pytest.mark.parametrize("features", [1, 2, 15, 16, 17, 63, 64, 127, 128, 129, 255, 256, 257, 1000, 4096])
def test_features(features):
    for count in (1, 7, 200):
        check_linear(1, count, 384, features, "bf16", bias=True, seed=features)
    check_linear(2, 131, 384, features, "bf16", out_last=True, bias=True, seed=features)


@pytest.mark.parametrize("x_last", [False, True])
@pytest.mark.parametrize("out_last", [False, True])
@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_layouts(x_last, out_last, io):
    check_linear(3, 77, 260, 190, io, x_last, out_last, True)
    check_linear(1, 600, 512, 768, io, x_last, out_last)
    check_linear(5, 1, 130, 33, io, x_last, out_last, True)


def test_large():
    check_linear(1, 2500, 1024, 1600, "bf16", False, True)
    check_linear(2, 1100, 2048, 1100, "bf16", True, False)


def test_sums_are_exact():
    """The largest sum that the contraction index allows, where float32 sums would be off."""
    dim = 131072
    q = torch.full((2, dim), 127, dtype=torch.int8, device="cuda")
    q[1, ::2] = -127
    w = torch.full((3, dim), 127, dtype=torch.int8, device="cuda")
    w[2, 5] = 126
    one = torch.ones(3, device="cuda")
    for count in (1, 2):
        out = B.ss_qlinear(q[:count], w, one, x_scale=one[:count], dim=dim, out_dtype=torch.float32)
        top = 127 * 127 * dim
        want = torch.tensor([[top, top, top - 127], [0, 0, -127]], dtype=torch.float64)[:count]
        assert torch.equal(out.double().cpu(), want.float().double())


def test_nothing_and_shapes():
    w, s = B.ss_quant_rows(torch.randn(6, 20, device="cuda"))
    assert B.ss_qlinear(torch.empty(0, 20, device="cuda"), w, s).shape == (0, 6)
    assert B.ss_qlinear(torch.empty(2, 20, 0, device="cuda"), w, s, x_seq_last=True, out_seq_last=True).shape == (2, 6, 0)
    x = torch.randn(20, device="cuda")
    assert torch.equal(B.ss_qlinear(x, w, s), B.ss_qlinear(x[None], w, s)[0])
    assert B.ss_qlinear(torch.randn(2, 3, 4, 20, device="cuda"), w, s).shape == (2, 3, 4, 6)


def test_outputs_stay_in_their_memory():
    for io in ("f32", "bf16"):
        for count, features in ((1, 3), (3, 37), (20, 129), (150, 131)):
            pool = torch.full((count * features + 40,), 3.0, dtype=u.TYPES[io], device="cuda")
            w, s = B.ss_quant_rows(torch.randn(features, 100, device="cuda"))
            x = torch.randn(1, count, 100, device="cuda").to(u.TYPES[io])
            for last in (False, True):
                shape = (1, features, count) if last else (1, count, features)
                out = pool[17:17 + count * features].view(shape)
                B.ss_qlinear(x, w, s, out=out, out_seq_last=last)
                assert torch.equal(out, B.ss_qlinear(x, w, s, out_seq_last=last))
                assert (pool[:17] == 3).all() and (pool[17 + count * features:] == 3).all()


def test_scratch_streams_graphs():
    w, s = B.ss_quant_rows(torch.randn(500, 700, device="cuda"))
    for count, last in ((1, False), (3, False), (40, False), (700, True)):
        x = torch.randn(1, count, 700, device="cuda").bfloat16()
        want = B.ss_qlinear(x, w, s, out_seq_last=last)
        scratch = torch.full((max(256, B.ss_qlinear_scratch_bytes(1, count, 700, 500, out_seq_last=last)),), 0xAB, dtype=torch.uint8, device="cuda")
        assert torch.equal(B.ss_qlinear(x, w, s, out_seq_last=last, scratch=scratch), want)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            got = B.ss_qlinear(x, w, s, out_seq_last=last)
        side.synchronize()
        assert torch.equal(got, want)
        out, graph = torch.empty_like(want), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            B.ss_qlinear(x, w, s, out_seq_last=last, out=out, scratch=scratch)
        for _ in range(3):
            x.copy_(torch.randn_like(x))
            want = B.ss_qlinear(x, w, s, out_seq_last=last)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_offsets_past_32_bits():
    free, _ = torch.cuda.mem_get_info()
    if free < 30 << 30:
        pytest.skip("needs 30 GiB")
    count, features = 263000, 8200
    w, s = B.ss_quant_rows(torch.randn(features, 64, device="cuda"))
    x = torch.zeros(count, 64, dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.randn(64, device="cuda").bfloat16()
    out = B.ss_qlinear(x, w, s)
    assert torch.equal(out[-1], B.ss_qlinear(x[-300:], w, s)[-1]) and not out[:-1].any()


def test_refusals():
    w, s = B.ss_quant_rows(torch.randn(6, 20, device="cuda"))
    x = torch.randn(2, 3, 20, device="cuda")
    for bad in (dict(x=x.half()), dict(scale=s.double()), dict(weight=w.float()), dict(out_dtype=torch.bfloat16)):
        with pytest.raises(TypeError):
            B.ss_qlinear(**{**dict(x=x, weight=w, scale=s), **bad})
    for bad in (dict(x=x[..., :10]), dict(scale=s[:3]), dict(weight=w[:, :64]), dict(weight=w[0]), dict(x=x.cpu()), dict(x=x[0], out_seq_last=True),
                dict(x_scale=s), dict(bias=s[:2]), dict(out=torch.empty(2, 3, 5, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            B.ss_qlinear(**{**dict(x=x, weight=w, scale=s), **bad})
    with pytest.raises(B.SsError):
        B.ss_qlinear(x, w, s, scratch=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(B.SsError):
        B.ss_quant_rows(torch.randn(1, 140000, device="cuda"))
