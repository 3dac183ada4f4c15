"""Embedding and its gradient on the GPU against the float64 oracle.

Tolerances in multiples of 2^-24 (op_util.close).  A row of the result is one product: 1 of its own size.  A row of the gradient is a
sum in pieces of at least 8 tokens and 8 more (of more where there are more than 4096 pieces) whose sums are added, a quarter of them one after another: every
term passes at most piece + 8 + pieces additions and one product, so its error is at most that many roundings of the sum of magnitudes; random signs take the
square root of them, times 8."""
import numpy as np
import pytest
import torch

from oracle import model_oracle as mo
from paper_2312_00752_amd import autograd as ag
from paper_2312_00752_amd import binding as B
from tests import op_util as u

pytestmark = pytest.mark.gpu
TYPES = [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")]   # of the table, of the result


def zipf(rng, vocab, n):
    return np.minimum(np.exp(rng.uniform(0, np.log(vocab + 1), n)).astype(np.int64) - 1, vocab - 1)


def steps(n):
    piece = 8
    while (n + piece - 1) // piece > 4096:
        piece *= 2
    return 8 * np.sqrt(min(n, piece + 8) + n / piece) + 2


def check(ids, vocab, dim, table, io, scale=1.0, seed=0, id_type=torch.int64):
    rng = np.random.default_rng(seed)
    w = u.rounded(rng.standard_normal((vocab, dim)), table)
    dout = u.rounded(rng.standard_normal(ids.shape + (dim,)), io)
    scale = float(np.float32(scale))
    ti = torch.from_numpy(ids).cuda().to(id_type)
    out = B.ss_embed_fwd(ti, u.upload(w, table), scale=scale, out_dtype=u.TYPES[io])
    ref = mo.embed_fwd(ids, w, scale)
    u.close(out, ref, 1, "out", size=np.abs(ref))
    room = torch.full((vocab + 2, dim), float("nan"), dtype=u.TYPES[table], device="cuda")   # every element is written, and no other
    grad = B.ss_embed_bwd(u.upload(dout, io), ti, vocab, scale=scale, dtype=u.TYPES[table], out=room[1:-1])
    assert torch.isnan(room[0]).all() and torch.isnan(room[-1]).all()
    g = mo.embed_bwd(dout, ids, vocab, scale)
    u.close(grad, g["dtable"], steps(ids.size), "dtable", size=g["dtable_size"])
    assert torch.equal(grad, B.ss_embed_bwd(u.upload(dout, io), ti, vocab, scale=scale, dtype=u.TYPES[table]))


@pytest.mark.parametrize("table,io", TYPES)
@pytest.mark.parametrize("dim", [1, 3, 7, 8, 9, 64, 65, 127, 512, 513, 1021, 2048, 2056, 4099])
def test_widths(dim, table, io):
    rng = np.random.default_rng(dim)
    check(zipf(rng, 50, 150), 50, dim, table, io, scale=1.7)


# around a wave, a tile, several tiles and pieces
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 255, 257, 1023, 1024, 1025, 2049, 5199])
def test_tokens(n):
    rng = np.random.default_rng(n)
    check(zipf(rng, 300, n), 300, 24, "f32", "bf16")
    check(rng.integers(0, 70000, n), 70000, 8, "f32", "f32")


# ids of one to three digits
@pytest.mark.parametrize("vocab", [1, 2, 3, 255, 256, 257, 511, 512, 513, 65535, 65536, 262143, 262144, 300001])
def test_vocabularies(vocab):
    rng = np.random.default_rng(vocab)
    check(rng.integers(0, vocab, 3000), vocab, 5, "f32", "f32")
    check(zipf(rng, vocab, 2000), vocab, 8, "bf16", "bf16")


@pytest.mark.parametrize("n", [1, 7, 8, 9, 16, 17, 32, 64, 65, 512, 520, 521, 528, 3000])
def test_one_id_has_all_tokens(n):
    check(np.full(n, 3), 7, 33, "f32", "f32", seed=n)


def test_neighbouring_ids_share_pieces():
    """Runs that end at, before and behind the end of a piece, over one and several pieces."""
    runs = [1, 31, 32, 33, 63, 1, 64, 96, 31, 200, 5, 27, 32, 32, 7, 8, 9, 1, 7, 8, 16, 17, 15, 23, 3, 600, 520, 511]
    ids = np.repeat(np.arange(len(runs)), runs)
    check(ids, len(runs), 16, "f32", "f32")
    check(np.random.default_rng(0).permutation(ids), len(runs), 2050, "f32", "bf16")


# 2048 pieces at 512 columns, 512 at 2048 and more: of 8 tokens up to there, then of 16 and 32
@pytest.mark.parametrize("n,dim", [(16384, 16), (16385, 16), (40000, 8), (4096, 2056), (4097, 2056), (9000, 1537)])
def test_longer_pieces(n, dim):
    rng = np.random.default_rng(n)
    lengths = []
    while sum(lengths) < n:   # runs around the pieces' lengths, and some over many pieces
        lengths.append(int(rng.choice([1, 7, 8, 9, 15, 16, 17, 31, 32, 33, 40, 41, 64, 200, 3000])))
    ids = np.repeat(np.arange(len(lengths)), lengths)[:n]
    check(ids, len(lengths), dim, "f32", "f32", seed=n)
    check(rng.permutation(ids), len(lengths), dim, "bf16", "bf16", seed=n)
    check(np.full(n, 1), 3, dim, "f32", "bf16", seed=n)


@pytest.mark.parametrize("id_type", [torch.int32, torch.int64])
def test_padding(id_type):
    rng = np.random.default_rng(1)
    ids = zipf(rng, 40, 500).reshape(5, 100)
    ids[rng.uniform(size=ids.shape) < 0.3] = -1
    ids[0, 0], ids[1, 1], ids[2, 2] = 40, 2 ** 31 - 1, -2 ** 31
    check(ids, 40, 72, "f32", "bf16", id_type=id_type)
    check(np.full(300, -1), 40, 72, "f32", "f32", id_type=id_type)
    check(np.arange(40, 90), 40, 8, "f32", "f32", id_type=id_type)
    if id_type is torch.int64:   # not cut to 32 bits
        check(np.array([2 ** 32 + 1, 2, -2 ** 32, 2 ** 62]), 40, 8, "f32", "f32")


def test_padding_holds_anything():
    ids = torch.tensor([1, -1, 2, 99, 1], device="cuda")
    dout = torch.ones(5, 16, device="cuda")
    dout[1], dout[3] = float("nan"), float("inf")
    grad = B.ss_embed_bwd(dout, ids, 4)
    assert grad.cpu().tolist() == [[0.0] * 16, [2.0] * 16, [1.0] * 16, [0.0] * 16]


def test_infinities_and_nan_stay_in_their_rows():
    ids = torch.tensor([0, 1, 2, 1] * 40, device="cuda")
    dout = torch.ones(160, 24, device="cuda")
    dout[1, 3], dout[2, 5] = float("nan"), float("inf")
    grad = B.ss_embed_bwd(dout, ids, 4).cpu()
    assert torch.isnan(grad[1, 3]) and grad[2, 5] == float("inf")
    grad[1, 3], grad[2, 5] = 80.0, 40.0
    assert grad.tolist() == [[40.0] * 24, [80.0] * 24, [40.0] * 24, [0.0] * 24]


def test_no_tokens():
    ids = torch.empty(0, 3, dtype=torch.int64, device="cuda")
    assert B.ss_embed_fwd(ids, torch.randn(5, 7, device="cuda")).shape == (0, 3, 7)
    out = torch.full((5, 7), 3.0, device="cuda")
    assert (B.ss_embed_bwd(torch.empty(0, 3, 7, device="cuda"), ids, 5, out=out) == 0).all()


def test_many_tokens_in_order():
    """More pieces than 32 tokens each would allow; whole numbers, so that sums are exact and their order does not matter, and the tokens of an
    id told apart by a digit each."""
    n, vocab = 300000, 1000
    g = torch.Generator(device="cuda").manual_seed(0)
    ids = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    ids[: n // 2] = 17
    dout = torch.randint(-8, 9, (n, 12), generator=g, device="cuda").float()
    ref = torch.zeros(vocab, 12, dtype=torch.float64, device="cuda").index_add_(0, ids, dout.double())
    assert torch.equal(B.ss_embed_bwd(dout, ids, vocab).double(), ref)


def test_offsets_beyond_32_bits():
    """A gradient of 2^31 elements and some."""
    vocab, dim = 262147, 8200
    ids = torch.tensor([0, vocab - 1, 262000, vocab - 1], device="cuda")
    dout = torch.randn(4, dim, device="cuda", dtype=torch.bfloat16)
    grad = B.ss_embed_bwd(dout, ids, vocab)
    assert torch.equal(grad[0], dout[0]) and torch.equal(grad[262000], dout[2])
    assert torch.equal(grad[-1], (dout[1].float() + dout[3].float()).bfloat16())
    out = B.ss_embed_fwd(ids, grad)
    assert torch.equal(out[1], grad[-1]) and torch.equal(out[2], grad[262000])
    grad[[0, 262000, vocab - 1]] = 0
    assert not grad.view(torch.int16).any()
    del grad
    torch.cuda.empty_cache()


def test_unaligned_memory():
    for io in (torch.float32, torch.bfloat16):
        table = torch.randn(20 * 40 + 1, device="cuda").to(io)[1:].view(20, 40)
        ids = torch.randint(0, 20, (91,), device="cuda")[1:]
        dout = torch.randn(90 * 40 + 1, device="cuda").to(io)[1:].view(90, 40)
        assert torch.equal(B.ss_embed_fwd(ids, table), table[ids])
        room = torch.full((20 * 40 + 3,), 9.0, device="cuda", dtype=io)
        grad = B.ss_embed_bwd(dout, ids, 20, out=room[1:-2].view(20, 40))
        assert torch.equal(grad, B.ss_embed_bwd(dout.clone(), ids.clone(), 20)) and room[0] == 9 and (room[-2:] == 9).all()


@pytest.mark.parametrize("table,io", TYPES)
def test_autograd(table, io):
    ids = torch.randint(-1, 30, (3, 50), device="cuda")
    w = torch.randn(30, 65, device="cuda").to(u.TYPES[table]).requires_grad_(True)
    out = ag.embedding(ids, w, scale=3.0, out_dtype=u.TYPES[io])
    assert out.dtype == u.TYPES[io] and torch.equal(out.detach(), B.ss_embed_fwd(ids, w.detach(), scale=3.0, out_dtype=u.TYPES[io]))
    dout = torch.randn_like(out)
    g, = torch.autograd.grad(out, w, dout)
    assert g.dtype == w.dtype and torch.equal(g, B.ss_embed_bwd(dout, ids, 30, scale=3.0, dtype=w.dtype))
    # a gradient whose rows do not lie beside each other; one that is the same for all
    out = ag.embedding(ids, w, out_dtype=u.TYPES[io])
    out.transpose(0, 1).sum().backward()
    assert torch.equal(w.grad, B.ss_embed_bwd(torch.ones_like(out), ids, 30, dtype=w.dtype))


def test_the_same_in_python(monkeypatch):
    """Where the compiled module does not serve the call."""
    ids, w = torch.randint(-1, 30, (3, 50), device="cuda"), torch.randn(30, 65, device="cuda", requires_grad=True)
    out = ag.embedding(ids, w, scale=3.0, out_dtype=torch.bfloat16)
    dout = torch.randn_like(out)
    g, = torch.autograd.grad(out, w, dout)
    one = B.ss_embed_fwd(ids, w.detach(), scale=3.0, out_dtype=torch.bfloat16)
    monkeypatch.setattr(B, "_native", B._NoMarshal)
    again = ag.embedding(ids, w, scale=3.0, out_dtype=torch.bfloat16)
    assert again.grad_fn.name() != out.grad_fn.name()
    assert torch.equal(again, out) and torch.equal(one, out) and torch.equal(torch.autograd.grad(again, w, dout)[0], g)
    assert torch.equal(B.ss_embed_fwd(ids, w.detach(), scale=3.0, out_dtype=torch.bfloat16), one)
    test_second_derivative_is_refused()
    test_refusals()


def test_gradient_against_differences():
    torch.manual_seed(1)
    ids = torch.randint(0, 6, (40,), device="cuda")
    w = torch.randn(6, 9, device="cuda", requires_grad=True)
    c = torch.randn(40, 9, device="cuda", dtype=torch.float64)
    loss = lambda t: (ag.embedding(ids, t, scale=0.5).double() * c).sum()
    g, = torch.autograd.grad(loss(w), w)
    v = torch.randn_like(w)
    # linear: 360 terms of a rounding of 2^-24 over a step of 1/4
    assert abs((loss(w.detach() + v / 8) - loss(w.detach() - v / 8)) * 4 - (g.double() * v.double()).sum()) < 360 * 4 * 4 * 2.0 ** -24 * 10


def test_second_derivative_is_refused():
    w = torch.randn(6, 9, device="cuda", requires_grad=True)
    dout = torch.randn(4, 9, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(ag.embedding(torch.arange(4, device="cuda"), w), w, dout, create_graph=True)
    with pytest.raises(RuntimeError, match="cannot be differentiated again"):
        torch.autograd.grad(g.sum(), dout)


def test_captured_and_replayed():
    ids, w = torch.randint(0, 100, (3000,), device="cuda"), torch.randn(100, 64, device="cuda")
    dout = torch.randn(3000, 64, device="cuda")
    B.ss_embed_bwd(dout, ids, 100)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, grad = B.ss_embed_fwd(ids, w), B.ss_embed_bwd(dout, ids, 100)
    for k in range(4):
        ids.copy_(torch.randint(-1, 100, (3000,), device="cuda"))
        dout.copy_(torch.randn_like(dout))
        grad.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(grad, B.ss_embed_bwd(dout, ids, 100)) and torch.equal(out, B.ss_embed_fwd(ids, w))


def test_two_streams_at_once():
    ids, dout = torch.randint(0, 5000, (20000,), device="cuda"), torch.randn(20000, 256, device="cuda")
    want = B.ss_embed_bwd(dout, ids, 5000)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [B.ss_embed_bwd(dout, ids, 5000, stream=s) for _ in range(3) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_refusals():
    ids, w = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.randn(5, 6, device="cuda")
    with pytest.raises(TypeError):
        B.ss_embed_fwd(ids.float(), w)
    with pytest.raises(TypeError):
        B.ss_embed_fwd(ids, w.half())
    with pytest.raises(TypeError):
        B.ss_embed_fwd(ids, w, out_dtype=torch.float16)
    with pytest.raises(ValueError):
        B.ss_embed_fwd(ids, w.t())
    with pytest.raises(ValueError):
        B.ss_embed_fwd(ids.cpu(), w)
    with pytest.raises(ValueError):
        B.ss_embed_fwd(ids, w[0])
    with pytest.raises(ValueError):
        B.ss_embed_bwd(torch.randn(3, 6, device="cuda"), ids, 5)
    with pytest.raises(B.SsError):
        B.ss_embed_bwd(torch.randn(4, 6, device="cuda"), ids, 0)
    with pytest.raises(B.SsError):
        B.ss_embed_bwd(torch.randn(4, 6, device="cuda"), ids, 5, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))


def test_refuses_shared_memory():
    room = torch.zeros(64, 8, device="cuda")
    ids = torch.zeros(32, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError, match="table"):
        B.ss_embed_fwd(ids, room[:40], out=room[32:])
    with pytest.raises(ValueError, match="dout"):
        B.ss_embed_bwd(room[:32], ids, 40, out=room[24:])
    with pytest.raises(ValueError, match="ids"):
        B.ss_embed_bwd(room[:32], room[40:48].view(torch.int64).view(-1), 20, out=room[44:])
    B.ss_embed_bwd(room[:32], ids, 32, out=room[32:])
