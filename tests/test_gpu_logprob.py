"""Log probabilities of tokens, entropies, alternatives and their gradient on the GPU against the float64 oracle.

Tolerances in multiples of 2^-24 (op_util.close).  exp(d), d = x - max, is exp2 of a product that is rounded (an absolute error of |d| 2^-24 of the
exponent) and a few units of its own; the sum S has terms of one sign, up to W / 256 of them one after another and then a tree.  So
log S is off by W / 256 + 24 steps of 1 + sum p |d|, which is no more than 1 + log S + entropy's terms; log probabilities add their own roundings of
their terms.  The entropy is log S - U / S, whose terms p d have errors of p d^2 and those of S.  A gradient's p has the errors of exp(d) and 1 / S,
its factor those of the entropy and of log p.  The sizes are the oracle's."""
import numpy as np
import pytest
import torch

from oracle import model_oracle as mo
from paper_2312_00752_amd import autograd as ag
from paper_2312_00752_amd import binding as B
from tests import op_util as u

pytestmark = pytest.mark.gpu


def on_gpu(v):
    return None if v is None else torch.from_numpy(v).cuda()


def compare(x, targets, top, io, dlogp, dentropy, tx=None):
    """x (rows, vocab): values of the type; tx: the tensor that holds them, if it is not dense."""
    vocab = x.shape[1]
    steps = 24 + vocab / 256
    tx = u.upload(x, io) if tx is None else tx
    tt = on_gpu(targets)
    ref = mo.logprob_fwd(x, targets, top)
    logp, entropy, stats, top_logp, top_ids = B.ss_logprob_fwd(tx, tt, top=top)
    if targets is not None:
        u.close(logp, ref["logp"], steps, "logp", size=ref["logp_size"])
    u.close(entropy, ref["entropy"], steps, "entropy", size=ref["entropy_size"])
    if top:
        assert np.array_equal(top_ids.cpu().numpy(), ref["top_ids"])
        u.close(top_logp, ref["top_logp"], steps, "top_logp", size=ref["top_size"])
    g = mo.logprob_bwd(ref, targets, dlogp, dentropy)
    room = torch.full((x.shape[0] + 2, vocab), 7.0, dtype=u.TYPES[io], device="cuda")   # every element is written, and no other
    dx = B.ss_logprob_bwd(tx, stats, tt, dlogp=on_gpu(dlogp), entropy=entropy, dentropy=on_gpu(dentropy), out=room[1:-1])
    assert (room[0] == 7).all() and (room[-1] == 7).all()
    # the hardware's exponential gives 0 below 2^-126, the least normal number, so there (p = e / S <= e, as S >= 1) the whole of the result may be missing
    flushed = np.where(ref["p"] < 2.0 ** -126, np.abs(g["dlogits"]), 0.0)
    u.close(dx, g["dlogits"], steps, "dlogits", size=g["dlogits_size"] + flushed / (steps * u.EPS))
    again = B.ss_logprob_fwd(tx, tt, top=top)
    assert torch.equal(again[1].view(torch.int32), entropy.view(torch.int32)) and (not top or torch.equal(again[4], top_ids))
    return logp, entropy, stats, top_logp, top_ids, dx


def make(rows, vocab, io, seed=0, scale=3.0):
    rng = np.random.default_rng(seed)
    x = u.rounded(scale * rng.standard_normal((rows, vocab)), io)
    return rng, x, rng.integers(0, vocab, rows), (rng.standard_normal(rows)).astype(np.float32), rng.standard_normal(rows).astype(np.float32)


# around a slice, a wave's row, a workgroup's step and pieces
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 64, 257, 511, 512, 513, 2047, 2048, 2049, 2056, 4096, 4099, 8192, 8193, 50021, 131077])
def test_vocabularies(vocab, io):
    rng, x, t, dl, dh = make(5, vocab, io, vocab)
    compare(x, t, min(vocab, 8), io, dl, dh)
    compare(x, t, 0, io, dl, None)
    compare(x, None, min(vocab, 3), io, None, dh)


@pytest.mark.parametrize("rows,vocab", [(1, 300), (3, 300), (4, 300), (1023, 300), (1, 9000), (100, 9000), (1025, 4099), (2047, 2100), (2048, 2100), (2100, 2100)])
def test_rows(rows, vocab):
    rng, x, t, dl, dh = make(rows, vocab, "bf16", rows)
    compare(x, t, 4, "bf16", dl, dh)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("top", [1, 2, 20, 63, 64])
@pytest.mark.parametrize("vocab", [64, 100, 2048, 3000, 20000])
def test_top(top, vocab, io):
    rng, x, t, dl, dh = make(6, vocab, io, top)
    # rows whose best come late, early, all equal, and equal in groups; the rows of bf16 have ties by themselves
    x[0], x[1] = np.sort(x[0]), np.sort(x[1])[::-1]
    x[2] = 1.5
    x[3] = rng.integers(0, 3, vocab)
    x[4] = np.where(np.arange(vocab) % 64 == 5, 9.0, x[4])   # all in few lanes
    compare(x, t, top, io, dl, dh)


def test_top_of_zeros_of_both_signs():
    x = np.zeros((2, 3000), np.float32)
    x[0, ::2] = -0.0
    x[1, 1::2] = -0.0
    assert (B.ss_logprob_fwd(on_gpu(x), top=5)[4].cpu() == torch.arange(5)).all()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 5000, 50021])
def test_masked(vocab, io):
    """Logits of -infinity, up to all of them but one and all of them; targets that are masked; the type's lowest value."""
    rng, x, t, dl, dh = make(9, vocab, io, vocab)
    low = float(torch.finfo(u.TYPES[io]).min)
    x[0, rng.uniform(size=vocab) < 0.5] = -np.inf
    x[1, np.arange(vocab) != 17] = -np.inf
    x[2] = -np.inf
    x[3, : vocab // 2] = -np.inf
    x[4, vocab // 3:] = -np.inf
    x[5, np.arange(vocab) != 9] = low
    x[6] = low
    x[7, ::2] = low
    t[1], t[3] = 17, vocab - 1
    *_, dx = compare(x, t, 6, io, dl, dh)
    assert (dx[2] == 0).all() and (dx[1] == 0).all()
    t[0], t[1], t[3], t[5] = int(np.argmax(np.isinf(x[0]))), 18, 0, 8   # tokens that cannot be
    compare(x, t, 6, io, dl, None)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 5000])
def test_infinity_and_nan(vocab, io):
    rng, x, t, dl, dh = make(6, vocab, io, vocab)
    x[0, 5], x[1, vocab - 1], x[2], x[3, 3:] = np.nan, np.inf, np.nan, np.nan
    x[4, 0], x[4, 2] = -np.inf, np.nan
    logp, entropy, stats, top_logp, top_ids, dx = compare(x, t, 8, io, dl, dh)
    assert torch.isnan(logp[:5]).all() and torch.isnan(entropy[:5]).all() and torch.isnan(dx[:5]).all()
    t[:] = -1
    dh[:] = 0.0
    *_, dx = compare(x, t, 0, io, dl, dh)   # nothing is asked for: no gradient, whatever the rows hold
    assert (dx == 0).all()


@pytest.mark.parametrize("id_type", [torch.int32, torch.int64])
def test_targets_outside(id_type):
    rng, x, t, dl, dh = make(8, 700, "f32")
    t[[0, 2, 4, 6]] = [-1, 700, 2 ** 31 - 1, -2 ** 31]
    tx, tt = on_gpu(x.astype(np.float32)), on_gpu(t).to(id_type)
    logp, entropy, stats, _, _ = B.ss_logprob_fwd(tx, tt)
    ref = mo.logprob_fwd(x, t)
    u.close(logp, ref["logp"], 30, "logp", size=ref["logp_size"])
    assert (logp[::2] == 0).all()
    dl[[0, 2]] = np.nan   # what stands at tokens that are not asked for does not matter
    dx = B.ss_logprob_bwd(tx, stats, tt, dlogp=on_gpu(dl))
    u.close(dx, mo.logprob_bwd(ref, t, dl)["dlogits"], 30, "dlogits", size=mo.logprob_bwd(ref, t, dl)["dlogits_size"])
    if id_type is torch.int64:   # not cut to 32 bits
        assert (B.ss_logprob_fwd(tx, tt + 2 ** 32)[0] == 0).all()


@pytest.mark.parametrize("scale", [1e-6, 1e3, 1e30])
def test_sizes_of_values(scale):
    rng, x, t, dl, dh = make(4, 3000, "f32", scale=scale)
    compare(x, t, 5, "f32", dl, dh)
    compare(u.rounded(x + 1e4, "f32"), t, 5, "f32", dl, dh)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,pad", [(7, 1), (300, 27), (5000, 8), (50021, 27)])
def test_slice_of_a_padded_vocabulary(vocab, pad, io):
    """What stands in the padding does not matter, and stays."""
    rng, x, t, dl, dh = make(5, vocab, io, vocab)
    wide = torch.full((5, vocab + pad), float("nan"), dtype=u.TYPES[io], device="cuda")
    wide[:, :vocab] = u.upload(x, io)
    compare(x, t, min(vocab, 5), io, dl, dh, tx=wide[:, :vocab])
    assert torch.isnan(wide[:, vocab:]).all()


def test_axes_and_strides():
    x = torch.randn(2, 3, 4, 50, device="cuda")
    t = torch.randint(0, 50, (2, 3, 4), device="cuda")
    logp, entropy, stats, top_logp, top_ids = B.ss_logprob_fwd(x, t, top=3)
    assert logp.shape == (2, 3, 4) and top_ids.shape == (2, 3, 4, 3) and stats.shape == (2, 24)
    flat = B.ss_logprob_fwd(x.view(24, 50), t.view(24), top=3)
    assert torch.equal(flat[0].view(2, 3, 4), logp) and torch.equal(flat[4].view(2, 3, 4, 3), top_ids)
    one = B.ss_logprob_fwd(x[0, 0, 0], t[0, 0, 0])
    assert one[0].shape == () and one[0] == logp[0, 0, 0]
    every_other = x[:, :, ::2]   # rows equally far from each other, but not over both axes
    with pytest.raises(ValueError):
        B.ss_logprob_fwd(x[:, :2], t[:, :2].contiguous())
    assert torch.equal(B.ss_logprob_fwd(every_other, t[:, :, ::2].contiguous())[0], logp[:, :, ::2])
    with pytest.raises(ValueError):
        B.ss_logprob_fwd(x.transpose(2, 3), t)
    with pytest.raises(ValueError):
        B.ss_logprob_fwd(torch.randn(60, device="cuda").as_strided((11, 50), (1, 1)), None)
    assert B.ss_logprob_fwd(x[:0], t[:0])[0].shape == (0, 3, 4)
    assert B.ss_logprob_bwd(x[:0], torch.empty(2, 0, device="cuda"), t[:0]).shape == (0, 3, 4, 50)
    same = torch.randn(50, device="cuda")   # the same row, broadcast
    with pytest.raises(ValueError):
        B.ss_logprob_fwd(same.expand(4, 50))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 5001])
def test_autograd(vocab, io):
    rng, x, t, dl, dh = make(12, vocab, io)
    t[3] = -1
    tx, tt = u.upload(x, io).view(3, 4, vocab).requires_grad_(True), on_gpu(t).view(3, 4)
    tdl, tdh = on_gpu(dl).view(3, 4), on_gpu(dh).view(3, 4)
    logp, entropy, stats, top_logp, top_ids = B.ss_logprob_fwd(tx.detach(), tt, top=4)
    got = ag.token_logprobs(tx, tt, top=4)
    assert all(torch.equal(a, b) for a, b in zip(got, (logp, entropy, top_logp, top_ids))) and not got[2].requires_grad
    want = B.ss_logprob_bwd(tx.detach(), stats, tt, dlogp=tdl, entropy=entropy, dentropy=tdh)
    assert torch.equal(torch.autograd.grad(got[:2], tx, [tdl, tdh])[0], want)
    # one of the two alone; a gradient that is the same for all
    logp, entropy = ag.token_logprobs(tx, tt)
    assert torch.equal(torch.autograd.grad(logp, tx, tdl, retain_graph=True)[0], B.ss_logprob_bwd(tx.detach(), stats, tt, dlogp=tdl))
    assert torch.equal(torch.autograd.grad(entropy, tx, tdh, retain_graph=True)[0],
                       B.ss_logprob_bwd(tx.detach(), stats, tt, entropy=entropy.detach(), dentropy=tdh))
    logp.sum().backward()
    assert torch.equal(tx.grad, B.ss_logprob_bwd(tx.detach(), stats, tt, dlogp=torch.ones(3, 4, device="cuda")))


def test_the_same_in_python(monkeypatch):
    """Where the compiled module does not serve the call."""
    wide = torch.randn(3, 4, 303, device="cuda")
    x, t = wide[..., :300].requires_grad_(True), torch.randint(-1, 300, (3, 4), device="cuda")
    douts = [torch.randn(3, 4, device="cuda") for _ in range(2)]
    def go():
        res = ag.token_logprobs(x, t, top=5)
        return [v.detach() for v in res] + list(torch.autograd.grad(res[:2], x, douts)), list(B.ss_logprob_fwd(x.detach(), t, top=5)), res[0].grad_fn.name()
    a = go()
    monkeypatch.setattr(B, "_native", B._NoMarshal)
    b = go()
    assert a[2] != b[2] and all(torch.equal(v, w) for k in (0, 1) for v, w in zip(a[k], b[k]))
    test_axes_and_strides()
    test_second_derivative_is_refused()
    test_refusals()


def test_against_cross_entropy():
    x = torch.randn(40, 900, device="cuda", requires_grad=True)
    t = torch.randint(0, 900, (40,), device="cuda")
    t[::3] = -1
    mine, theirs = -ag.token_logprobs(x, t)[0].sum(), torch.nn.functional.cross_entropy(x.double(), t, ignore_index=-1, reduction="sum")
    assert abs(mine.item() - theirs.item()) < 1e-3
    a, b = torch.autograd.grad(mine, x)[0], torch.autograd.grad(theirs, x)[0]
    assert (a - b).abs().max() < 1e-5


def test_gradient_against_differences():
    torch.manual_seed(0)
    x, t = torch.randn(3, 60, device="cuda", requires_grad=True), torch.tensor([5, 59, -1], device="cuda")
    c = torch.randn(2, 3, device="cuda", dtype=torch.float64)
    def loss(v):
        logp, entropy = ag.token_logprobs(v, t)
        return (c[0] * logp.double()).sum() + (c[1] * entropy.double()).sum()
    g, = torch.autograd.grad(loss(x), x)
    v = torch.randn_like(x)
    at = lambda e: loss(x.detach() + e * v).item()
    # values of a size of 4 with 2^-22 of noise each, over a step of 2e-2: 3e-4; third derivatives times h^2 / 6: 1e-3
    assert abs((at(1e-2) - at(-1e-2)) / 2e-2 - (g.double() * v.double()).sum().item()) < 5e-3


def test_second_derivative_is_refused():
    x = torch.randn(3, 60, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(ag.token_logprobs(x, torch.tensor([1, 2, 3], device="cuda"))[0].sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="cannot be differentiated again"):
        torch.autograd.grad(g.sum(), x)


def test_captured_and_replayed():
    x, t = torch.randn(30, 20000, device="cuda"), torch.randint(0, 20000, (30,), device="cuda")
    dl = torch.randn(30, device="cuda")
    B.ss_logprob_fwd(x, t, top=5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logp, entropy, stats, top_logp, top_ids = B.ss_logprob_fwd(x, t, top=5)
        dx = B.ss_logprob_bwd(x, stats, t, dlogp=dl)
    for k in range(4):
        x.copy_(torch.randn_like(x))
        t.copy_(torch.randint(-1, 20000, (30,), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = B.ss_logprob_fwd(x, t, top=5)
        for a, b in zip((logp, entropy, stats, top_logp, top_ids), want):
            assert torch.equal(a, b)
        assert torch.equal(dx, B.ss_logprob_bwd(x, want[2], t, dlogp=dl))


def test_two_streams_at_once():
    x, t = torch.randn(100, 50000, device="cuda"), torch.randint(0, 50000, (100,), device="cuda")
    want = B.ss_logprob_fwd(x, t, top=7)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [B.ss_logprob_fwd(x, t, top=7, stream=s) for _ in range(3) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))


def test_offsets_beyond_32_bits():
    """2^31 logits and some: the last rows."""
    rows, vocab = 33000, 65552
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.randn(vocab, device="cuda").bfloat16()
    t = torch.full((rows,), vocab - 1, device="cuda")
    logp, entropy, stats, _, ids = B.ss_logprob_fwd(x, t, top=2)
    last = B.ss_logprob_fwd(x[-1:].clone(), t[-1:], top=2)
    assert abs(logp[-1] - last[0][0]) < 1e-4 and abs(entropy[-1] - last[1][0]) < 1e-4 and torch.equal(ids[-1], last[4][0])
    assert (ids[:-1] == torch.arange(2, device="cuda")).all() and (logp[:-1] + np.log(vocab)).abs().max() < 1e-4
    dl = torch.zeros(rows, device="cuda")
    dl[-1] = 1.0
    dx = B.ss_logprob_bwd(x, stats, t, dlogp=dl)
    want = B.ss_logprob_bwd(x[-1:].clone(), stats[:, -1:].contiguous(), t[-1:], dlogp=dl[-1:])
    assert torch.equal(dx[-1], want[0]) and not dx[:-1].view(torch.int16).any()
    del x, dx
    torch.cuda.empty_cache()


def test_refusals():
    x, t = torch.randn(3, 60, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    logp, entropy, stats, _, _ = B.ss_logprob_fwd(x, t)
    for bad in (61, 65, -1):
        with pytest.raises((ValueError, B.SsError)):
            B.ss_logprob_fwd(x, t, top=bad)
    with pytest.raises(TypeError):
        B.ss_logprob_fwd(x.half(), t)
    with pytest.raises(TypeError):
        B.ss_logprob_fwd(x, t.float())
    with pytest.raises(ValueError):
        B.ss_logprob_fwd(x, t[:2])
    with pytest.raises(ValueError):
        B.ss_logprob_fwd(x.cpu(), t)
    with pytest.raises(ValueError):
        B.ss_logprob_bwd(x, stats, t, dlogp=logp, dentropy=logp)
    with pytest.raises(ValueError):
        B.ss_logprob_bwd(x, stats[:, :2], t, dlogp=logp)
    with pytest.raises(ValueError):
        B.ss_logprob_bwd(x, stats, t, dlogp=logp, out=x)
    with pytest.raises(ValueError):
        B.ss_logprob_fwd(torch.randn(3, 0, device="cuda"), t)
    with pytest.raises(B.SsError):
        B.ss_logprob_fwd(torch.randn(3, 60000, device="cuda"), t, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_longest_row():
    """The largest vocabulary that is served, whose last piece ends where 32 bits do: zeros but for two logits, so that every sum is known."""
    vocab = 2 ** 31 - 1 - 65536
    x = torch.zeros(1, vocab, dtype=torch.bfloat16, device="cuda")
    x[0, vocab - 3], x[0, 5] = 20.0, 18.0
    t = torch.tensor([vocab - 3], device="cuda")
    logp, entropy, stats, top_logp, top_ids = B.ss_logprob_fwd(x, t, top=3)
    total = np.exp(20.0) + np.exp(18.0) + (vocab - 2)
    ref = [20 - np.log(total), 18 - np.log(total), -np.log(total)]
    assert top_ids.tolist() == [[vocab - 3, 5, 0]]
    # a lane's 2^13 ones and the pieces' sums are short: the bound of the shorter rows
    assert np.abs(top_logp.cpu().numpy()[0] - ref).max() <= 64 * 2.0 ** -24 * 44 and logp.item() == top_logp[0, 0].item()
    p = np.exp(ref)
    assert abs(entropy.item() + (p[0] * ref[0] + p[1] * ref[1] + (vocab - 2) * p[2] * ref[2])) <= 64 * 2.0 ** -24 * 200
    grad = B.ss_logprob_bwd(x, stats, t, dlogp=torch.ones(1, device="cuda"))
    for k, want in ((5, -p[1]), (vocab - 3, 1 - p[0]), (0, -p[2]), (vocab - 1, -p[2]), (vocab // 2, -p[2])):
        assert abs(grad[0, k].item() - want) <= (2.0 ** -9 + 64 * 44 * 2.0 ** -24) * abs(want)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_masked_target(io):
    """A target that the mask rules out: -infinity, and the gradient of the formula."""
    for vocab in (300, 9001):
        rng, x, t, dl, dh = make(4, vocab, io, vocab)
        x[np.arange(4), t] = -np.inf
        compare(x, t, 3, io, dl, dh)
