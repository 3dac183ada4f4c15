"""The gradient functions of the compiled module and those in Python: the same kernels, so the same bits; streams, hooks of torch's
graph, errors."""
import pytest
import torch

from paper_2312_00752_amd import autograd as ag
from paper_2312_00752_amd import binding as B

pytestmark = pytest.mark.gpu


def grads(out, inputs, douts):
    return torch.autograd.grad(out, inputs, douts, allow_unused=True)


def same(a, b):
    for p, q in zip(a, b):
        assert (p is None) == (q is None) and (p is None or torch.equal(p, q))


@pytest.mark.parametrize("io,held", [("f32", None), ("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("weight,bias", [(True, True), (True, False), (False, False)])
def test_norm(io, held, weight, bias):
    types = {"f32": torch.float32, "bf16": torch.bfloat16}
    x = torch.randn(3, 50, 72, device="cuda").to(types[io]).requires_grad_(True)
    r = None if held is None else torch.randn(3, 50, 72, device="cuda").to(types[held]).requires_grad_(True)
    w = torch.randn(72, device="cuda", requires_grad=True) if weight else None
    b = torch.randn(72, device="cuda", requires_grad=True) if bias else None
    inputs = [v for v in (x, w, b, r) if v is not None]
    a = ag.layer_norm(x, w, b, residual=r, eps=1e-4)
    p = ag._LayerNorm.apply(x, w, b, r, 1e-4)
    assert B.layer_norm_node(x, w, b, r, 1e-4) is not None
    a, p = (list(v) if held else [v] for v in (a, p))
    same(a, p)
    d = [torch.randn_like(v) for v in a]
    same(grads(a, inputs, d), grads(p, inputs, d))
    if held:   # one of the two results alone
        for k in range(2):
            a, p = ag.layer_norm(x, w, b, residual=r)[k], ag._LayerNorm.apply(x, w, b, r, 1e-5)[k]
            same(grads([a], inputs, d[k:k + 1]), grads([p], inputs, d[k:k + 1]))


@pytest.mark.parametrize("last", [False, True])
@pytest.mark.parametrize("full", [False, True])
def test_recurrence(full, last):
    wide = torch.randn(2, 40, 33, device="cuda").bfloat16().requires_grad_(True)
    x, f, i, z = wide.chunk(4, 1)   # slices: their gradients meet in one tensor
    rate = torch.rand(10, device="cuda", requires_grad=True)
    h0 = torch.randn(2, 10, device="cuda", requires_grad=True)
    kw = dict(i=i, z=z, f_bias=rate, i_bias=rate, reset=torch.rand(2, 33, device="cuda") < 0.1, h0=h0) if full else {}
    a = ag.gated_recurrence(x, f, rate, return_last_state=last, **kw)
    p = ag._GatedRecurrence.apply(x, f, rate, kw.get("i"), kw.get("z"), kw.get("f_bias"), kw.get("i_bias"), kw.get("reset"), kw.get("h0"), last)
    a, p = (list(v) if last else [v] for v in (a, p))
    same(a, p)
    d = [torch.randn_like(v) for v in a]
    inputs = [wide, rate, h0]
    same(grads(a, inputs, d), grads(p, inputs, d))


def test_no_gradients_wanted():
    x = torch.randn(4, 24, device="cuda")
    out, s = ag.layer_norm(x, residual=x)
    assert not out.requires_grad and torch.equal(s, 2 * x)
    with torch.no_grad():
        y = ag.gated_recurrence(*(torch.randn(1, 4, 24, device="cuda", requires_grad=True) for _ in range(2)), torch.ones(4, device="cuda"))
    assert not y.requires_grad


def test_own_stream():
    """Forward on a side stream; the backward pass follows there."""
    x = torch.randn(64, 2048, device="cuda", requires_grad=True)
    w = torch.randn(2048, device="cuda", requires_grad=True)
    d = torch.randn_like(x)
    want = grads([ag.layer_norm(x, w)], [x, w], [d])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y = x
        for _ in range(20):
            y = y + 0.0
        out = ag.layer_norm(y, w)
        got = grads([out], [x, w], [d])
    s.synchronize()
    same(got, want)


def test_refused_calls():
    x = torch.randn(2, 3, 16, device="cuda", requires_grad=True)
    rate = torch.ones(3, device="cuda")
    for bad in (dict(rate=rate.double()), dict(f=x.bfloat16()), dict(i_bias=rate), dict(h0=torch.zeros(3, 2, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            ag.gated_recurrence(**{**dict(x=x, f=x, rate=rate), **bad})
    with pytest.raises(B.SsError):
        ag.layer_norm(x, eps=-1.0)
    with pytest.raises(TypeError):
        ag.layer_norm(x, residual=x.bfloat16())
    out = ag.layer_norm(x)
    with torch.no_grad():
        x.add_(1.0)
    with pytest.raises(RuntimeError):   # x is needed as it was
        out.sum().backward()


def test_memory_of_a_call_belongs_to_its_stream():
    """A call's own scratch and results on a side stream are not handed out again while it runs: current-stream work that
    allocates and writes at once after each call leaves its results alone."""
    side = torch.cuda.Stream()
    x = torch.randn(1, 700, 1500, device="cuda").bfloat16()
    w, s = B.ss_quant_rows(torch.randn(600, 1500, device="cuda"))
    res = torch.randn(3000, 1100, device="cuda")
    long = torch.randn(1, 8, 60000, device="cuda")
    rate = torch.ones(8, device="cuda")
    _, _, stats = B.ss_norm_fwd(res, save_stats=True)
    wn = torch.ones(1100, device="cuda")
    calls = [lambda st: B.ss_qlinear(x, w, s, out_seq_last=True, stream=st), lambda st: B.ss_gate_fwd(long, long, rate, stream=st)[0],
             lambda st: B.ss_norm_bwd(res, res, stats, wn, stream=st)["dweight"], lambda st: B.ss_norm_fwd(res, stream=st)[0],
             lambda st: B.ss_quant_rows(x, seq_last=True, stream=st)[0]]
    want = [c(None) for c in calls]
    torch.cuda.synchronize()
    for c, ref in zip(calls, want):
        for stream in (side, side.cuda_stream):
            got = []
            for _ in range(5):
                got.append(c(stream))
                for _ in range(4):
                    torch.full((4 << 20,), 7, dtype=torch.uint8, device="cuda")
            torch.cuda.synchronize()
            assert all(torch.equal(g, ref) for g in got)
    assert torch.equal(B.ss_norm_fwd(res, stream=0)[0], want[3])


def test_axes():
    one = torch.tensor(1.0, device="cuda")
    rate = torch.ones(3, device="cuda")
    for call in (lambda: B.ss_norm_fwd(one), lambda: B.ss_quant_rows(one), lambda: B.ss_quant_rows(rate, seq_last=True),
                 lambda: B.ss_gate_fwd(rate, rate, rate), lambda: B.ss_gate_step(one, rate, rate, rate),
                 lambda: B.ss_qlinear(one, *B.ss_quant_rows(torch.ones(2, 3, device="cuda")))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("compiled", [True, False])
def test_gradients_cannot_be_differentiated_again(compiled, monkeypatch):
    """They are computed outside of the graph: a second pass through them is refused, not silently without their part."""
    if not compiled:
        monkeypatch.setattr(B, "_native", B._NoMarshal)
    x, res, f = (torch.randn(2, 8, 40, device="cuda", requires_grad=True) for _ in range(3))
    w, rate = torch.ones(40, device="cuda", requires_grad=True), torch.ones(8, device="cuda", requires_grad=True)
    out, summed = ag.layer_norm(x, w, residual=res)
    for y, inputs in ((out, (x, w, res)), (summed, (x, res)), (ag.gated_recurrence(x, f, rate), (x, f, rate))):
        once = torch.autograd.grad(y.square().sum(), inputs, create_graph=True)
        plain = torch.autograd.grad(y.square().sum(), inputs, retain_graph=True)
        assert all(torch.allclose(a, b) for a, b in zip(once, plain))
        with pytest.raises(RuntimeError):
            sum(g.square().sum() for g in once).backward()
