"""RMS norm on the GPU against the float64 oracle, and both norms with their result in 8 bits against the norm followed by the quantiser.

Tolerances in multiples of 2^-24 (op_util.close).  The sum of squares is a tree of W non-negative terms, up to W / 1024 of them one after
another: its relative error is that many roundings and a few for the tree, 1 / sqrt halves it; the result is two products
more: 16 + W / 2048 of |w| rstd max|s| + |b|.  Gradients: rstd (g - xh mean(g xh)), whose second
term is a tree of W products of a size up to max|g| max|xh|: 32 of rstd max|g| (1 + max|xh|^2).  Sums over rows: 32 of the sum of the terms'
magnitudes, and their own errors."""
import numpy as np
import pytest
import torch

from oracle import model_oracle as mo
from paper_2312_00752_amd import autograd as ag
from paper_2312_00752_amd import binding as B
from tests import op_util as u

pytestmark = pytest.mark.gpu
HELD = [("f32", None), ("f32", "f32"), ("bf16", None), ("bf16", "bf16"), ("bf16", "f32")]


def inputs(rows, width, io, residual, weight, bias, scale=1.0, seed=0):
    rng = np.random.default_rng(seed)
    x = u.rounded(scale * rng.standard_normal((rows, width)), io)
    w = (1 + 0.1 * rng.standard_normal(width)).astype(np.float32) if weight else None
    b = rng.standard_normal(width).astype(np.float32) if bias else None
    r = u.rounded(2 * scale * rng.standard_normal((rows, width)), residual) if residual else None
    return rng, x, w, b, r


def on_gpu(w):
    return None if w is None else torch.from_numpy(w).cuda()


def check(rows, width, io, residual=None, weight=True, bias=False, dsummed=True, scale=1.0, eps=1e-5, seed=0):
    rng, x, w, b, r = inputs(rows, width, io, residual, weight, bias, scale, seed)
    tx, tw, tb, tr = u.upload(x, io), on_gpu(w), on_gpu(b), None if r is None else u.upload(r, residual)
    held, s = (residual, u.rounded(x.astype(np.float32) + r.astype(np.float32), residual)) if residual else (io, x)
    out, summed, stats = B.ss_norm_fwd(tx, tw, tb, residual=tr, eps=eps, save_stats=True, rms=True)
    ro, xhat, rstd = mo.rms_fwd(s, w, b, eps)
    if residual:
        assert np.array_equal(u.host(summed), s)
    aw = 1.0 if w is None else np.abs(w).max()
    steps = 16 + width / 2048
    u.close(out, ro, steps, "out", size=aw * rstd * np.abs(s).max(1, keepdims=True) + (0.0 if b is None else np.abs(b).max()))
    assert stats.shape == (rows,)
    u.close(stats, rstd[:, 0], steps, "rstd", size=rstd[:, 0])
    dout = u.rounded(rng.standard_normal((rows, width)), io)
    more = u.rounded(rng.standard_normal((rows, width)), held) if residual and dsummed else None
    g = B.ss_norm_bwd(u.upload(dout, io), summed if residual else tx, stats, tw, has_bias=bias, rms=True,
                      residual_dtype=u.TYPES[held] if residual else None, dsummed=None if more is None else u.upload(more, held), eps=eps)
    ref = mo.rms_bwd(dout, s, w, more, eps)
    gsize = np.abs(dout).max(1, keepdims=True) * aw * rstd * (1 + np.abs(xhat).max(1, keepdims=True) ** 2)
    msize = 0.0 if more is None else np.abs(more)
    u.close(g["dx"], ref["ds"], 32, "dx", size=gsize + msize)
    if residual:
        u.close(g["dresidual"], ref["ds"], 32, "dresidual", size=gsize + msize)
    if weight:
        u.close(g["dweight"], ref["dweight"], 32, "dweight", size=ref["dweight_size"])
    if bias:
        u.close(g["dbias"], ref["dbias"], 32, "dbias", size=ref["dbias_size"])
    assert (g["dweight"] is None) == (not weight) and (g["dbias"] is None) == (not bias)


# widths around a slice, the forms' limits, and rows that no registers hold
@pytest.mark.parametrize("io,residual", HELD)
@pytest.mark.parametrize("width", [1, 3, 8, 9, 127, 128, 129, 511, 513, 1021, 2048, 2050, 4097, 8192, 8200, 16384, 16391, 40001])
def test_widths(width, io, residual):
    check(5, width, io, residual, seed=width)


@pytest.mark.parametrize("width", [64, 100, 1000, 2048])
@pytest.mark.parametrize("rows", [1, 2, 1023, 1024, 4099])
def test_rows(rows, width):
    check(rows, width, "bf16", "f32", seed=rows)
    check(rows, width, "f32", seed=rows)


@pytest.mark.parametrize("weight,bias", [(False, False), (True, True), (False, True)])
def test_optional(weight, bias):
    check(33, 515, "bf16", "bf16", weight=weight, bias=bias)
    check(33, 20001, "f32", weight=weight, bias=bias)
    check(33, 515, "f32", "f32", weight=weight, bias=bias, dsummed=False)


@pytest.mark.parametrize("scale,eps", [(1e-12, 1e-5), (1e-12, 0.0), (1e12, 1e-5)])
def test_sizes_of_values(scale, eps):
    check(9, 700, "f32", scale=scale, eps=eps)
    check(9, 20000, "f32", "f32", scale=scale, eps=eps, dsummed=False)


def test_zeros_infinities_nan():
    x = torch.ones(5, 300, device="cuda")
    x[0] = 0.0
    x[1, 7] = float("inf")
    x[2, 299] = float("nan")
    out = B.ss_norm_fwd(x, rms=True)[0].cpu()
    assert (out[0] == 0).all() and torch.isnan(out[2]).all()
    assert torch.isnan(out[1, 7]) and (out[1, :7] == 0).all() and (out[1, 8:] == 0).all()
    assert torch.allclose(out[3:], torch.ones(2, 300), atol=1e-5)
    q, scale, _ = B.ss_norm_quant(x, rms=True)
    assert scale[0] == 0 and (q[0] == 0).all() and torch.isnan(scale[1:3]).all() and (q[1:3] == 0).all()


# ---- results in 8 bits ------------------------------------------------------------------------------
def check_quant(rows, width, io, residual, rms, weight=True, bias=True, seed=0, scale=1.0):
    _, x, w, b, r = inputs(rows, width, io, residual, weight, bias, scale, seed)
    tx, tw, tb, tr = u.upload(x, io), on_gpu(w), on_gpu(b), None if r is None else u.upload(r, residual)
    out, summed, _ = B.ss_norm_fwd(tx, tw, tb, residual=tr, rms=rms)
    q0, s0 = B.ss_quant_rows(out)
    q, s, held = B.ss_norm_quant(tx, tw, tb, residual=tr, rms=rms)
    assert torch.equal(q, q0) and torch.equal(s, s0)
    assert (held is None) == (residual is None) and (held is None or torch.equal(held, summed))
    # in Python's marshalling, the stream carried on in place
    q, s, held = B.ss_norm_quant(tx, tw, tb, residual=tr, rms=rms, summed=tr)
    assert torch.equal(q, q0) and torch.equal(s, s0) and held is tr and (tr is None or torch.equal(tr, summed))


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("io,residual", HELD)
@pytest.mark.parametrize("width", [1, 8, 9, 120, 128, 129, 513, 1021, 2048, 4097, 8192, 16384, 16391, 40001])
def test_quant_widths(width, io, residual, rms):
    check_quant(5, width, io, residual, rms, seed=width)


@pytest.mark.parametrize("rows", [1, 2, 1023, 1024, 4099])
def test_quant_rows(rows):
    check_quant(rows, 2048, "bf16", "f32", True, bias=False, seed=rows)
    check_quant(rows, 100, "f32", None, False, weight=False, seed=rows)


@pytest.mark.parametrize("rows,width", [(3, 100), (2000, 515), (5, 20001)])
def test_quant_writes_its_rows_alone(rows, width):
    """What lies behind the result, and the padding of its rows."""
    x = torch.randn(rows, width, device="cuda")
    pitch = B.ss_quant_pitch(width)
    room = torch.full((rows + 1, pitch), 77, dtype=torch.int8, device="cuda")
    scale = torch.full((rows + 1,), 5.0, device="cuda")
    p = B.NormQuantParams()
    p.fwd.rows, p.fwd.width, p.fwd.eps, p.fwd.flags, p.fwd.x = rows, width, 1e-5, B.SS_NORM_RMS, x.data_ptr()
    p.q, p.scale = room.data_ptr(), scale.data_ptr()
    import ctypes
    assert B.lib().ss_norm_quant(ctypes.byref(p), torch.cuda.current_stream().cuda_stream) == B.SS_OK
    q, s, _ = B.ss_norm_quant(x, rms=True)
    assert torch.equal(room[:rows], q) and (room[rows] == 77).all() and (room[:rows, width:] == 0).all()
    assert torch.equal(scale[:rows], s) and scale[rows] == 5.0


def test_quant_then_product():
    """As it is used: the 8-bit product takes the result."""
    x = torch.randn(3, 70, 260, device="cuda", dtype=torch.bfloat16)
    w, s = B.ss_quant_rows(torch.randn(96, 260, device="cuda"))
    q, scale, _ = B.ss_norm_quant(x, rms=True)
    got = B.ss_qlinear(q.view(3, 70, -1), w, s, x_scale=scale, dim=260, out_seq_last=True)
    assert torch.equal(got, B.ss_qlinear(B.ss_norm_fwd(x, rms=True)[0], w, s, out_seq_last=True))


# ---- through autograd -------------------------------------------------------------------------------
@pytest.mark.parametrize("io,residual", HELD)
def test_autograd(io, residual):
    rng, x, w, _, r = inputs(37, 301, io, residual, True, False)
    tx, tw = u.upload(x, io).requires_grad_(True), on_gpu(w).requires_grad_(True)
    tr = u.upload(r, residual).requires_grad_(True) if residual else None
    res = ag.rms_norm(tx, tw, residual=tr)
    outs = res if residual else (res,)
    douts = [torch.randn_like(v) for v in outs]
    leaves = [tx, tw] + ([tr] if residual else [])
    grads = torch.autograd.grad(outs, leaves, douts)
    out, summed, stats = B.ss_norm_fwd(tx.detach(), tw.detach(), residual=None if tr is None else tr.detach(), save_stats=True, rms=True)
    g = B.ss_norm_bwd(douts[0], summed if residual else tx.detach(), stats, tw.detach(), residual_dtype=None if tr is None else tr.dtype,
                      dsummed=douts[1] if residual else None, rms=True)
    assert torch.equal(outs[0], out) and torch.equal(grads[0], g["dx"]) and torch.equal(grads[1], g["dweight"])
    if residual:
        assert torch.equal(grads[2], g["dresidual"])
    # the same in Python, where the compiled module does not serve the call
    again = ag._LayerNorm.apply(tx, tw, None, tr, 1e-5, True)
    for a, b in zip(torch.autograd.grad(again if residual else (again,), leaves, douts), grads):
        assert torch.equal(a, b)


def test_gradient_against_differences():
    torch.manual_seed(0)
    x, w = torch.randn(4, 50, device="cuda", requires_grad=True), torch.randn(50, device="cuda", requires_grad=True)
    c = torch.randn(4, 50, device="cuda", dtype=torch.float64)
    loss = lambda a, b: (ag.rms_norm(a, b).double() * c).sum()
    grads = torch.autograd.grad(loss(x, w), (x, w))
    for k, (t, g) in enumerate(zip((x, w), grads)):
        v = torch.randn_like(t)
        at = lambda e: loss(*((t.detach() + e * v) if j == k else q.detach() for j, q in enumerate((x, w)))).item()
        # float32 outputs of a size of 3 summed over 200 terms: 2e-5 of noise over a step of 2e-2; third derivatives of a size of 10 times h^2 / 6
        assert abs((at(1e-2) - at(-1e-2)) / 2e-2 - (g.double() * v.double()).sum().item()) < 2e-2


def test_second_derivative_is_refused():
    x = torch.randn(3, 40, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(ag.rms_norm(x).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="cannot be differentiated again"):
        torch.autograd.grad(g.sum(), x)


def test_captured_and_replayed():
    x, w = torch.randn(40, 2048, device="cuda", dtype=torch.bfloat16), torch.randn(2048, device="cuda")
    B.ss_norm_quant(x, w, rms=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, s, _ = B.ss_norm_quant(x, w, rms=True)
    for k in range(3):
        x.copy_(torch.randn_like(x))
        graph.replay()
        q0, s0, _ = B.ss_norm_quant(x, w, rms=True)
        torch.cuda.synchronize()
        assert torch.equal(q, q0) and torch.equal(s, s0)


def test_other_stream():
    x = torch.randn(4096, 2048, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    q, s, _ = B.ss_norm_quant(x, rms=True, stream=st)
    st.synchronize()
    q0, s0, _ = B.ss_norm_quant(x, rms=True)
    assert torch.equal(q, q0) and torch.equal(s, s0)


def test_refusals():
    x = torch.randn(3, 40, device="cuda")
    with pytest.raises(ValueError):
        B.ss_norm_quant(x, torch.randn(41, device="cuda"))
    with pytest.raises(TypeError):
        B.ss_norm_quant(x.half())
    with pytest.raises(ValueError):
        B.ss_norm_quant(x.t())
    with pytest.raises(ValueError):
        B.ss_norm_quant(x, summed=torch.empty_like(x))
    with pytest.raises(B.SsError):
        B.ss_norm_quant(torch.randn(1, 131073, device="cuda"))
    with pytest.raises(ValueError):   # statistics of the other norm
        B.ss_norm_bwd(x, x, B.ss_norm_fwd(x, save_stats=True)[2], rms=True)
