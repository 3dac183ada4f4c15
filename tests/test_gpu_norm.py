"""Layer norm on the GPU against the float64 oracle.

Tolerances in multiples of 2^-24 (op_util.close): an output is a difference from the mean (the sum of W terms held in a
tree: a few roundings of the largest |s|), a product with rstd (relative error of the variance: a few roundings) and with the weight:
32 of |w| rstd max|s - mean| + |b| + |w| rstd |mean|.  Gradients: 64 of rstd times the largest |g| and its two means.  Sums
over rows: 32 of the sum of the terms' magnitudes and its terms' own errors."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2312_00752_amd import autograd as ag
from paper_2312_00752_amd import binding as B
from tests import op_util as u

pytestmark = pytest.mark.gpu


def check(rows, width, io, residual=None, weight=True, bias=True, dsummed=True, offset=0.0, scale=1.0, eps=1e-5, seed=0, place=None):
    rng = np.random.default_rng(seed)
    x = u.rounded(scale * rng.standard_normal((rows, width)) + offset, io)
    w = (1 + 0.1 * rng.standard_normal(width)).astype(np.float32) if weight else None
    b = rng.standard_normal(width).astype(np.float32) if bias else None
    tx, tw, tb = u.upload(x, io), None if w is None else torch.from_numpy(w).cuda(), None if b is None else torch.from_numpy(b).cuda()
    held, s, tr = io, x, None
    if residual:
        held = residual
        r = u.rounded(2 * scale * rng.standard_normal((rows, width)), held)
        tr = u.upload(r, held)
        s = u.rounded((x.astype(np.float32) + r.astype(np.float32)), held)
    out, summed, stats = B.ss_norm_fwd(tx, tw, tb, residual=tr, eps=eps, save_stats=True, summed=tr if place else None)
    ro, xhat, rstd = bo.norm_fwd(s, w, b, eps)
    if residual:
        assert np.array_equal(u.host(summed), s)
    aw = 1.0 if w is None else np.abs(w).max()
    size = aw * rstd * np.abs(s).max(1, keepdims=True) + (0.0 if b is None else np.abs(b).max())
    u.close(out, ro, 32, "out", size=size)
    u.close(stats[0], s.mean(1), 16, "mean", size=np.abs(s).max(1))
    # the variance's own error: 16 roundings, and those of s - mean where the mean is large
    u.close(stats[1], rstd[:, 0], 16, "rstd", size=rstd[:, 0] * (1 + np.abs(s).max(1) * rstd[:, 0]))
    plain = B.ss_norm_fwd(tx, tw, tb, residual=None if tr is None else (u.upload(r, held)), eps=eps)
    assert torch.equal(plain[0], out) and plain[2] is None
    dout = u.rounded(rng.standard_normal((rows, width)), io)
    more = u.rounded(rng.standard_normal((rows, width)), held) if residual and dsummed else None
    g = B.ss_norm_bwd(u.upload(dout, io), summed if residual else tx, stats, tw, has_bias=bias,
                      residual_dtype=u.TYPES[held] if residual else None, dsummed=None if more is None else u.upload(more, held), eps=eps)
    r = bo.norm_bwd(dout, s, w, more, eps)
    gsize = np.abs(dout).max(1, keepdims=True) * aw * rstd * (1 + np.abs(xhat).max(1, keepdims=True)) * (1 + np.abs(s).max(1, keepdims=True) * rstd)
    msize = 0.0 if more is None else np.abs(more)
    u.close(g["dx"], r["ds"], 64, "dx", size=gsize + msize)
    if residual:
        u.close(g["dresidual"], r["ds"], 64, "dresidual", size=gsize + msize)
        assert (g["dresidual"] is g["dx"]) == (held == io)
    shift = (1 + np.abs(s).max(1) * rstd[:, 0]).max()
    if weight:
        u.close(g["dweight"], r["dweight"], 32, "dweight", size=r["dweight_size"] + np.abs(dout).sum(0) * shift)
    if bias:
        u.close(g["dbias"], r["dbias"], 32, "dbias", size=r["dbias_size"])
    assert (g["dweight"] is None) == (not weight) and (g["dbias"] is None) == (not bias)


# widths around a slice, the forms' limits, and rows that no registers hold
@pytest.mark.parametrize("io,residual", [("f32", None), ("f32", "f32"), ("bf16", None), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("width", [1, 3, 8, 9, 127, 128, 129, 511, 513, 1021, 1025, 2048, 2050, 4097, 8192, 8200, 16384, 16391, 40001])
def test_widths(width, io, residual):
    check(5, width, io, residual, seed=width)


@pytest.mark.parametrize("width", [64, 100, 1000, 1024, 2047, 2048])
@pytest.mark.parametrize("rows", [1023, 1024, 4099])
def test_many_rows(rows, width):
    check(rows, width, "bf16", "bf16", seed=rows)
    check(rows, width, "f32", None, bias=False, seed=rows)


def test_rows_beyond_the_parts():
    check(70001, 24, "f32", "f32")
    check(9001, 520, "bf16", None)
    check(700, 20000, "bf16", None)


@pytest.mark.parametrize("rows", [1, 2, 63])
def test_few_rows(rows):
    for width in (2048, 768, 40):
        check(rows, width, "bf16", "f32")
        check(rows, width, "bf16", "bf16", weight=False, bias=False, dsummed=False)


def test_options():
    for weight in (False, True):
        for bias in (False, True):
            check(70, 96, "f32", "f32", weight=weight, bias=bias, dsummed=weight)
            check(1100, 600, "bf16", None, weight=weight, bias=bias)


def test_in_place_stream():
    for width in (64, 2048, 5000, 20000):
        check(1500 if width < 3000 else 9, width, "bf16", "bf16", place=True)
        check(1500 if width < 3000 else 9, width, "bf16", "f32", place=True)


def test_large_mean_small_variance():
    """Two sweeps: a mean a thousand times the deviation costs three digits, not six."""
    check(40, 1000, "f32", offset=1000.0)
    check(40, 3000, "f32", offset=-50.0, scale=1e-3, eps=1e-12)
    check(9, 17000, "f32", offset=1000.0)


def test_constant_rows():
    x = torch.full((4, 256), 3.0, device="cuda")
    b = torch.arange(256, device="cuda", dtype=torch.float32)
    out, _, stats = B.ss_norm_fwd(x, None, b, save_stats=True)
    assert torch.equal(out, b.expand(4, 256)) and torch.allclose(stats[1], torch.tensor(1e-5, device="cuda").rsqrt())
    one, _, _ = B.ss_norm_fwd(torch.randn(6, 1, device="cuda"), None, b[:1])
    assert not one.any()


def test_bad_rows_stay_alone():
    for width in (64, 700, 2048, 6000, 20000):
        x = torch.randn(9, width, device="cuda")
        want, _, _ = B.ss_norm_fwd(x)
        x[2, width // 2], x[5, 0], x[8, width - 1] = float("nan"), float("inf"), float("-inf")
        got, _, _ = B.ss_norm_fwd(x)
        keep = [0, 1, 3, 4, 6, 7]
        assert torch.equal(got[keep], want[keep])
        assert not torch.isfinite(got[[2, 5, 8]]).any()


def test_no_rows():
    w = torch.ones(24, device="cuda")
    e = torch.empty(0, 24, device="cuda")
    out, s, stats = B.ss_norm_fwd(e, w, w, residual=e, save_stats=True)
    assert out.shape == s.shape == (0, 24)
    g = B.ss_norm_bwd(e, e, stats, w, has_bias=True, residual_dtype=torch.float32)
    assert not g["dweight"].any() and not g["dbias"].any()


def test_outputs_stay_in_their_memory():
    for io in ("f32", "bf16"):
        for width in (1, 13, 130, 1021, 9001, 16390):
            pool = torch.full((3 * width + 40,), 3.0, dtype=u.TYPES[io], device="cuda")
            held = pool.clone()
            x = torch.randn(3, width, device="cuda").to(u.TYPES[io])
            B.ss_norm_fwd(x, residual=x, out=pool[17:17 + 3 * width].view(3, width), summed=held[17:17 + 3 * width].view(3, width))
            for p in (pool, held):
                assert (p[:17] == 3).all() and (p[17 + 3 * width:] == 3).all()


def test_unaligned_inputs():
    for io in ("f32", "bf16"):
        for width in (64, 1000, 2048):
            pool = torch.randn(1100 * width + 3, device="cuda").to(u.TYPES[io])
            x = pool[3:].view(1100, width)
            assert torch.equal(B.ss_norm_fwd(x)[0], B.ss_norm_fwd(x.clone())[0])


def test_autograd():
    for io, held in (("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")):
        rng = np.random.default_rng(1)
        x, r = u.rounded(rng.standard_normal((3, 11, 40)), io), u.rounded(rng.standard_normal((3, 11, 40)), held)
        w, b = rng.standard_normal(40).astype(np.float32), rng.standard_normal(40).astype(np.float32)
        t = [u.upload(x, io), u.upload(r, held), torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda()]
        for v in t:
            v.requires_grad_(True)
        out, s = ag.layer_norm(t[0], t[2], t[3], residual=t[1])
        do, ds = u.rounded(rng.standard_normal((3, 11, 40)), io), u.rounded(rng.standard_normal((3, 11, 40)), held)
        g = torch.autograd.grad((out, s), t, (u.upload(do, io), u.upload(ds, held)))
        sv = u.host(s).reshape(33, 40)
        ref = bo.norm_bwd(do.reshape(33, 40), sv, w, ds.reshape(33, 40))
        size = 64 * np.ones((33, 40))
        u.close(g[0].reshape(33, 40), ref["ds"], 64, "dx", size=size)
        u.close(g[1].reshape(33, 40), ref["ds"], 64, "dresidual", size=size)
        u.close(g[2], ref["dweight"], 64, "dweight", size=ref["dweight_size"] + 33)
        u.close(g[3], ref["dbias"], 64, "dbias", size=ref["dbias_size"])
        # only one of the two results used
        out, s = ag.layer_norm(t[0], t[2], t[3], residual=t[1])
        gx, gr = torch.autograd.grad(s, t[:2], u.upload(ds, held))
        assert gx.dtype == t[0].dtype and torch.equal(gr, u.upload(ds, held))
        out, s = ag.layer_norm(t[0], t[2], t[3], residual=t[1])
        gx, = torch.autograd.grad(out, t[:1], u.upload(do, io))
        u.close(gx.reshape(33, 40), bo.norm_bwd(do.reshape(33, 40), sv, w)["ds"], 64, "dx", size=size)
    x = torch.randn(5, 24, device="cuda", requires_grad=True)
    ag.layer_norm(x).sum().backward()   # an expanded gradient; of no weight, no residual
    u.close(x.grad, np.zeros((5, 24)), 64, "dx", size=8.0)


def test_differences():
    rng = np.random.default_rng(5)
    x, w = u.upload(rng.standard_normal((20, 130)), "f32"), u.upload(rng.standard_normal(130), "f32")
    do = u.upload(rng.standard_normal((20, 130)), "f32")
    _, _, stats = B.ss_norm_fwd(x, w, save_stats=True)
    g = B.ss_norm_bwd(do, x, stats, w)
    for name, grad in (("x", "dx"), ("w", "dweight")):
        base = {"x": x, "w": w}
        v = u.upload(rng.standard_normal(tuple(base[name].shape)), "f32")

        def loss(sign):
            t = {**base, name: base[name] + sign * 1e-2 * v}
            return (B.ss_norm_fwd(t["x"], t["w"])[0].double() * do.double()).sum().item()
        num, terms = (loss(1) - loss(-1)) / 2e-2, g[grad].double() * v.double()
        assert abs(num - terms.sum().item()) < 2e-3 * terms.abs().sum().item() + 1e-2, name


def test_deterministic_and_other_streams():
    x = torch.randn(5000, 1500, device="cuda").bfloat16()
    w = torch.randn(1500, device="cuda")

    def both(stream=None):
        out, s, stats = B.ss_norm_fwd(x, w, w, residual=x, save_stats=True, stream=stream)
        g = B.ss_norm_bwd(x, s, stats, w, has_bias=True, residual_dtype=torch.bfloat16, dsummed=x, stream=stream)
        return [out, s, stats, g["dx"], g["dweight"], g["dbias"]]
    a = both()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = both()
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_offsets_past_32_bits():
    rows, width = 1050000, 2048
    free, _ = torch.cuda.mem_get_info()
    if free < 30 << 30:
        pytest.skip("needs 30 GiB")
    x = torch.zeros(rows, width, device="cuda")
    x[-2:] = torch.randn(2, width, device="cuda")
    out, s, _ = B.ss_norm_fwd(x, residual=x)
    want = B.ss_norm_fwd(x[-2:].clone(), residual=x[-2:].clone())[0]
    u.close(out[-2:], u.host(want), 32, "out")
    assert not out[:-2].any() and torch.equal(s[-2:], 2 * x[-2:])


def test_refusals():
    x = torch.randn(4, 32, device="cuda")
    w = torch.ones(32, device="cuda")
    for bad in (dict(x=x.half()), dict(weight=w.bfloat16()), dict(residual=x.bfloat16()), dict(x=x.double())):
        with pytest.raises(TypeError):
            B.ss_norm_fwd(**{**dict(x=x), **bad})
    for bad in (dict(x=x[:, ::2]), dict(weight=w[:16]), dict(residual=x[:2]), dict(x=x.cpu()), dict(summed=x)):
        with pytest.raises(ValueError):
            B.ss_norm_fwd(**{**dict(x=x), **bad})
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(B.SsError):
            B.ss_norm_fwd(x, eps=eps)
    _, _, stats = B.ss_norm_fwd(x, save_stats=True)
    with pytest.raises(ValueError):
        B.ss_norm_bwd(x, x, stats, dsummed=x)
    with pytest.raises(B.SsError):
        B.ss_norm_bwd(x, x, stats, w, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
