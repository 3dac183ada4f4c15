"""Gated linear recurrence on the GPU against the float64 oracle.

Tolerances in multiples of 2^-24 (op_util.close): a step's decay is off by at most four roundings, which accumulate over
the state's memory, at most about a thousand steps here (a up to 0.999): 512, between the 4 sqrt(1000) of random and the 4000 of
one-sided errors.  Gradients multiply two such quantities (1024).  Sums are held to the same multiples of the sum of the terms'
magnitudes."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2312_00752_amd import autograd as ag
from paper_2312_00752_amd import binding as B
from tests import op_util as u

pytestmark = pytest.mark.gpu
FWD, BWD = 512, 1024


def make(nb, nd, nl, io, seed=0, i=True, z=True, bias=True, reset=0.0, h0=False):
    rng = np.random.default_rng(seed)
    big = ("x", "f") + (("i",) if i else ()) + (("z",) if z else ())
    d = {k: u.rounded(rng.standard_normal((nb, nd, nl)), io) for k in big}
    d["rate"] = rng.uniform(0.5, 2.0, nd).astype(np.float32)
    if bias:
        half = -np.log(rng.uniform(0.9, 0.999, nd)) / d["rate"]
        d["f_bias"] = np.log(half / (1 - half)).astype(np.float32)
        if i:
            d["i_bias"] = rng.standard_normal(nd).astype(np.float32)
    if reset:
        d["reset"] = rng.random((nb, nl)) < reset
    if h0:
        d["h0"] = rng.standard_normal((nb, nd)).astype(np.float32)
    return d, big


def on_gpu(d, big, io):
    g = {k: u.upload(v, io) if k in big else torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in d.items()}
    return g


def check(nb, nd, nl, io, seed=0, dh_last=True, **kw):
    d, big = make(nb, nd, nl, io, seed, **kw)
    g = on_gpu(d, big, io)
    rng = np.random.default_rng(seed + 1)
    dout = u.rounded(rng.standard_normal((nb, nd, nl)), io)
    dhl = rng.standard_normal((nb, nd)).astype(np.float32) if dh_last else None
    ws = torch.full((max(256, B.ss_gate_workspace_bytes(nb, nd, nl)),), 0xFF, dtype=torch.uint8, device="cuda")
    out, last = B.ss_gate_fwd(**g, return_last_state=True, workspace=ws, save_for_bwd=True)
    grads = B.ss_gate_bwd(u.upload(dout, io), workspace=ws, dh_last=None if dhl is None else torch.from_numpy(dhl).cuda(),
                          want_dh0="h0" in d, **g)
    plain, plain_last = B.ss_gate_fwd(**g, return_last_state=True)
    torch.cuda.synchronize()
    ro, _, rl = bo.gate_fwd(**d)
    u.close(out, ro, FWD, "out")
    u.close(last, rl, FWD, "h_last")
    assert torch.equal(out, plain) and torch.equal(last, plain_last)
    r = bo.gate_bwd(dout, dh_last=dhl, **d)
    for name, t in grads.items():
        if t is None:
            continue
        u.close(t, r[name], BWD, name, r.get(name + "_size"))
    assert {k for k, v in grads.items() if v is not None} == {k for k in ("dx", "df", "di", "dz", "drate", "df_bias", "di_bias", "dh0")
                                                             if k[1:] in d}


# lengths around a lane's slice, a row of lanes, a wave's piece and two of them, and several segments
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("nl", [1, 2, 7, 8, 9, 31, 32, 33, 63, 127, 128, 129, 511, 512, 513, 1023, 1024, 1537, 4100])
def test_lengths(nl, io):
    check(2, 5, nl, io, seed=nl, h0=nl % 2 == 0)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("reset", [0.0, 0.02])
@pytest.mark.parametrize("z", [False, True])
@pytest.mark.parametrize("i", [False, True])
def test_forms(i, z, reset, io):
    for nl in (20, 100, 700):
        check(3, 17, nl, io, seed=5, i=i, z=z, reset=reset, h0=True, dh_last=z)
    check(1, 3, 45, io, seed=6, i=i, z=z, reset=reset, bias=False)


@pytest.mark.parametrize("nb,nd,nl", [(1, 1, 1), (1, 2300, 600), (7, 301, 96), (1, 4, 20000), (3, 700, 1030), (2, 64, 2048)])
def test_rows(nb, nd, nl):
    check(nb, nd, nl, "bf16", seed=nd, reset=0.001, h0=True)
    check(nb, nd, nl, "f32", seed=nd)


def test_every_step_a_reset():
    check(2, 9, 600, "f32", reset=1.0, h0=True)
    check(2, 9, 40, "bf16", reset=1.0, h0=True)


@pytest.mark.parametrize("nl", [30, 120, 1400, 6000])
def test_nothing_passes_a_reset(nl):
    """Infinities and NaN in one document, in inputs and in the gradient, leave its neighbours as they are."""
    d, big = make(2, 6, nl, "f32", i=True, z=True)
    a, b = nl // 3, 2 * nl // 3
    reset = np.zeros((2, nl), bool)
    reset[:, [a, b]] = True
    d["reset"] = reset
    dout = np.random.default_rng(1).standard_normal((2, 6, nl))
    ref, refg = bo.gate_fwd(**d), bo.gate_bwd(dout, **d)
    bad = {**d, "x": d["x"].copy()}
    bad["x"][:, ::2, (a + b) // 2] = np.nan
    bad["x"][:, 1::2, (a + b) // 2] = np.inf
    dbad = dout.copy()
    dbad[:, :, (a + b) // 2] = np.nan
    g = on_gpu(bad, big, "f32")
    ws = torch.empty(B.ss_gate_workspace_bytes(2, 6, nl), dtype=torch.uint8, device="cuda")
    out, last = B.ss_gate_fwd(**g, workspace=ws, save_for_bwd=True, return_last_state=True)
    grads = B.ss_gate_bwd(u.upload(dbad, "f32"), workspace=ws, **g)
    for sl in (slice(0, a), slice(b, nl)):
        u.close(out[..., sl], ref[0][..., sl], FWD, "out")
        for name in ("dx", "df", "di", "dz"):
            u.close(grads[name][..., sl], refg[name][..., sl], BWD, name)
    u.close(last, ref[2], FWD, "h_last")
    assert not torch.isfinite(out[..., (a + b) // 2]).any()


def test_logits_at_the_ends():
    """Logits of +-infinity and the type's extremes: a is exp(-rate) or 1, g is 1 or 0."""
    inf = float("inf")
    for io in ("f32", "bf16"):
        top = torch.finfo(u.TYPES[io]).max
        d, big = make(1, 2, 48, io, bias=False)
        for k, vals in (("f", (inf, -inf, top, -top, 90.0, -90.0)), ("i", (-inf, inf, -top, top, -90.0, 90.0))):
            d[k][0, :, 5:41:6] = np.array(vals).reshape(1, -1)
        g = on_gpu(d, big, io)
        ws = torch.empty(max(256, B.ss_gate_workspace_bytes(1, 2, 48)), dtype=torch.uint8, device="cuda")
        out, _ = B.ss_gate_fwd(**g, workspace=ws, save_for_bwd=True)
        ref = bo.gate_fwd(**d)[0]
        u.close(out, ref, FWD, "out")
        dout = np.ones((1, 2, 48))
        r, grads = bo.gate_bwd(dout, **d), B.ss_gate_bwd(u.upload(dout, io), workspace=ws, **g)
        for name in ("dx", "df", "di", "dz"):
            u.close(grads[name], r[name], BWD, name)


def test_rate_zero_holds_the_state():
    d, big = make(1, 3, 70, "f32", h0=True)
    d["rate"][1] = 0.0
    g = on_gpu(d, big, "f32")
    ws = torch.empty(max(256, B.ss_gate_workspace_bytes(1, 3, 70)), dtype=torch.uint8, device="cuda")
    out, last = B.ss_gate_fwd(**g, workspace=ws, save_for_bwd=True, return_last_state=True)
    assert last[0, 1].item() == d["h0"][0, 1]
    dout = np.random.default_rng(1).standard_normal((1, 3, 70))
    r, grads = bo.gate_bwd(dout, **d), B.ss_gate_bwd(u.upload(dout, "f32"), workspace=ws, want_dh0=True, **g)
    for name, t in grads.items():
        u.close(t, r[name], BWD, name, r.get(name + "_size"))


@pytest.mark.parametrize("s0", [1e-7, 1e-5, 1e-3, 0.03, 0.06, 0.07, 0.2])
def test_decay_near_one(s0):
    """m = sqrt(1 - a^2) keeps its relative accuracy however near a is to 1 (and about y = 2 rate s = 1/8, where the form changes).
    Single steps from the zero state: h = m x with x = 1; ten roundings."""
    f = np.log(s0 / (1 - s0)) + np.linspace(-0.2, 0.2, 64)
    d = {"x": np.ones((1, 1, 64)), "f": u.rounded(f, "f32").reshape(1, 1, 64), "rate": np.ones(1, np.float32), "reset": None}
    x, ff = (u.upload(d[k].reshape(1, 64, 1), "f32") for k in ("x", "f"))
    out, _ = B.ss_gate_fwd(x, ff, torch.ones(64, device="cuda"))
    s = 1 / (1 + np.exp(-d["f"].reshape(-1)))
    ref = np.sqrt(-np.expm1(-2 * s)).reshape(1, 64, 1)
    u.close(out, ref, 24, "m", size=np.abs(ref))


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_slices_of_wider_tensors(io):
    """x, f, i, z and their gradients as slices along dim 1 of one (B, 4D, L) tensor, at odd lengths, NaN around them."""
    nb, nd, nl = 3, 10, 37
    d, big = make(nb, nd, nl, io, h0=True)
    wide = torch.full((nb, 4 * nd + 3, nl), float("nan"), dtype=u.TYPES[io], device="cuda")
    gwide = torch.full_like(wide, 7.0)
    g = on_gpu(d, big, io)
    cut = {}
    for k, name in enumerate(big):
        wide[:, 1 + k * nd: 1 + (k + 1) * nd] = g[name]
        cut[name] = wide[:, 1 + k * nd: 1 + (k + 1) * nd]
    grads = {"d" + name: gwide[:, 1 + k * nd: 1 + (k + 1) * nd] for k, name in enumerate(big)}
    ws = [torch.empty(max(256, B.ss_gate_workspace_bytes(nb, nd, nl)), dtype=torch.uint8, device="cuda") for _ in range(2)]
    dout = u.upload(np.random.default_rng(1).standard_normal((nb, nd, nl)), io)
    rest = {k: v for k, v in g.items() if k not in big}
    a = B.ss_gate_fwd(**g, workspace=ws[0], save_for_bwd=True)[0]
    b = B.ss_gate_fwd(**cut, **rest, workspace=ws[1], save_for_bwd=True)[0]
    assert torch.equal(a, b)
    ga = B.ss_gate_bwd(dout, workspace=ws[0], want_dh0=True, **g)
    gb = B.ss_gate_bwd(dout, workspace=ws[1], want_dh0=True, grads=grads, **cut, **rest)
    for name in ga:
        assert torch.equal(ga[name], gb[name]), name
    assert (gwide[:, 0] == 7).all() and (gwide[:, 1 + 4 * nd:] == 7).all()


def test_outputs_stay_in_their_memory():
    for io in ("f32", "bf16"):
        for nl in (1, 5, 13, 130, 519):
            d, big = make(1, 3, nl, io)
            g = on_gpu(d, big, io)
            pool = torch.full((3 * nl + 32,), 3.0, dtype=u.TYPES[io], device="cuda")
            out = pool[16:16 + 3 * nl].view(1, 3, nl)
            B.ss_gate_fwd(**g, out=out)
            assert (pool[:16] == 3).all() and (pool[16 + 3 * nl:] == 3).all()


def test_pieces_continue():
    d, big = make(2, 7, 1100, "f32", h0=True)
    g = on_gpu(d, big, "f32")
    whole, last = B.ss_gate_fwd(**g, return_last_state=True)
    h, outs = g["h0"], []
    for sl in (slice(0, 333), slice(333, 334), slice(334, 1100)):
        part = {k: (v[..., sl].contiguous() if k in big else v) for k, v in g.items()}
        part["h0"] = h
        o, h = B.ss_gate_fwd(**part, return_last_state=True)
        outs.append(o)
    u.close(torch.cat(outs, -1), u.host(whole), FWD, "out")
    u.close(h, u.host(last), FWD, "h_last")


def test_no_steps():
    rate, h0 = torch.ones(4, device="cuda"), torch.randn(2, 4, device="cuda")
    e = torch.empty(2, 4, 0, device="cuda")
    out, last = B.ss_gate_fwd(e, e, rate, h0=h0, return_last_state=True)
    assert out.shape == (2, 4, 0) and torch.equal(last, h0)
    assert not B.ss_gate_fwd(e, e, rate, return_last_state=True)[1].any()
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    g = B.ss_gate_bwd(e, e, e, rate, ws, f_bias=rate, dh_last=h0, want_dh0=True)
    assert torch.equal(g["dh0"], h0) and not g["drate"].any() and not g["df_bias"].any()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("nb,nd,i,z,bias,reset", [(1, 1, True, True, True, 0.0), (3, 257, True, True, True, 0.5), (64, 4096, True, False, True, 0.0),
                                                  (2, 100, False, True, False, 0.0), (5, 4098, False, False, True, 0.3)])
def test_step(nb, nd, i, z, bias, reset, io):
    d, big = make(nb, nd, 1, io, i=i, z=z, bias=bias, reset=reset, h0=True)
    g = on_gpu(d, big, io)
    h = g.pop("h0").clone()
    wide = torch.full((nb, 4 * nd + 1), float("nan"), dtype=u.TYPES[io], device="cuda")
    t = {}
    for k, name in enumerate(("x", "f", "i", "z")):
        if name in big:
            wide[:, k * nd + 1: (k + 1) * nd + 1] = g[name][..., 0]
            t[name + "_t"] = wide[:, k * nd + 1: (k + 1) * nd + 1]
    args = {k: g[k] for k in ("rate", "f_bias", "i_bias") if k in g}
    if reset:
        args["reset_t"] = g["reset"][:, 0].contiguous()
    h1 = h.clone()
    out = B.ss_gate_step(h, **t, **args)
    ro, _, rl = bo.gate_fwd(**d)
    u.close(out, ro[..., 0], 32, "out", size=np.max(np.abs(ro)))
    u.close(h, rl, 32, "h")
    out1 = B.ss_gate_step(h1, **{k: v.contiguous() for k, v in t.items()}, **args)
    assert torch.equal(out, out1) and torch.equal(h, h1)


def test_steps_follow_a_prompt():
    d, big = make(2, 50, 24, "f32", reset=0.1)
    g = on_gpu(d, big, "f32")
    ref, _, last = bo.gate_fwd(**d)
    part = {k: (v[..., :20].contiguous() if k in big or k == "reset" else v) for k, v in g.items()}
    _, h = B.ss_gate_fwd(**part, return_last_state=True)
    for t in range(20, 24):
        o = B.ss_gate_step(h, *(g[k][..., t] if False else g[k][..., t].contiguous() for k in ("x", "f")), g["rate"], i_t=g["i"][..., t].contiguous(),
                           z_t=g["z"][..., t].contiguous(), f_bias=g["f_bias"], i_bias=g["i_bias"], reset_t=g["reset"][:, t].contiguous())
        u.close(o, ref[..., t], FWD, "out", size=np.max(np.abs(ref)))
    u.close(h, last, FWD, "h")


def test_autograd():
    """Every input's gradient through the front-end, shared and broadcast inputs, a gradient of the last state alone."""
    d, big = make(2, 6, 75, "f32", reset=0.05, h0=True)
    g = on_gpu(d, big, "f32")
    reset = g.pop("reset")
    for v in g.values():
        v.requires_grad_(True)
    out, last = ag.gated_recurrence(**g, reset=reset, return_last_state=True)
    w, wl = np.random.default_rng(3).standard_normal((2, 6, 75)), np.random.default_rng(4).standard_normal((2, 6))
    r = bo.gate_bwd(w, dh_last=wl, **d)
    grads = torch.autograd.grad((out, last), list(g.values()), (u.upload(w, "f32"), u.upload(wl, "f32")))
    for name, t in zip(g, grads):
        n = {"f_bias": "df_bias", "i_bias": "di_bias"}.get(name, "d" + name)
        u.close(t, r[n], BWD, n, r.get(n + "_size"))
    # only the last state
    last = ag.gated_recurrence(**g, reset=reset, return_last_state=True)[1]
    r = bo.gate_bwd(np.zeros_like(w), dh_last=wl, **d)
    gx, = torch.autograd.grad(last, g["x"], u.upload(wl, "f32"))
    u.close(gx, r["dx"], BWD, "dx")
    # x in two places, a gradient that is an expanded tensor
    x = g["x"].detach().requires_grad_(True)
    rate = g["rate"].detach()
    y = ag.gated_recurrence(x, x, rate)
    y.sum().backward()
    r = bo.gate_bwd(np.ones_like(w), d["x"], d["x"], d["rate"])
    u.close(x.grad, r["dx"] + r["df"], BWD, "dx + df")


def test_differences():
    """The gradient against differences of the GPU's own forward pass, in float32 over a direction (error of the quotient: about
    2^-24 |loss| / step)."""
    d, big = make(2, 8, 300, "f32", h0=True)
    g = on_gpu(d, big, "f32")
    rng = np.random.default_rng(9)
    w = u.upload(rng.standard_normal((2, 8, 300)), "f32")
    ws = torch.empty(max(256, B.ss_gate_workspace_bytes(2, 8, 300)), dtype=torch.uint8, device="cuda")
    B.ss_gate_fwd(**g, workspace=ws, save_for_bwd=True)
    grads = B.ss_gate_bwd(w, workspace=ws, want_dh0=True, **g)
    names = {"x": "dx", "f": "df", "i": "di", "z": "dz", "rate": "drate", "f_bias": "df_bias", "i_bias": "di_bias", "h0": "dh0"}
    for name, grad in names.items():
        v = u.upload(rng.standard_normal(tuple(g[name].shape)), "f32")
        e = 1e-2

        def loss(sign):
            out = B.ss_gate_fwd(**{**g, name: g[name] + sign * e * v})[0]
            return (out.double() * w.double()).sum().item()
        num = (loss(1) - loss(-1)) / (2 * e)
        ana = (grads[grad].double() * v.double()).sum().item()
        size = (grads[grad].double() * v.double()).abs().sum().item()
        assert abs(num - ana) < 5e-3 * size + 1e-2, (name, num, ana)


def test_deterministic_and_other_streams():
    d, big = make(4, 300, 1500, "bf16")
    g = on_gpu(d, big, "bf16")
    dout = u.upload(np.random.default_rng(1).standard_normal((4, 300, 1500)), "bf16")

    def both(stream=None):
        ws = torch.empty(B.ss_gate_workspace_bytes(4, 300, 1500), dtype=torch.uint8, device="cuda")
        out, _ = B.ss_gate_fwd(**g, workspace=ws, save_for_bwd=True, stream=stream)
        r = B.ss_gate_bwd(dout, workspace=ws, stream=stream, **g)
        return [out, ws] + [v for v in r.values() if v is not None]
    a = both()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    b = both(s)
    s.synchronize()
    with torch.cuda.stream(s):
        c = both()
    s.synchronize()
    for i, (p, q, r) in enumerate(zip(a, b, c)):
        if i != 1:
            assert torch.equal(p, q) and torch.equal(p, r), i


def test_graph_replays():
    d, big = make(2, 100, 1, "bf16", h0=True)
    g = on_gpu(d, big, "bf16")
    h = g.pop("h0")
    t = {k + "_t": g[k][..., 0].contiguous() for k in big}
    args = {k: g[k] for k in ("rate", "f_bias", "i_bias")}
    want_h, want = h.clone(), []
    for _ in range(4):
        want.append(B.ss_gate_step(want_h, **t, **args).clone())
    out = torch.empty_like(t["x_t"])
    hs = h.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.ss_gate_step(hs, **t, **args, out_t=out)
    hs.copy_(h)
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[k])
        torch.zeros(1000, device="cuda").sum().item()
    assert torch.equal(hs, want_h)


def test_offsets_past_32_bits():
    """More than 2^31 elements in each tensor; the first and the last rows against the same rows by themselves."""
    nd, nl = 2090, 1 << 20
    free, _ = torch.cuda.mem_get_info()
    if free < 30 << 30:
        pytest.skip("needs 30 GiB")
    x = torch.zeros(1, nd, nl, device="cuda")
    ends = torch.randn(1, 4, nl, device="cuda")
    x[:, :2], x[:, -2:] = ends[:, :2], ends[:, 2:]
    rate = torch.linspace(0.01, 1.0, nd, device="cuda")
    out, last = B.ss_gate_fwd(x, x, rate, return_last_state=True)
    few = torch.cat((rate[:2], rate[-2:]))
    want, wl = B.ss_gate_fwd(ends, ends, few, return_last_state=True)
    u.close(torch.cat((out[:, :2], out[:, -2:]), 1), u.host(want), FWD, "out")
    u.close(torch.cat((last[:, :2], last[:, -2:]), 1), u.host(wl), FWD, "h_last")
    assert not out[:, 2:-2].any()


def test_refusals():
    x = torch.randn(2, 3, 16, device="cuda")
    rate = torch.ones(3, device="cuda")
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    fwd = lambda **k: B.ss_gate_fwd(**{**dict(x=x, f=x, rate=rate), **k})
    for bad in (dict(f=x.bfloat16()), dict(rate=rate.double()), dict(x=x.half(), f=x.half()), dict(reset=torch.zeros(2, 16, device="cuda"))):
        with pytest.raises(TypeError):
            fwd(**bad)
    for bad in (dict(f=x[..., :8]), dict(x=x.transpose(1, 2), f=x.transpose(1, 2)), dict(rate=rate[:2]), dict(x=x.cpu(), f=x), dict(i_bias=rate),
                dict(h0=torch.zeros(3, 2, device="cuda")), dict(reset=torch.zeros(2, 8, dtype=torch.bool, device="cuda")), dict(save_for_bwd=True),
                dict(f=x.as_strided((2, 3, 16), (16, 16, 1))), dict(x=x[..., ::2], f=x[..., ::2])):
        with pytest.raises(ValueError):
            fwd(**bad)
    with pytest.raises(B.SsError):
        B.ss_gate_bwd(x, x, x, rate, ws[:16])
    with pytest.raises(ValueError):
        B.ss_gate_bwd(x, x, x, rate, ws, grads={"di": x})
    with pytest.raises(ValueError):
        B.ss_gate_step(torch.zeros(2, 3, device="cuda"), x[..., 0], x[..., 0], rate)
