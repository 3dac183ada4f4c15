"""AdamW on the GPU against the float64 oracle and, bit by bit, against its definition in float32.

The moments are two products and a sum of float32 numbers, each rounded, and the 8-bit codes are made from them in float32 operations
that are exact or rounded to the nearest: numpy's give the same bits.  Tolerance of a parameter, in multiples of 2^-24: one rounding of the decayed
value and one of the sum, 3 of |param|, and for the step lr / c1 m / (sqrt(v) / sqrt(c2) + eps): c1 = -expm1(t log beta) with a rounded argument, two quotients,
a reciprocal to a unit in the last place, products: 24 of |step|, where the errors of m, the rounded sum of two rounded products that may cancel, are relative
to the sum of their magnitudes: |step| is what that sum in m's place would make."""
import copy
import io as io_module

import numpy as np
import pytest
import torch

from oracle import model_oracle as mo
from paper_2312_00752_amd import binding as B
from paper_2312_00752_amd import optim
from tests import op_util as u

pytestmark = pytest.mark.gpu
F = np.float32
OPTIONS = dict(betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


def codes_in_f32(x, step, signed):
    """adamw_codes of the header in float32, operation by operation."""
    x = np.asarray(x, F)
    n, top = len(x), F(127 if signed else 255)
    c0, c1 = (0x6A09E667, 0xBB67AE85) if signed else (0x3C6EF372, 0xA54FF53A)
    codes, scale = np.zeros(n, np.int64), np.zeros(-(-n // 256), F)
    for b in range(len(scale)):
        at = slice(b * 256, min(n, (b + 1) * 256))
        a = np.abs(x[at]).max()
        if not np.isfinite(a):
            scale[b] = np.nan
            continue
        if a < F(2.0 ** -100):
            continue
        scale[b] = a
        y = np.abs(x[at]) * (top * top * (F(1) / a))
        q = np.floor(np.sqrt(y))
        u = ((np.arange(at.start, at.stop, dtype=np.uint64) * c0 + step * c1) % 2 ** 32 >> 8).astype(F) * F(2.0 ** -24)
        q = np.minimum(q + (y - q * q > u * (F(2) * q + F(1))), top)
        codes[at] = np.where(x[at] < 0, -q, q) if signed else np.where(x[at] > 0, np.maximum(q, 1), 0)
    return codes, scale


def values_in_f32(codes, scale, signed):
    q, top = np.asarray(codes).astype(F), F(127 if signed else 255)
    return q * np.abs(q) * (np.repeat(scale, 256)[: len(q)] * (F(1) / (top * top)))


class Case:
    """Tensors of the given sizes; their state as numpy arrays beside it."""

    def __init__(self, sizes, bits, low_param=False, low_grad=False, master=False, steps=7, seed=0, spread=1.0):
        rng = np.random.default_rng(seed)
        self.bits, self.low, self.has_master, self.taken = bits, low_param, master, steps
        pio, gio = ("bf16" if low_param else "f32"), ("bf16" if low_grad else "f32")
        size = lambda n: np.exp(spread * rng.standard_normal(n))
        self.p = [u.rounded(rng.standard_normal(n), "f32" if master else pio) for n in sizes]
        self.g = [u.rounded(rng.standard_normal(n) * size(n) * 1e-2, gio) for n in sizes]
        m = [(1e-3 * rng.standard_normal(n) * size(n)).astype(F) for n in sizes]
        v = [(1e-4 * rng.uniform(size=n) * size(n)).astype(F) for n in sizes]
        up = lambda a, t: [torch.from_numpy(np.asarray(x)).to("cuda").to(t) for x in a]
        self.params, self.grads = up([u.rounded(p, pio) for p in self.p], u.TYPES[pio]), up(self.g, u.TYPES[gio])
        self.master = up(self.p, torch.float32) if master else None
        self.m_scale = self.v_scale = None
        if bits == 8:
            cm, cv = [codes_in_f32(x, steps, True) for x in m], [codes_in_f32(np.sqrt(x), steps, False) for x in v]
            self.m, self.v = up([c[0] for c in cm], torch.int8), up([c[0] for c in cv], torch.uint8)
            self.m_scale, self.v_scale = up([c[1] for c in cm], torch.float32), up([c[1] for c in cv], torch.float32)
            m = [values_in_f32(*c, True) for c in cm]
            s = [values_in_f32(*c, False) for c in cv]
            v = [x * x for x in s]
        else:
            self.m, self.v = up(m, torch.float32), up(v, torch.float32)
        self.nm, self.nv = m, v
        self.count = torch.tensor([steps, 0], dtype=torch.int32, device="cuda")

    def run(self, lr=1e-2, grad_scale=None, **options):
        B.ss_adamw_step(self.params, self.grads, self.m, self.v, self.count, lr, master=self.master, m_scale=self.m_scale, v_scale=self.v_scale,
                        grad_scale=grad_scale, **{**OPTIONS, **options})

    def check(self, lr=1e-2, scale=1.0, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1):
        step = self.taken + 1
        assert self.count.tolist() == [step, 0]
        self.taken = step
        b1, r1, b2, r2 = F(betas[0]), F(1 - betas[0]), F(betas[1]), F(1 - betas[1])
        for k, (p, g) in enumerate(zip(self.p, self.g)):
            if not p.size:
                continue
            gs = (g.astype(F) * F(scale))
            ref, _, _, size = mo.adamw(np.asarray(p, np.float64), gs.astype(np.float64), self.nm[k].astype(np.float64), self.nv[k].astype(np.float64), step,
                                       float(F(lr)), *betas, eps, weight_decay)
            limit = np.abs(p) / 8 + size
            if self.has_master:
                u.close(self.master[k], ref, 24, "master %d" % k, size=limit)
                assert torch.equal(self.params[k], self.master[k].bfloat16())
                self.p[k] = u.host(self.master[k])
            else:
                u.close(self.params[k], ref, 24, "param %d" % k, size=limit)
                self.p[k] = u.host(self.params[k])
            m = self.nm[k] * b1 + gs * r1
            v = self.nv[k] * b2 + gs * gs * r2
            if self.bits == 32:
                assert np.array_equal(self.m[k].cpu().numpy(), m) and np.array_equal(self.v[k].cpu().numpy(), v)
            else:
                for x, codes, held, signed in ((m, self.m[k], self.m_scale[k], True), (np.sqrt(v), self.v[k], self.v_scale[k], False)):
                    want, a = codes_in_f32(x, step, signed)
                    assert np.array_equal(held.cpu().numpy(), a) and np.array_equal(codes.cpu().numpy().astype(np.int64), want)
                    # and next to what exact arithmetic gives: a code that a rounding decides may be its neighbour.  y has three roundings, so its place
                    # between two codes is off by 1.5 2^-24 y / (2 q + 1), 2.3e-5 at most: that share of the elements, and a few
                    apart = np.abs(mo.adamw_codes(x, step, signed)[0] - want)
                    most, differ = int(apart.max()), int((apart > 0).sum())
                    assert most <= 1 and differ <= 4 + 1e-4 * x.size
                    value = values_in_f32(want, a, signed)
                    got = B.ss_adamw_values(codes, held)
                    assert np.array_equal(got.cpu().numpy(), value)
                    if signed:
                        m = value
                    else:
                        v = value * value
            self.nm[k], self.nv[k] = m, v


KINDS = {"f32": {}, "bf16": dict(low_param=True, low_grad=True), "master": dict(low_param=True, low_grad=True, master=True),
         "mixed": dict(low_param=True, master=True), "low_grad": dict(low_grad=True)}
SIZES = [1, 2, 3, 4, 5, 63, 64, 65, 255, 256, 257, 511, 1023, 1024, 1025, 4099, 0, 8192, 8193, 20000]


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("kind", sorted(KINDS))
def test_sizes(kind, bits):
    c = Case(SIZES, bits, **KINDS[kind])
    for _ in range(3):
        c.run()
        c.check()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("sizes", [[65536], [1, 60000, 3, 5000], [65537], [70001, 2047, 2049, 1, 300000], [530001, 4095, 4097, 255],
                                   [700001, 1, 8191, 8193, 500000, 4096], [1 << 21, 12287, 12289]])
def test_workgroups(sizes, bits):
    """Workgroups of every size, with one step and two, whole and cut short."""
    c = Case(sizes, bits, low_param=True, master=True, seed=len(sizes))
    for _ in range(2):
        c.run()
        c.check()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("n", [0, 1, 47, 48, 49, 96, 97, 200])
def test_many_tensors(n, bits):
    """As many as a launch's arguments hold, and more; the step is counted once."""
    c = Case([1 + 37 * k % 700 for k in range(n)], bits, seed=n)
    for _ in range(2):
        c.run()
        c.check()


@pytest.mark.parametrize("bits", [8, 32])
def test_options(bits):
    for options in (dict(betas=(0.0, 0.0)), dict(betas=(0.0, 0.999)), dict(betas=(0.9, 0.999), eps=1e-3), dict(weight_decay=0.0)):
        c = Case([700, 5], bits, steps=0)
        c.run(**options)
        c.check(**{**OPTIONS, **options})
    c = Case([700, 5], bits, steps=2 ** 20)
    c.run()
    c.check()


@pytest.mark.parametrize("bits", [8, 32])
def test_numbers_on_the_device(bits):
    lr, scale = torch.tensor([3e-3], device="cuda"), torch.tensor(0.125, device="cuda")
    c = Case([700, 1000], bits)
    c.run(lr=lr, grad_scale=scale)
    c.check(lr=3e-3, scale=0.125)


@pytest.mark.parametrize("bits", [8, 32])
def test_one_tensor_of_many_elements(bits):
    """Chunks of several steps; the first, some inner and the last elements."""
    n = 40_000_003
    p, g = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    p0 = p.clone()
    if bits == 8:
        m, v = torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
        scales = dict(m_scale=[torch.zeros(-(-n // 256), device="cuda")], v_scale=[torch.zeros(-(-n // 256), device="cuda")])
    else:
        m, v, scales = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), {}
    count = torch.zeros(2, dtype=torch.int32, device="cuda")
    B.ss_adamw_step([p], [g], [m], [v], count, 1e-3, weight_decay=0.0, **scales)
    # the first step is lr along the gradient's sign: g / (|g| + eps)
    want = p0.double() - 1e-3 * g.double() / (g.double().abs() + 1e-8)
    assert ((p.double() - want).abs() <= 24 * 2.0 ** -24 * (p0.double().abs() / 8 + 1e-3)).all()
    if bits == 8:
        first = codes_in_f32(g[:768].cpu().numpy() * F(1 - 0.9), 1, True)[0]
        assert np.array_equal(m[:768].cpu().numpy(), first)
        back = B.ss_adamw_values(m, scales["m_scale"][0])
        # off by a code's distance at most: (2 q + 1) / 127^2 of the block's scale, and the scale is no more than 0.1 max |g|
        assert ((back - 0.1 * g).abs() <= 0.1 * g.abs().max() * 2 / 127 + 1e-6).all()
    assert count.tolist() == [1, 0]


@pytest.mark.parametrize("bits", [8, 32])
def test_unaligned_memory(bits):
    a = Case([1000, 257, 5], bits, low_param=True, low_grad=True, master=True)
    b = Case([1000, 257, 5], bits, low_param=True, low_grad=True, master=True)
    off = lambda list_: [torch.cat((t.new_zeros(1), t))[1:] for t in list_]
    for name in ("params", "grads", "m", "v", "master") + (("m_scale", "v_scale") if bits == 8 else ()):
        setattr(b, name, off(getattr(b, name)))
    a.run()
    b.run()
    for name in ("params", "m", "v", "master") + (("m_scale", "v_scale") if bits == 8 else ()):
        assert all(torch.equal(x, y) for x, y in zip(getattr(a, name), getattr(b, name))), name


@pytest.mark.parametrize("bits", [8, 32])
def test_neighbours_stay(bits):
    """Tensors that lie side by side in one memory, with room between them."""
    c = Case([300, 5, 1025], bits)
    rooms = {}
    for name in ("params", "m", "v") + (("m_scale", "v_scale") if bits == 8 else ()):
        list_ = getattr(c, name)
        room = torch.full((sum(t.numel() + 3 for t in list_) + 3,), 77, device="cuda").to(list_[0].dtype)
        mask, at, new = torch.ones_like(room, dtype=torch.bool), 3, []
        for t in list_:
            room[at:at + t.numel()] = t
            mask[at:at + t.numel()] = False
            new.append(room[at:at + t.numel()])
            at += t.numel() + 3
        setattr(c, name, new)
        rooms[name] = (room, mask)
    c.run()
    c.check()
    for room, mask in rooms.values():
        assert (room[mask] == 77).all()


def test_infinities_nan_and_small_values():
    c = Case([1024], 8, steps=0)
    c.g[0][:] = 1e-3
    c.g[0][5], c.g[0][300], c.g[0][512:768], c.g[0][768:] = np.nan, np.inf, 0.0, 1e-33
    c.nm[0][:] = c.nv[0][:] = 0.0
    c.grads = [torch.from_numpy(c.g[0]).float().cuda()]
    for t in c.m + c.v + c.m_scale + c.v_scale:
        t.zero_()
    p0 = c.params[0].clone()
    c.run(weight_decay=0.0)
    moved = c.params[0] - p0
    assert torch.isnan(moved[5]) and torch.isnan(c.m_scale[0][0]) and torch.isnan(c.m_scale[0][1]) and torch.isnan(c.v_scale[0][0])
    assert (torch.cat((moved[:5], moved[6:256])) < 0).all()   # in this step, only the element itself
    assert (moved[512:768] == 0).all() and (c.m[0][512:] == 0).all() and (c.v[0][512:768] == 0).all() and (c.m_scale[0][2:] == 0).all()
    back = B.ss_adamw_values(c.m[0], c.m_scale[0])
    assert torch.isnan(back[:512]).all() and (back[512:] == 0).all()


def test_small_second_moments_do_not_vanish():
    """Next to a large element, a small one keeps a code of 1, so its next step is bounded."""
    c = Case([256], 8, steps=0)
    c.g[0][:] = 1e-9
    c.g[0][0] = 1e3
    c.grads = [torch.from_numpy(c.g[0]).float().cuda()]
    for t in c.m + c.v + c.m_scale + c.v_scale:
        t.zero_()
    c.run()
    assert (c.v[0][1:] == 1).all() and c.v[0][0] == 255


def test_a_long_run():
    """A second moment that moves by less than a code's distance in every step, over a thousand of them: the same bits as in float32 numpy, and it has moved."""
    n, steps, beta2 = 512, 1000, 0.999
    g = np.random.default_rng(0).uniform(0.05, 1.0, n).astype(F)
    g[::256] = 1.0
    tg, p, m, v = torch.from_numpy(g).cuda(), torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.int8, device="cuda"), torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    ms, vs, count = torch.zeros(2, device="cuda"), torch.full((2,), 1.0, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    codes, scale = np.full(n, 255), np.ones(2, F)
    for k in range(steps):
        B.ss_adamw_step([p], [tg], [m], [v], count, 0.0, betas=(0.9, beta2), m_scale=[ms], v_scale=[vs])
        s = values_in_f32(codes, scale, False)
        codes, scale = codes_in_f32(np.sqrt(s * s * F(beta2) + g * g * F(1 - beta2)), k + 1, False)
    assert np.array_equal(v.cpu().numpy(), codes) and np.array_equal(vs.cpu().numpy(), scale) and count.tolist() == [steps, 0]
    assert (codes[g < 0.5] < 230).all()   # sqrt(exp(-1) + 0.64 g^2) is 0.72 at most, 217 of 255


# ---- the optimiser ----------------------------------------------------------------------------------
def against_torch(steps, **options):
    torch.manual_seed(0)
    shapes = [(30, 50), (7,), (300,), ()]
    mine = [torch.nn.Parameter(torch.randn(s, device="cuda")) for s in shapes]
    theirs = [torch.nn.Parameter(p.detach().double()) for p in mine]
    a = optim.AdamW(mine, lr=1e-2, weight_decay=0.05, **options)
    b = torch.optim.AdamW(theirs, lr=1e-2, weight_decay=0.05)
    moved = 0.0
    for k in range(steps):
        for p, q in zip(mine, theirs):
            g = torch.randn_like(p) + 0.5
            p.grad, q.grad = g, g.double()
        a.step()
        b.step()
    return mine, theirs


def test_like_torch():
    mine, theirs = against_torch(20)
    for p, q in zip(mine, theirs):   # 20 steps of 1e-2, each to 24 roundings, of values of a size of 3
        assert ((p - q).abs() <= 20 * 2.0 ** -24 * (3 * q.abs() + 24 * 1e-2)).all()


def test_like_torch_in_8_bits():
    mine, theirs = against_torch(20, state_bits=8)
    for p, q in zip(mine, theirs):
        # a moment's code is off by its distance: of values near the block's largest 1 % and 2 %, of ten times smaller ones 5 % and 3 %; steps of 1e-2
        assert ((p - q).abs().mean() <= 20 * 1e-2 * 0.03).all()


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_state_dict(bits, dtype):
    torch.manual_seed(0)
    make = lambda: [torch.nn.Parameter(torch.ones(300, 2, device="cuda", dtype=dtype)), torch.nn.Parameter(torch.ones(5, device="cuda"))]
    grads = [[torch.randn(300, 2, device="cuda").to(dtype), torch.randn(5, device="cuda")] for _ in range(6)]
    def go(o, ps, gs):
        for pair in gs:
            for p, g in zip(ps, pair):
                p.grad = g
            o.step()
    pa = make()
    a = optim.AdamW(pa, lr=1e-2, state_bits=bits)
    go(a, pa, grads[:3])
    file = io_module.BytesIO()
    torch.save(a.state_dict(), file)
    file.seek(0)
    pb = make()
    with torch.no_grad():
        for p, q in zip(pb, pa):
            p.copy_(q)
    b = optim.AdamW(pb, lr=7.0, state_bits=bits)
    b.load_state_dict(torch.load(file, map_location="cpu", weights_only=True))
    assert b.param_groups[0]["lr"] == 1e-2 and b.param_groups[0]["count"].tolist() == [3, 0]
    go(a, pa, grads[3:])
    go(b, pb, grads[3:])
    assert all(torch.equal(p, q) for p, q in zip(pa, pb))
    with pytest.raises(ValueError):
        optim.AdamW(make(), state_bits=40 - bits).load_state_dict(a.state_dict())
    with pytest.raises(ValueError):
        optim.AdamW(make()[:1], state_bits=bits).load_state_dict(a.state_dict())


@pytest.mark.parametrize("bits", [8, 32])
def test_captured_and_replayed(bits):
    """Each replay is a step of its own, with the rate as it is then."""
    torch.manual_seed(0)
    shapes = [(70, 50), (300,)] + [(5,)] * 60
    start = [torch.randn(s, device="cuda") for s in shapes]
    grads = [[torch.randn(s, device="cuda") for s in shapes] for _ in range(4)]
    eager, graphed = [[torch.nn.Parameter(t.clone()) for t in start] for _ in range(2)]
    a = optim.AdamW(eager, lr=1e-2, state_bits=bits)
    rate = torch.tensor([1e-2], device="cuda")
    b = optim.AdamW(graphed, lr=rate, state_bits=bits)
    for p in graphed:
        p.grad = torch.zeros_like(p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    assert b.param_groups[0]["count"].tolist() == [0, 0]
    for k, gs in enumerate(grads):
        a.param_groups[0]["lr"] = 1e-2 / (k + 1)
        rate.fill_(1e-2 / (k + 1))
        for p, q, g in zip(eager, graphed, gs):
            p.grad = g
            q.grad.copy_(g)
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        assert b.param_groups[0]["count"].tolist() == [k + 1, 0]
        for p, q in zip(eager, graphed):
            assert torch.equal(p, q)


def test_groups_and_missing_gradients():
    p, q, r = (torch.nn.Parameter(torch.ones(10, device="cuda")) for _ in range(3))
    o = optim.AdamW([{"params": [p, q], "lr": 1e-1}, {"params": [r], "weight_decay": 0.5, "state_bits": 8}], lr=1e-2, weight_decay=0.0)
    p.grad, r.grad = torch.ones(10, device="cuda"), torch.zeros(10, device="cuda")
    o.step()
    assert torch.allclose(p, torch.full_like(p, 0.9)) and (q == 1).all() and torch.allclose(r, torch.full_like(r, 1 - 0.005))
    assert o.step(lambda: 3.5) == 3.5
    for g in torch.optim.lr_scheduler.StepLR(o, 1, gamma=0.5).optimizer.param_groups:
        assert g["count"].tolist() == [2, 0]


def test_a_graph_that_needs_the_old_values_is_told():
    p = torch.nn.Parameter(torch.ones(10, device="cuda"))
    loss = (p * p).sum()
    o = optim.AdamW([p])
    p.grad = torch.ones(10, device="cuda")
    o.step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_the_same_in_python(monkeypatch):
    """The marshalling in Python, where the compiled module does not serve the call."""
    for bits in (8, 32):
        a, b = Case(SIZES, bits, low_param=True, master=True), Case(SIZES, bits, low_param=True, master=True)
        a.run()
        with monkeypatch.context() as patch:
            patch.setattr(B, "_native", B._NoMarshal)
            b.run()
        for name in ("params", "m", "v", "master") + (("m_scale", "v_scale") if bits == 8 else ()):
            assert all(torch.equal(x, y) for x, y in zip(getattr(a, name), getattr(b, name))), name


def test_refusals():
    f, h = torch.ones(300, device="cuda"), torch.ones(300, device="cuda").bfloat16()
    m, v, s, count = torch.zeros_like(f), torch.zeros_like(f), torch.zeros(2, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    m8, v8 = m.to(torch.int8), v.to(torch.uint8)
    step = lambda *a, **k: B.ss_adamw_step(*a, count, 1e-3, **k)
    step([f], [f.clone()], [m], [v])
    with pytest.raises(ValueError, match="twice"):
        step([f, f], [m, m], [m, m.clone()], [v, v.clone()])
    with pytest.raises(ValueError):
        step([f], [], [m], [v])
    with pytest.raises(ValueError):
        step([f], [f[:5]], [m], [v])
    with pytest.raises(ValueError):
        step([f[::2]], [f[:150]], [m[:150]], [v[:150]])
    with pytest.raises(ValueError):
        step([f], [f], [m8], [v8], m_scale=[s])
    with pytest.raises(TypeError):
        step([f], [f], [m8], [v8])
    with pytest.raises(ValueError):
        step([f], [f], [m8], [v8], m_scale=[s[:1]], v_scale=[s])
    with pytest.raises(TypeError):
        step([f], [f], [m], [v], master=[f.clone()])
    with pytest.raises(TypeError):
        step([f.half()], [f], [m], [v])
    with pytest.raises(ValueError):
        B.ss_adamw_step([f], [f], [m], [v], count[:1], 1e-3)
    with pytest.raises(ValueError):
        B.ss_adamw_step([f], [f], [m], [v], count, torch.ones(2, device="cuda"))
    for bad in (dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(weight_decay=float("nan"))):
        with pytest.raises(B.SsError):
            step([f], [f], [m], [v], **bad)
    with pytest.raises(B.SsError):
        B.ss_adamw_step([f], [f], [m], [v], count, float("inf"))
    with pytest.raises(TypeError):
        B.ss_adamw_values(f, s)
    with pytest.raises(ValueError):
        B.ss_adamw_values(m8, s[:1])
    with pytest.raises(ValueError):
        optim.AdamW([torch.nn.Parameter(torch.ones(3))])
    with pytest.raises(ValueError):
        optim.AdamW([torch.nn.Parameter(f)], state_bits=16)
    assert count.tolist() == [1, 0]
