"""The operators around the selective scan whose speed matters to a user: layer norm with its residual sum, the gated
linear recurrence, and products in 8-bit integers; the sizes they have in use, and what one pass of each is.

A case is a dict of plain values.  Its ``kind`` says which call one pass stands for:

  norm_fwd    binding.ss_norm_fwd: residual sum and norm of (batch * seqlen) tokens, without gradients
  norm_train  autograd.layer_norm and the gradients of all inputs
  gate_fwd    binding.ss_gate_fwd, the last state returned (a prompt)
  gate_train  autograd.gated_recurrence and the gradients of all inputs
  gate_step   binding.ss_gate_step, one token
  linear      binding.ss_qlinear: tokens brought to 8 bits, times weights held in 8 bits

Where ``own`` is false the same results come from elementary torch operations in float32.
Activations are unit normal (tokens of a residual stream: with a few wide channels, as trained models have them), weights
fan-in scaled; decay logits have a bias that spreads the memory of the channels from a few steps to thousands.
"""
import math

import torch

own = False

_EPS = 1e-5
_LEAST = 2.0 ** -120   # a token whose largest magnitude is below this counts as zero


def _case(kind, batch, seqlen, dim, dtype, **options):
    c = {"kind": kind, "batch": batch, "seqlen": seqlen, "dim": dim, "dtype": dtype}
    if kind.startswith("norm"):
        c.update({"residual": "", "bias": True})
    elif kind.startswith("gate"):
        c.update({"input_gate": True, "z": True, "resets": 0, "h0": False})
    else:
        c.update({"features": dim, "x_seq_last": False, "out_seq_last": False, "bias": False})
    c.update(options)
    return c


def _named(name, case):
    return {"name": name, **case}


def listed():
    return [
        # one token of a single user: the norm before a layer of model width 2048; latency
        _named("norm_token", _case("norm_fwd", 1, 1, 2048, "bf16", residual="bf16")),
        # a prompt's tokens with the residual stream kept in float32
        _named("norm_prompt", _case("norm_fwd", 8, 2048, 2048, "bf16", residual="f32")),
        # training at context 2048
        _named("norm_train_2048", _case("norm_train", 8, 2048, 2048, "bf16", residual="bf16")),
        # documents as they come, in float32, a width that is no multiple of anything
        _named("norm_train_odd_fp32", _case("norm_train", 3, 1733, 1021, "f32")),
        # generation for a served batch at inner width 4096
        _named("gate_step_b64", _case("gate_step", 64, 1, 4096, "bf16")),
        # a prompt of any length, continued from an earlier state
        _named("gate_prompt_l1531", _case("gate_fwd", 4, 1531, 4096, "bf16", h0=True)),
        # training at inner width 4096, context 2048
        _named("gate_train_4096", _case("gate_train", 8, 2048, 4096, "bf16")),
        # documents packed into rows of odd length: the state is reset at their boundaries
        _named("gate_train_packed_fp32", _case("gate_train", 2, 4097, 768, "f32", resets=12)),
        # a sequence of 2^20 symbols: few rows, split along the sequence
        _named("gate_train_1m_fp32", _case("gate_train", 1, 1048576, 256, "f32", z=False)),
        # one token through the input projection 2048 -> 2 * 4096: latency and the weights' bytes
        _named("linear_token", _case("linear", 1, 1, 2048, "bf16", features=8192)),
        # a prompt batch through the same projection, results with the sequence last for the recurrence
        _named("linear_prompt_in", _case("linear", 8, 2048, 2048, "bf16", features=8192, out_seq_last=True)),
        # the output projection of prompts of odd length: sequence last in, tokens first out
        _named("linear_prompt_out", _case("linear", 4, 1531, 4096, "bf16", features=2048, x_seq_last=True, bias=True)),
    ]


def _log_int(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _length(rng, low, high):
    """Half of them multiples of 64 (contexts of training runs), half as they come (prompts, documents)."""
    n = _log_int(rng, low, high)
    return max(low, n // 64 * 64) if rng.random() < 0.5 and n >= 64 else n


def _width(rng, low, high):
    """Mostly multiples of 64, some of 16, a few as they come."""
    n, r = _log_int(rng, low, high), rng.random()
    step = 64 if r < 0.7 else (16 if r < 0.9 else 1)
    return max(low, n // step * step)


def _shrink(c, cost, most):
    """Halve batch, then length, then width until the case fits."""
    while cost(c) > most:
        key = "batch" if c["batch"] > 1 else ("seqlen" if c["seqlen"] > 256 else "dim")
        c[key] = max(1, c[key] // 2)
    return c


def _elements(c):
    return c["batch"] * c["seqlen"] * c["dim"]


def draw(rng):
    c = _draw(rng)
    for key in ("seqlen", "dim", "features"):   # no configuration has a size of 3072
        if c.get(key) == 3072:
            c[key] -= 64
    return c


def _draw(rng):
    kind = rng.choice(("norm_fwd", "norm_train", "gate_fwd", "gate_train", "gate_train", "gate_step", "linear", "linear"))
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    if kind.startswith("norm"):
        c = _case(kind, _log_int(rng, 1, 16), _length(rng, 1, 8192), _width(rng, 64, 16384), dtype,
                  residual=rng.choice(("", dtype, "f32")), bias=rng.random() < 0.7)
        return _shrink(c, _elements, 6e7)
    if kind == "gate_step":
        return _case(kind, _log_int(rng, 1, 256), 1, _width(rng, 256, 5120), dtype, input_gate=rng.random() < 0.8, z=rng.random() < 0.7)
    if kind.startswith("gate"):
        c = _case(kind, _log_int(rng, 1, 16), _length(rng, 16, 262144), _width(rng, 64, 5120), dtype,
                  input_gate=rng.random() < 0.8, z=rng.random() < 0.6, h0=rng.random() < 0.3)
        _shrink(c, _elements, 1.2e8)
        if rng.random() < 0.3:
            c["resets"] = _log_int(rng, 1, 1 + c["seqlen"] // 16)
        return c
    c = _case(kind, _log_int(rng, 1, 16), 1 if rng.random() < 0.4 else _length(rng, 2, 4096), _width(rng, 256, 5120), dtype,
              features=_width(rng, 256, 10240), bias=rng.random() < 0.3)
    if c["seqlen"] > 1:
        c["x_seq_last"], c["out_seq_last"] = rng.choice(((False, False), (False, True), (True, False), (True, True)))
    else:
        c["batch"] = _log_int(rng, 1, 256)
    return _shrink(c, lambda c: _elements(c) * c["features"], 2.7e11)


# ---- inputs ----------------------------------------------------------------------------------------
class _Draws:
    """Tensors on the GPU from one generator, in a fixed order."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32).to(dtype)

    def uniform(self, low, high, *shape, dtype=torch.float32):
        return torch.empty(shape, device="cuda", dtype=torch.float32).uniform_(low, high, generator=self.g).to(dtype)

    def places(self, n, *shape):
        return torch.randint(0, n, shape, generator=self.g, device="cuda")


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _stream(r, dim):
    """Scales of the channels of a residual stream: one, and for one in 64 up to eight."""
    return 1.0 + 7.0 * r.uniform(0, 1, dim) * (r.uniform(0, 1, dim) < 1 / 64)


def _norm_inputs(c, r, io):
    nb, nl, nd = c["batch"], c["seqlen"], c["dim"]
    wide = _stream(r, nd)
    t = {"x": (r.normal(nb, nl, nd) * wide).to(io)}
    if c["residual"]:
        t["residual"] = (2.0 * r.normal(nb, nl, nd) * wide).to(_type(c["residual"]))
    t["weight"] = 1.0 + 0.1 * r.normal(nd)
    if c["bias"]:
        t["bias"] = 0.1 * r.normal(nd)
    return t


def _gate_inputs(c, r, io):
    nb, nl, nd = c["batch"], c["seqlen"], c["dim"]
    shape = (nb, nd) if c["kind"] == "gate_step" else (nb, nd, nl)
    t = {"x": r.normal(*shape, dtype=io), "f": r.normal(*shape, dtype=io)}
    if c["input_gate"]:
        t["i"] = r.normal(*shape, dtype=io)
    if c["z"]:
        t["z"] = r.normal(*shape, dtype=io)
    # a = exp(-rate sigmoid(f + f_bias)): at f = 0 between 0.9 and 0.999
    half = -torch.log(r.uniform(0.9, 0.999, nd))
    t["rate"] = r.uniform(0.5, 2.0, nd)
    t["f_bias"] = torch.logit(half / t["rate"])
    if c["input_gate"]:
        t["i_bias"] = 0.5 * r.normal(nd)
    if c["h0"]:
        t["h0"] = 0.5 * r.normal(nb, nd)
    return t


def _quantised(w):
    """Rows of w in 8 bits with a scale each; their pitch is a whole number of 128 bytes, filled with zeros."""
    amax = w.abs().amax(1)
    q = torch.zeros(w.shape[0], (w.shape[1] + 127) // 128 * 128, dtype=torch.int8, device=w.device)
    q[:, : w.shape[1]] = torch.round(w * (127.0 / amax)[:, None]).to(torch.int8)
    return q, amax / 127.0


def prepare(case, seed):
    r, io, kind = _Draws(seed), _type(case["dtype"]), case["kind"]
    nb, nl, nd = case["batch"], case["seqlen"], case["dim"]
    s = {"case": case}
    if kind == "linear":
        shape = (nb, nd, nl) if case["x_seq_last"] else (nb, nl, nd)
        wide = _stream(r, nd)
        x = r.normal(*shape) * (wide[:, None] if case["x_seq_last"] else wide)
        s["q"], s["scale"] = _quantised(r.normal(case["features"], nd) * nd ** -0.5)
        s["x"] = x.to(io)
        s["bias"] = 0.1 * r.normal(case["features"]) if case["bias"] else None
        return s
    s["t"] = t = _norm_inputs(case, r, io) if kind.startswith("norm") else _gate_inputs(case, r, io)
    if kind == "gate_step":
        s["h"] = r.normal(nb, nd)
    elif kind.startswith("gate") and case["resets"]:
        s["reset"] = torch.zeros(nb, nl, dtype=torch.bool, device="cuda")
        s["reset"].scatter_(1, r.places(nl, nb, case["resets"]), True)
    if kind == "norm_train":
        s["dout"] = r.normal(nb, nl, nd, dtype=io)
        if case["residual"]:
            s["dsummed"] = r.normal(nb, nl, nd, dtype=_type(case["residual"]))
    elif kind == "gate_train":
        s["dout"] = r.normal(nb, nd, nl, dtype=io)
    if kind.endswith("train"):
        for v in t.values():
            v.requires_grad_(True)
    return s


# ---- the plain forms ---------------------------------------------------------------------------------
def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _plain_norm(t):
    x = t["x"]
    s = x if "residual" not in t else (x.float() + t["residual"].float()).to(t["residual"].dtype)
    v = s.float()
    v = v - v.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((v * v).mean(-1, keepdim=True) + _EPS)
    xhat = v * rstd
    out = xhat * t["weight"]
    if "bias" in t:
        out = out + t["bias"]
    return out.to(x.dtype), s, xhat, rstd


def _plain_norm_train(state):
    t, io = state["t"], state["dout"].dtype
    out, s, xhat, rstd = _plain_norm(t)
    dout = state["dout"].float()
    g = dout * t["weight"]
    ds = rstd * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
    res = [out]
    grads = [ds.to(io)]
    if "residual" in t:
        ds = ds + state["dsummed"].float()
        res.append(s)
        grads = [ds.to(io), ds.to(s.dtype)]
    grads.append((dout * xhat).sum((0, 1)))
    if "bias" in t:
        grads.append(dout.sum((0, 1)))
    return res + grads


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the last axis, from zero: spans doubled until they reach the whole length."""
    k, n = 1, a.shape[-1]
    a, b = a.clone(), b.clone()
    while k < n:
        b[..., k:] += a[..., k:] * b[..., :-k]
        a[..., k:] = a[..., k:] * a[..., :-k]
        k *= 2
    return b


def _column(v, like):
    return v.reshape(-1, *([1] * (like.dim() - 2)))


def _plain_gates(t, reset=None):
    """a, m, g, sigmoid(f) of every step in float32."""
    f = t["f"].float()
    sg = _sigmoid(f + _column(t["f_bias"], f))
    la = -_column(t["rate"], f) * sg
    a, m = torch.exp(la), torch.sqrt(-torch.expm1(2.0 * la))
    if reset is not None:
        a, m = a.masked_fill(reset[:, None], 0.0), m.masked_fill(reset[:, None], 1.0)
    g = _sigmoid(t["i"].float() + _column(t["i_bias"], f)) if "i" in t else None
    return a, m, g, sg


def _plain_gate(t, reset=None):
    a, m, g, sg = _plain_gates(t, reset)
    x = t["x"].float()
    b = m * x if g is None else m * g * x
    if "h0" in t:
        b[..., 0] += a[..., 0] * t["h0"]
    h = _scan(a, b)
    out = h
    if "z" in t:
        z = t["z"].float()
        out = h * z * _sigmoid(z)
    return out.to(t["x"].dtype), h, (a, m, g, sg)


def _plain_gate_train(state):
    t, reset, dout = state["t"], state.get("reset"), state["dout"].float()
    io = state["dout"].dtype
    out, h, (a, m, g, sg) = _plain_gate(t, reset)
    rate = _column(t["rate"], a)
    grads = {}
    if "z" in t:
        z = t["z"].float()
        sz = _sigmoid(z)
        grads["z"] = (dout * h * sz * (1.0 + z * (1.0 - sz))).to(io)
        dout = dout * z * sz
    # the adjoint runs backwards: lam_t = dout_t + a_{t+1} lam_{t+1}
    later = torch.cat((a[..., 1:], torch.zeros_like(a[..., :1])), -1)
    lam = _scan(later.flip(-1), dout.flip(-1)).flip(-1)
    del later, dout
    first = t["h0"][..., None] if "h0" in t else torch.zeros_like(h[..., :1])
    x = t["x"].float()
    dm = lam * x if g is None else lam * x * g
    grads["x"] = (lam * m if g is None else lam * m * g).to(io)
    if g is not None:
        di = lam * m * x * g * (1.0 - g)
        grads["i"], grads["i_bias"] = di.to(io), di.sum((0, 2))
        del di
    inner = dm * a * a / m
    dla = lam * torch.cat((first, h[..., :-1]), -1) * a - inner
    if reset is not None:
        dla = dla.masked_fill(reset[:, None], 0.0)
    del inner, dm
    grads["rate"] = -(dla * sg).sum((0, 2))
    df = -dla * rate * sg * (1.0 - sg)
    grads["f"], grads["f_bias"] = df.to(io), df.sum((0, 2))
    if "h0" in t:
        grads["h0"] = lam[..., 0] * a[..., 0]
    return [out] + [grads[k] for k in t]


def _plain_gate_step(state):
    t = state["t"]
    f = t["f"].float()
    sg = _sigmoid(f + t["f_bias"])
    la = -t["rate"] * sg
    b = torch.sqrt(-torch.expm1(2.0 * la)) * t["x"].float()
    if "i" in t:
        b = b * _sigmoid(t["i"].float() + t["i_bias"])
    state["h"].copy_(torch.exp(la) * state["h"] + b)
    out = state["h"]
    if "z" in t:
        z = t["z"].float()
        out = out * z * _sigmoid(z)
    return [out.to(t["x"].dtype), state["h"]]


def _plain_linear(state):
    case, x, io = state["case"], state["x"].float(), state["x"].dtype
    if case["x_seq_last"]:
        x = x.transpose(1, 2)
    amax = x.abs().amax(-1, keepdim=True)
    some = amax >= _LEAST
    q = torch.round(x * torch.where(some, 127.0 / amax, torch.zeros_like(amax)))
    scale = torch.where(some, amax / 127.0, torch.zeros_like(amax))
    w = state["q"][:, : case["dim"]].float()
    out = torch.matmul(q, w.t()) * (scale * state["scale"])
    if state["bias"] is not None:
        out = out + state["bias"]
    out = out.to(io)
    return out.transpose(1, 2).contiguous() if case["out_seq_last"] else out


# ---- one pass ----------------------------------------------------------------------------------------
def _run_plain(state):
    kind = state["case"]["kind"]
    with torch.no_grad():
        if kind == "linear":
            return _plain_linear(state)
        if kind == "norm_fwd":
            out, s, _, _ = _plain_norm(state["t"])
            return [out, s] if "residual" in state["t"] else [out]
        if kind == "norm_train":
            return _plain_norm_train(state)
        if kind == "gate_fwd":
            out, h, _ = _plain_gate(state["t"], state.get("reset"))
            return [out, h[..., -1].clone()]
        if kind == "gate_train":
            return _plain_gate_train(state)
        return _plain_gate_step(state)


def run(state):
    if not own:
        return _run_plain(state)
    from paper_2312_00752_amd import autograd
    from paper_2312_00752_amd import binding as B
    case, t = state["case"], state.get("t")
    kind = case["kind"]
    if kind == "linear":
        return B.ss_qlinear(state["x"], state["q"], state["scale"], bias=state["bias"], x_seq_last=case["x_seq_last"],
                            out_seq_last=case["out_seq_last"])
    if kind == "norm_fwd":
        out, summed, _ = B.ss_norm_fwd(t["x"], t["weight"], t.get("bias"), residual=t.get("residual"), eps=_EPS)
        return [out] if summed is None else [out, summed]
    if kind == "norm_train":
        res = autograd.layer_norm(t["x"], t["weight"], t.get("bias"), residual=t.get("residual"), eps=_EPS)
        outs, douts = (res, [state["dout"], state["dsummed"]]) if "residual" in t else ([res], [state["dout"]])
        return [v.detach() for v in outs] + list(torch.autograd.grad(outs, list(t.values()), douts))
    if kind == "gate_step":
        out = B.ss_gate_step(state["h"], t["x"], t["f"], t["rate"], i_t=t.get("i"), z_t=t.get("z"), f_bias=t["f_bias"],
                             i_bias=t.get("i_bias"))
        return [out, state["h"]]
    args = dict(i=t.get("i"), z=t.get("z"), f_bias=t["f_bias"], i_bias=t.get("i_bias"), reset=state.get("reset"), h0=t.get("h0"))
    if kind == "gate_fwd":
        return list(B.ss_gate_fwd(t["x"], t["f"], t["rate"], return_last_state=True, **args))
    out = autograd.gated_recurrence(t["x"], t["f"], t["rate"], **args)
    return [out.detach(), *torch.autograd.grad(out, list(t.values()), state["dout"])]


# ---- what a pass cannot do without -------------------------------------------------------------------
def work(case):
    """Inputs read once, outputs written once; flops as the formulas have them (an exponential counts as one)."""
    kind, nd, dtype = case["kind"], case["dim"], case["dtype"]
    esz, n = (2 if dtype == "bf16" else 4), _elements(case)
    rows = case["batch"] * case["seqlen"]
    if kind == "linear":
        nf = case["features"]
        return {"bytes": esz * rows * (nd + nf) + nf * (nd + 4 + (4 if case["bias"] else 0)), "flops": 2 * rows * nd * nf}
    if kind.startswith("norm"):
        rsz = {"": 0, "bf16": 2, "f32": 4}[case["residual"]]
        par = 4 * nd * (2 if case["bias"] else 1)
        if kind == "norm_fwd":
            return {"bytes": n * (2 * esz + 2 * rsz) + par, "flops": 8 * n}
        return {"bytes": n * (4 * esz + 4 * rsz) + 2 * par, "flops": 20 * n}
    tensors = 2 + int(case["input_gate"]) + int(case["z"])
    gates = 12 + 6 * int(case["input_gate"]) + 6 * int(case["z"])
    par = 4 * nd * (3 if case["input_gate"] else 2)
    state = 4 * case["batch"] * nd
    if kind == "gate_step":
        return {"bytes": n * esz * (tensors + 1) + par + 2 * state, "flops": gates * n}
    start = state if case["h0"] else 0
    marks = rows if case["resets"] else 0
    if kind == "gate_fwd":
        return {"bytes": n * esz * (tensors + 1) + par + start + marks + state, "flops": gates * n}
    return {"bytes": n * esz * (2 * tensors + 2) + 2 * (par + start) + marks, "flops": 3 * gates * n}


# ---- the definitions in 64 bits ------------------------------------------------------------------------
def _exact_norm(case, s):
    t = {k: v.detach().double().requires_grad_(True) for k, v in s["t"].items()}
    summed = None
    if "residual" in t:
        summed = t["x"] + t["residual"]
        held = s["t"]["residual"].dtype   # what is normalised is the sum as it is held
        summed = summed + (summed.detach().to(held).double() - summed.detach())
    v = t["x"] if summed is None else summed
    var, mean = torch.var_mean(v, -1, correction=0, keepdim=True)
    out = (v - mean) * torch.rsqrt(var + _EPS) * t["weight"]
    if "bias" in t:
        out = out + t["bias"]
    outs = [out] if summed is None else [out, summed]
    if case["kind"] == "norm_fwd":
        return [v.detach() for v in outs]
    douts = [s["dout"].double()] + ([s["dsummed"].double()] if summed is not None else [])
    return [v.detach() for v in outs] + list(torch.autograd.grad(outs, list(t.values()), douts))


def _recurrence(a, b, carry, backwards=False):
    """Step by step within pieces, the pieces side by side; then the pieces one after another. (rows, L), carry (rows)."""
    rows, n = a.shape
    c = max(1, math.isqrt(n))
    m = -(-n // c)
    pad = m * c - n
    side = (pad, 0) if backwards else (0, pad)
    a = torch.nn.functional.pad(a, side, value=1.0).reshape(rows, m, c).permute(2, 0, 1).contiguous()
    h = torch.nn.functional.pad(b, side).reshape(rows, m, c).permute(2, 0, 1).contiguous()
    at = range(c - 1, -1, -1) if backwards else range(c)
    last = None
    for k in at:
        if last is not None:
            h[k] += a[k] * h[last]
            a[k] *= a[last]
        last = k
    starts = torch.empty(rows, m, dtype=a.dtype, device=a.device)
    for j in range(m - 1, -1, -1) if backwards else range(m):
        starts[:, j] = carry
        carry = h[last, :, j] + a[last, :, j] * carry
    h += a * starts
    h = h.permute(1, 2, 0).reshape(rows, m * c)
    return h[:, pad:] if backwards else h[:, :n]


def _exact_gate(case, s):
    with torch.no_grad():
        t, step = s["t"], case["kind"] == "gate_step"
        shape = t["x"].shape
        three = lambda v: v.detach().double().reshape(shape[0], shape[1], -1)  # noqa: E731
        row = lambda k: t[k].detach().double()[None, :, None]  # noqa: E731
        sf = torch.sigmoid(three(t["f"]) + row("f_bias"))
        alpha = -row("rate") * sf
        a = torch.exp(alpha)
        m2 = -torch.expm1(2 * alpha)
        keep = None if s.get("reset") is None else (~s["reset"]).double()[:, None]
        if keep is not None:
            a = a * keep
            m2 = 1 - keep * (1 - m2)
        m = torch.sqrt(m2)
        gi = torch.sigmoid(three(t["i"]) + row("i_bias")) if "i" in t else torch.ones_like(a[..., :1])
        x = three(t["x"])
        rows, n = shape[0] * shape[1], x.shape[-1]
        start = s["h"] if step else t.get("h0")
        start = torch.zeros(rows, dtype=torch.float64, device=a.device) if start is None else start.detach().double().reshape(rows)
        flat = lambda v: v.expand(shape[0], shape[1], n).reshape(rows, n)  # noqa: E731
        h = _recurrence(flat(a), flat(m * gi * x), start).reshape(x.shape)
        y, z = h, None
        if "z" in t:
            z = three(t["z"])
            silu = z * torch.sigmoid(z)
            y = h * silu
        if case["kind"] != "gate_train":
            return [y.reshape(shape), h[..., -1]]
        dout = three(s["dout"])
        res = {"x": None}
        dy = dout
        if z is not None:
            sz = torch.sigmoid(z)
            res["z"] = dout * h * (sz + z * sz * (1 - sz))
            dy = dout * silu
        ahead = torch.cat((a[..., 1:], torch.ones_like(a[..., :1])), -1)
        lam = _recurrence(flat(ahead), flat(dy), torch.zeros_like(start), backwards=True).reshape(x.shape)
        del ahead, dy
        before = torch.cat((start.reshape(shape[0], shape[1], 1), h[..., :-1]), -1)
        res["x"] = lam * m * gi
        if "i" in t:
            res["i"] = lam * m * x * gi * (1 - gi)
            res["i_bias"] = res["i"].sum((0, 2))
        dalpha = lam * (before * a - gi * x * a * a / m)
        if keep is not None:
            dalpha = dalpha * keep
        res["f"] = dalpha * alpha * (1 - sf)
        res["f_bias"] = res["f"].sum((0, 2))
        res["rate"] = -(dalpha * sf).sum((0, 2))
        if "h0" in t:
            res["h0"] = (lam * a)[..., 0]
        return [y] + [res[k] for k in t]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("norm"):
        return _exact_norm(case, s)
    if case["kind"].startswith("gate"):
        return _exact_gate(case, s)
    x = s["x"].double()
    if case["x_seq_last"]:
        x = x.mT
    top = x.abs().amax(-1, keepdim=True)
    top = torch.where(top < _LEAST, torch.inf, top)
    q = torch.round(127.0 * x / top)
    w = s["q"][:, : case["dim"]].double() * s["scale"].double()[:, None]
    out = (q.reshape(-1, case["dim"]) @ w.t()).reshape(*x.shape[:-1], -1)
    out = out * torch.where(torch.isinf(top), 0.0, top / 127.0)
    if s["bias"] is not None:
        out = out + s["bias"].double()
    return out.mT if case["out_seq_last"] else out
