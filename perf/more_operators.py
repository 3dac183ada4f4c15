"""The operators at the two ends of a model of the library's blocks and in its training step, whose speed matters to a user: root-mean-square
norm (also with an 8-bit output), embedding, log probabilities of tokens, AdamW; the sizes they have in use, and what one pass of each is.

A case is a dict of plain values.  Its ``kind`` says which call one pass stands for:

  rms_q8         binding.ss_norm_quant: residual sum, RMS norm, result in 8 bits with a scale a token (given back as the values it stands for)
  rms_train      autograd.rms_norm and the gradients of all inputs
  embed_fwd      binding.ss_embed_fwd: rows of a table for token ids
  embed_train    autograd.embedding and the table's gradient
  logprob_top    binding.ss_logprob_fwd: log probability of the token taken, entropy, the most probable alternatives
  logprob_train  autograd.token_logprobs and the logits' gradient
  adamw          binding.ss_adamw_step over the tensors of a stack of blocks; 8-bit states are given back as the values they stand for

Where ``own`` is false the same results come from elementary torch operations in float32.
Activations are unit normal with a few wide channels, token ids have frequencies that fall as one over their rank, logits are
what a trained model's are: a wide normal with a few large ones, gradients and moments differ in size from tensor to tensor.
"""
import math

import torch

own = False

_EPS = 1e-5
_LEAST = 2.0 ** -120   # a token whose largest magnitude is below this counts as zero in 8 bits
_BLOCK = 256           # values of an 8-bit state that share a scale
_LEAST_STATE = 2.0 ** -100
_LR, _BETA1, _BETA2, _ADAM_EPS, _DECAY = 3e-4, 0.9, 0.95, 1e-8, 0.1
# fractional parts of the square roots of 2, 3, 5 and 7 in 2^-32
_WEYL = (0x6A09E667, 0xBB67AE85, 0x3C6EF372, 0xA54FF53A)


def _norm_case(kind, batch, seqlen, dim, dtype, residual=""):
    return {"kind": kind, "batch": batch, "seqlen": seqlen, "dim": dim, "dtype": dtype, "residual": residual}


def _embed_case(kind, tokens, vocab, dim, table, dtype, padded=False):
    return {"kind": kind, "tokens": tokens, "vocab": vocab, "dim": dim, "table": table, "dtype": dtype, "padded": padded}


def _logprob_case(kind, rows, vocab, dtype, **options):
    c = {"kind": kind, "rows": rows, "vocab": vocab, "dtype": dtype, "padding": 0, "masked": False}
    c.update({"top": 8} if kind == "logprob_top" else {"entropy": False, "ignored": False})
    c.update(options)
    return c


def _adamw_case(layers, width, dtype, bits):
    return {"kind": "adamw", "layers": layers, "width": width, "dtype": dtype, "bits": bits}


def listed():
    return [
        # one token of a single user before the 8-bit projection of a block of width 2048; latency
        {"name": "rms_q8_token", **_norm_case("rms_q8", 1, 1, 2048, "bf16", "bf16")},
        # a prompt's tokens before the same projection, with the residual stream kept in float32
        {"name": "rms_q8_prompt", **_norm_case("rms_q8", 8, 2048, 2048, "bf16", "f32")},
        # training at context 2048
        {"name": "rms_train_2048", **_norm_case("rms_train", 8, 2048, 2048, "bf16", "bf16")},
        # generation for a served batch: one id each
        {"name": "embed_token_b64", **_embed_case("embed_fwd", 64, 51200, 2048, "bf16", "bf16")},
        # training at context 2048: a float32 table read in bf16, and its whole gradient
        {"name": "embed_train_2048", **_embed_case("embed_train", 16384, 51200, 2048, "f32", "bf16")},
        # bytes as tokens, documents of odd lengths padded at their ends: few rows that each have many tokens
        {"name": "embed_train_bytes_fp32", **_embed_case("embed_train", 5199, 257, 1021, "f32", "f32", padded=True)},
        # generation for a served batch: the sampled token's log probability with eight alternatives
        {"name": "logprob_top8_b64", **_logprob_case("logprob_top", 64, 51200, "bf16")},
        # a single user's token in float32, a vocabulary of which a grammar leaves a part; latency
        {"name": "logprob_top_token_fp32", **_logprob_case("logprob_top", 1, 50021, "f32", top=20, masked=True)},
        # the loss of training at context 2048: logits of four rows at a time
        {"name": "logprob_train_2048", **_logprob_case("logprob_train", 8192, 51200, "bf16")},
        # an objective with an entropy term on answers only, logits of a padded vocabulary in float32
        {"name": "logprob_train_odd_fp32", **_logprob_case("logprob_train", 777, 50021, "f32", entropy=True, ignored=True, padding=27)},
        # the block of the recall task: tensors of a few hundred to a hundred thousand values; latency
        {"name": "adamw_small", **_adamw_case(1, 128, "f32", 32)},
        # blocks of width 2048 in bf16 with a float32 copy to update, states in 8 bits
        {"name": "adamw_8bit_2048", **_adamw_case(3, 2048, "bf16", 8)},
    ]


def _log_int(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _width(rng, low, high):
    """Mostly multiples of 64, some of 16, a few as they come."""
    n, r = _log_int(rng, low, high), rng.random()
    step = 64 if r < 0.7 else (16 if r < 0.9 else 1)
    return max(low, n // step * step)


def _shrink(c, keys, most):
    """Halve the first of the keys that is not yet small until their product fits."""
    while math.prod(c[k] for k in keys) > most:
        key = next((k for k in keys if c[k] > 256), keys[-1])
        c[key] //= 2
    return c


def draw(rng):
    kind = rng.choice(("rms_q8", "rms_train", "embed_fwd", "embed_train", "logprob_top", "logprob_train", "adamw", "adamw"))
    dtype = "bf16" if rng.random() < 0.6 else "f32"
    if kind.startswith("rms"):
        c = _norm_case(kind, _log_int(rng, 1, 16), _log_int(rng, 1, 8192), _width(rng, 64, 16384), dtype, rng.choice(("", dtype, "f32")))
        return _shrink(c, ("seqlen", "batch", "dim"), 3.3e7)
    if kind.startswith("embed"):
        table = "bf16" if dtype == "bf16" and rng.random() < 0.5 else "f32"
        c = _embed_case(kind, _log_int(rng, 1, 65536), _log_int(rng, 256, 131072), _width(rng, 64, 8192), table, dtype, rng.random() < 0.3)
        return _shrink(_shrink(c, ("vocab", "dim"), 1.0e8), ("tokens", "dim"), 3.3e7)
    if kind == "logprob_top":
        c = _logprob_case(kind, _log_int(rng, 1, 256), _log_int(rng, 256, 262144), dtype, top=rng.choice((1, 5, 8, 20, 32)),
                          padding=rng.choice((0, 0, 27, 64)), masked=rng.random() < 0.4)
        return _shrink(c, ("rows", "vocab"), 2.0e7)
    if kind == "logprob_train":
        c = _logprob_case(kind, _log_int(rng, 1, 16384), _log_int(rng, 256, 262144), dtype, entropy=rng.random() < 0.4,
                          ignored=rng.random() < 0.5, padding=rng.choice((0, 0, 27, 64)), masked=rng.random() < 0.2)
        return _shrink(c, ("rows", "vocab"), 1.0e8)
    return _adamw_case(_log_int(rng, 1, 6), _width(rng, 16, 1280), dtype, rng.choice((8, 32)))


# ---- inputs ----------------------------------------------------------------------------------------
class _Draws:
    """Tensors on the GPU from one generator, in a fixed order."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32).to(dtype)

    def uniform(self, low, high, *shape):
        return torch.empty(shape, device="cuda", dtype=torch.float32).uniform_(low, high, generator=self.g)

    def tokens(self, vocab, *shape):
        """Ids whose frequency falls as one over their rank."""
        return (torch.exp(self.uniform(0, math.log(vocab + 1), *shape)) - 1).long().clamp_(0, vocab - 1)


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _prepare_norm(c, r):
    nb, nl, nd, io = c["batch"], c["seqlen"], c["dim"], _type(c["dtype"])
    wide = 1.0 + 7.0 * r.uniform(0, 1, nd) * (r.uniform(0, 1, nd) < 1 / 64)
    t = {"x": (r.normal(nb, nl, nd) * wide).to(io)}
    if c["residual"]:
        t["residual"] = (2.0 * r.normal(nb, nl, nd) * wide).to(_type(c["residual"]))
    t["weight"] = 1.0 + 0.1 * r.normal(nd)
    s = {"t": t}
    if c["kind"] == "rms_train":
        s["dout"] = r.normal(nb, nl, nd, dtype=io)
        if c["residual"]:
            s["dsummed"] = r.normal(nb, nl, nd, dtype=_type(c["residual"]))
        for v in t.values():
            v.requires_grad_(True)
    return s


def _prepare_embed(c, r):
    s = {"table": r.normal(c["vocab"], c["dim"], dtype=_type(c["table"])), "ids": r.tokens(c["vocab"], c["tokens"])}
    if c["padded"]:
        s["ids"][r.uniform(0, 1, c["tokens"]) < 0.1] = -1
    if c["kind"] == "embed_train":
        s["dout"] = r.normal(c["tokens"], c["dim"], dtype=_type(c["dtype"]))
        s["table"].requires_grad_(True)
    return s


def _prepare_logprob(c, r):
    rows, vocab, io = c["rows"], c["vocab"], _type(c["dtype"])
    x = torch.empty(rows, vocab + c["padding"], dtype=io, device="cuda")
    few = max(1, 2 ** 27 // x.shape[1])
    for k in range(0, rows, few):   # float32 values of a part at a time
        part = 3.0 * r.normal(min(few, rows - k), x.shape[1])
        x[k:k + few] = part + 12.0 * (r.uniform(0, 1, *part.shape) < 3 / vocab)
    s = {"logits": x[:, :vocab], "targets": r.tokens(vocab, rows)}
    if c["masked"]:   # what is not allowed has probability 0; the token taken is allowed
        allowed = r.uniform(0, 1, vocab) < 0.5
        allowed[s["targets"]] = True
        s["logits"].masked_fill_(~allowed, -math.inf)
    if c["kind"] == "logprob_train":
        s["dlogp"] = -r.uniform(0.5, 1.5, rows) / rows
        if c["ignored"]:
            s["targets"][r.uniform(0, 1, rows) < 0.4] = -1
        if c["entropy"]:
            s["dentropy"] = 0.1 * r.normal(rows) / rows
        s["logits"] = s["logits"].requires_grad_(True)
    return s


def _adamw_shapes(c):
    """(shapes of the float32 tensors, shapes of those of the projections' type) of a stack of blocks with an inner width of twice their width."""
    w, inner = c["width"], 2 * c["width"]
    small = [(w,), (w,), (inner,), (inner,), (inner,)] * c["layers"]
    large = [(4 * inner, w), (w, inner)] * c["layers"]
    return (small, large) if c["dtype"] == "bf16" else (small + large, [])


def _starts(shapes):
    """Where tensors of these shapes lie in one memory: each at a multiple of a block; and its end."""
    at, n = [], 0
    for s in shapes:
        at.append(n)
        n += -(-math.prod(s) // _BLOCK) * _BLOCK
    return at, n


def _prepare_arena(shapes, low, bits, r):
    """Tensors, gradients and moments side by side in one memory for each: the whole of it under "all", the tensors' parts of it under "each"."""
    at, n = _starts(shapes)
    own_size = torch.zeros(n, device="cuda")
    index = torch.zeros(n, dtype=torch.int64, device="cuda")
    used = torch.zeros(n, device="cuda")
    for s, k in zip(shapes, at):
        m = math.prod(s)
        own_size[k:k + m] = torch.exp(2.0 * r.normal(1))
        index[k:k + m] = torch.arange(m, device="cuda")
        used[k:k + m] = 1.0
    grads = 1e-3 * r.normal(n) * own_size * used
    moment = 3e-4 * r.normal(n) * own_size * used
    second = (1e-3 * own_size) ** 2 * r.uniform(0.2, 2.0, n) * used
    del own_size
    whole = {"grad": grads.to(torch.bfloat16) if low else grads, "master": 0.02 * r.normal(n) * used}
    del grads
    if low:
        whole["param"] = whole["master"].to(torch.bfloat16)
    if bits == 8:
        zero = torch.zeros((), dtype=torch.int32, device="cuda")
        whole["m"], whole["m_scale"] = _plain_encode(moment, True, index, zero)
        whole["v"], whole["v_scale"] = _plain_encode(torch.sqrt(second), False, index, zero)
    else:
        whole["m"], whole["v"] = moment, second
    each = {k: [] for k in whole}
    for s, k in zip(shapes, at):
        m = math.prod(s)
        for name, v in whole.items():
            each[name].append(v[k // _BLOCK: (k + m + _BLOCK - 1) // _BLOCK] if name.endswith("_scale") else v[k:k + m].view(s))
    return {"all": whole, "each": each, "index": index if bits == 8 else None, "low": low}


def prepare(case, seed):
    r, kind = _Draws(seed), case["kind"]
    if kind.startswith("rms"):
        s = _prepare_norm(case, r)
    elif kind.startswith("embed"):
        s = _prepare_embed(case, r)
        s["scale"] = math.sqrt(case["dim"])
    elif kind.startswith("logprob"):
        s = _prepare_logprob(case, r)
    else:
        # steps taken so far, and room for the call's own count
        s = {"count": torch.tensor([20 + seed % 1000, 0], dtype=torch.int32, device="cuda"),
             "arenas": [_prepare_arena(shapes, low, case["bits"], r) for shapes, low in zip(_adamw_shapes(case), (False, True)) if shapes]}
    s["case"] = case
    return s


# ---- the plain forms ---------------------------------------------------------------------------------
def _plain_norm(t):
    x = t["x"]
    s = x if "residual" not in t else (x.float() + t["residual"].float()).to(t["residual"].dtype)
    v = s.float()
    rstd = 1.0 / torch.sqrt((v * v).mean(-1, keepdim=True) + _EPS)
    xhat = v * rstd
    return (xhat * t["weight"]).to(x.dtype), s, xhat, rstd


def _plain_rms_q8(state):
    t = state["t"]
    out, s, _, _ = _plain_norm(t)
    out = out.float()
    amax = out.abs().amax(-1, keepdim=True)
    some = amax >= _LEAST
    q = torch.round(out * torch.where(some, 127.0 * (1.0 / amax), torch.zeros_like(amax)))
    values = (q * torch.where(some, amax / 127.0, torch.zeros_like(amax))).to(torch.bfloat16)
    return [values, s] if "residual" in t else [values]


def _plain_rms_train(state):
    t, io = state["t"], state["dout"].dtype
    out, s, xhat, rstd = _plain_norm(t)
    dout = state["dout"].float()
    g = dout * t["weight"]
    ds = rstd * (g - xhat * (g * xhat).mean(-1, keepdim=True))
    res, grads = [out], [ds.to(io)]
    if "residual" in t:
        ds = ds + state["dsummed"].float()
        res.append(s)
        grads = [ds.to(io), ds.to(s.dtype)]
    return res + grads + [(dout * xhat).sum((0, 1))]


def _plain_embed(state):
    ids, table, io = state["ids"], state["table"], _type(state["case"]["dtype"])
    there = (ids >= 0)[:, None]
    out = torch.where(there, table[ids.clamp(min=0)].float() * state["scale"], 0.0).to(io)
    if "dout" not in state:
        return [out]
    d = torch.where(there, state["dout"].float() * state["scale"], 0.0)
    grad = torch.zeros(table.shape, dtype=torch.float32, device=table.device).index_add_(0, ids.clamp(min=0), d)
    return [out, grad.to(table.dtype)]


def _plain_logprob(state):
    x, targets, case = state["logits"].float(), state["targets"], state["case"]
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    lse = top + torch.log(total)
    there = targets >= 0
    taken = x.gather(1, targets.clamp(min=0)[:, None])
    logp = torch.where(there, (taken - lse)[:, 0], 0.0)
    shifted = (x - top).masked_fill(e == 0, 0.0)
    entropy = torch.log(total)[:, 0] - (e * shifted).sum(-1) / total[:, 0]
    if case["kind"] == "logprob_top":
        values, places = torch.sort(x, dim=-1, descending=True, stable=True)
        return [logp, entropy, (values - lse)[:, :case["top"]].contiguous(), places[:, :case["top"]].contiguous()]
    del x
    p = e / total
    d = torch.where(there, state["dlogp"], 0.0)[:, None]
    dx = -(p * d)
    dx.scatter_add_(1, targets.clamp(min=0)[:, None], d)
    if "dentropy" in state:
        dx = dx - state["dentropy"][:, None] * p * (shifted - torch.log(total) + entropy[:, None])
    return [logp, entropy, dx.to(state["logits"].dtype)]


def _plain_encode(values, signed, index, step):
    """Values (not negative unless signed) in blocks: codes and scales.  A code q stands for (q / top)^2 of its block's scale; a value between two
    codes takes the upper one in a share of the steps that makes their mean the value."""
    top = 127 if signed else 255
    v = values.reshape(-1, _BLOCK)
    size = v.abs()
    scale = size.amax(1, keepdim=True)
    some = scale >= _LEAST_STATE
    y = size * torch.where(some, float(top * top) / scale, 0.0)
    q = torch.floor(torch.sqrt(y))
    a, b = _WEYL[:2] if signed else _WEYL[2:]
    u = (((index * a + step.long() * b) & 0xFFFFFFFF) >> 8).float().reshape(v.shape) * 2.0 ** -24
    q = torch.clamp(q + (y - q * q > u * (2.0 * q + 1.0)), max=top)
    if signed:
        codes = (q * torch.sign(v)).to(torch.int8)
    else:
        codes = torch.where((size > 0) & some, q.clamp(min=1.0), 0.0).to(torch.uint8)
    return codes.reshape(-1), torch.where(some, scale, 0.0)[:, 0].contiguous()


def _plain_decode(codes, scale):
    top = 127 if codes.dtype == torch.int8 else 255
    q = codes.float().reshape(-1, _BLOCK)
    return (q * q.abs() * (scale * (1.0 / (top * top)))[:, None]).reshape(-1)


def _plain_adamw(state):
    count = state["count"]
    count[0] += 1
    t = count[0].double()
    c1, c2 = 1.0 - torch.pow(_BETA1, t), 1.0 - torch.pow(_BETA2, t)
    rate, root = (_LR / c1).float(), torch.sqrt(c2).float()
    res = []
    for arena in state["arenas"]:
        w = arena["all"]
        g, low, eight = w["grad"].float(), arena["low"], arena["index"] is not None
        m = _plain_decode(w["m"], w["m_scale"]) if eight else w["m"]
        m = m * _BETA1 + g * (1.0 - _BETA1)
        v = torch.square(_plain_decode(w["v"], w["v_scale"])) if eight else w["v"]
        v = v * _BETA2 + (g * g) * (1.0 - _BETA2)
        s = torch.sqrt(v)
        w["master"].copy_(w["master"] * (1.0 - _LR * _DECAY) - rate * (m / (s / root + _ADAM_EPS)))
        if low:
            w["param"].copy_(w["master"])
            res.append(w["param"])
        if eight:
            for name, x, signed in (("m", m, True), ("v", s, False)):
                codes, scale = _plain_encode(x, signed, arena["index"], count[0])
                w[name].copy_(codes)
                w[name + "_scale"].copy_(scale)
            res += [w["master"], *(_plain_decode(w[k], w[k + "_scale"]).to(torch.bfloat16) for k in "mv")]
        else:
            w["m"].copy_(m)
            w["v"].copy_(v)
            res += [w["master"], w["m"], w["v"]]
    return res


# ---- one pass ----------------------------------------------------------------------------------------
def _run_plain(state):
    kind = state["case"]["kind"]
    with torch.no_grad():
        if kind == "rms_q8":
            return _plain_rms_q8(state)
        if kind == "rms_train":
            return _plain_rms_train(state)
        if kind.startswith("embed"):
            return _plain_embed(state)
        if kind.startswith("logprob"):
            return _plain_logprob(state)
        return _plain_adamw(state)


def run(state):
    if not own:
        return _run_plain(state)
    from paper_2312_00752_amd import autograd
    from paper_2312_00752_amd import binding as B
    case, t = state["case"], state.get("t")
    kind = case["kind"]
    if kind == "rms_q8":
        q, scale, summed = B.ss_norm_quant(t["x"], t["weight"], residual=t.get("residual"), eps=_EPS, rms=True)
        values = torch.empty(t["x"].shape, dtype=torch.bfloat16, device=q.device)
        torch.mul(q[:, :case["dim"]], scale[:, None], out=values.view(-1, case["dim"]))
        return [values] if summed is None else [values, summed]
    if kind == "rms_train":
        res = autograd.rms_norm(t["x"], t["weight"], residual=t.get("residual"), eps=_EPS)
        outs, douts = (res, [state["dout"], state["dsummed"]]) if "residual" in t else ([res], [state["dout"]])
        return [v.detach() for v in outs] + list(torch.autograd.grad(outs, list(t.values()), douts))
    if kind == "embed_fwd":
        return [B.ss_embed_fwd(state["ids"], state["table"], scale=state["scale"], out_dtype=_type(case["dtype"]))]
    if kind == "embed_train":
        out = autograd.embedding(state["ids"], state["table"], scale=state["scale"], out_dtype=_type(case["dtype"]))
        return [out.detach(), *torch.autograd.grad(out, state["table"], state["dout"])]
    if kind == "logprob_top":
        logp, entropy, _, top_logp, top_ids = B.ss_logprob_fwd(state["logits"], state["targets"], top=case["top"])
        return [logp, entropy, top_logp, top_ids]
    if kind == "logprob_train":
        logp, entropy = autograd.token_logprobs(state["logits"], state["targets"])
        outs, douts = ([logp, entropy], [state["dlogp"], state["dentropy"]]) if case["entropy"] else ([logp], [state["dlogp"]])
        return [logp.detach(), entropy.detach(), *torch.autograd.grad(outs, state["logits"], douts)]
    lists = {k: [] for k in ("param", "grad", "m", "v", "master", "m_scale", "v_scale")}
    for arena in state["arenas"]:
        e = arena["each"]
        lists["param"] += e["param"] if arena["low"] else e["master"]
        lists["master"] += e["master"] if arena["low"] else [None] * len(e["master"])
        for k in ("grad", "m", "v") + (("m_scale", "v_scale") if arena["index"] is not None else ()):
            lists[k] += e[k]
    eight = case["bits"] == 8
    B.ss_adamw_step(lists["param"], lists["grad"], lists["m"], lists["v"], state["count"], _LR, betas=(_BETA1, _BETA2), eps=_ADAM_EPS,
                    weight_decay=_DECAY, master=lists["master"], m_scale=lists["m_scale"] if eight else None,
                    v_scale=lists["v_scale"] if eight else None)
    res = []
    for arena in state["arenas"]:
        w = arena["all"]
        res += [w["param"], w["master"]] if arena["low"] else [w["master"]]
        res += [B.ss_adamw_values(w[k], w[k + "_scale"], dtype=torch.bfloat16) for k in "mv"] if eight else [w["m"], w["v"]]
    return res


# ---- what a pass cannot do without -------------------------------------------------------------------
def work(case):
    """Inputs read once, outputs written once; flops as the formulas have them (an exponential or a root counts as one)."""
    kind = case["kind"]
    size = lambda name: 2 if name == "bf16" else 4  # noqa: E731
    if kind.startswith("rms"):
        n, io, res = case["batch"] * case["seqlen"] * case["dim"], size(case["dtype"]), size(case["residual"]) if case["residual"] else 0
        if kind == "rms_q8":   # the values are given back in 16 bits, from 8
            return {"bytes": n * (io + 2 * res + 3) + 4 * case["dim"], "flops": 10 * n}
        return {"bytes": n * (4 * io + 4 * res) + 8 * case["dim"], "flops": 15 * n}
    if kind.startswith("embed"):
        tokens, vocab, dim = case["tokens"], case["vocab"], case["dim"]
        p = torch.diff(torch.log(torch.arange(1, vocab + 2, dtype=torch.float64))) / math.log(vocab + 1)
        rows = float((1.0 - (1.0 - p) ** tokens).sum())   # different ids to be expected
        n = 8 * tokens + dim * (rows * size(case["table"]) + tokens * size(case["dtype"]))
        if kind == "embed_train":
            n += dim * (tokens * size(case["dtype"]) + vocab * size(case["table"]))
        return {"bytes": n, "flops": tokens * dim * (1 if kind == "embed_fwd" else 3)}
    if kind.startswith("logprob"):
        n = case["rows"] * case["vocab"]
        if kind == "logprob_top":
            return {"bytes": n * size(case["dtype"]) + case["rows"] * (16 + 12 * case["top"]), "flops": 6 * n}
        return {"bytes": 2 * n * size(case["dtype"]) + case["rows"] * 24, "flops": (14 if case["entropy"] else 10) * n}
    total = {"bytes": 0, "flops": 0}
    for shapes, low in zip(_adamw_shapes(case), (False, True)):
        n = sum(math.prod(s) for s in shapes)
        # parameter and gradient, a copy to update, moments; 8-bit ones are given back in 16 bits
        total["bytes"] += n * ((2 + 2 + 8 if low else 12) + (4 + 6 if case["bits"] == 8 else 16))
        total["flops"] += 16 * n
    return total


# ---- the definitions in 64 bits ------------------------------------------------------------------------
def _exact_norm(case, s):
    t = {k: v.detach().double().requires_grad_(True) for k, v in s["t"].items()}
    summed = None
    if "residual" in t:
        summed = t["x"] + t["residual"]
        held = s["t"]["residual"].dtype   # what is normalised is the sum as it is held
        summed = summed + (summed.detach().to(held).double() - summed.detach())
    v = t["x"] if summed is None else summed
    out = v * torch.rsqrt(torch.linalg.vecdot(v, v)[..., None] / case["dim"] + _EPS) * t["weight"]
    if case["kind"] == "rms_q8":
        out = out.detach().to(s["t"]["x"].dtype).double()   # the 8 bits are those of the result as it would be held
        top = out.abs().amax(-1, keepdim=True).clamp(min=_LEAST)
        values = torch.round(127.0 * out / top) * top / 127.0
        return [values] if summed is None else [values, summed.detach()]
    outs = [out] if summed is None else [out, summed]
    douts = [s["dout"].double()] + ([s["dsummed"].double()] if summed is not None else [])
    return [v.detach() for v in outs] + list(torch.autograd.grad(outs, list(t.values()), douts))


def _exact_embed(case, s):
    with torch.no_grad():
        ids = torch.where(s["ids"] < 0, case["vocab"], s["ids"])   # a row of zeros behind the table
        table = torch.cat((s["table"].double(), torch.zeros(1, case["dim"], dtype=torch.float64, device=ids.device)))
        out = s["scale"] * torch.nn.functional.embedding(ids, table)
        if "dout" not in s:
            return [out]
        order = torch.argsort(ids)
        ends = torch.searchsorted(ids[order], torch.arange(case["vocab"], device=ids.device), right=True)
        sums = torch.cumsum(s["dout"][order].double(), 0)
        sums = torch.cat((torch.zeros_like(sums[:1]), sums))[ends]
        return [out, s["scale"] * torch.diff(sums, dim=0, prepend=torch.zeros_like(sums[:1]))]


def _exact_logprob(case, s):
    parts = []
    few = max(1, 2 ** 26 // case["vocab"])
    for k in range(0, case["rows"], few):
        x = s["logits"][k:k + few].detach().double()
        targets = s["targets"][k:k + few]
        logs = torch.log_softmax(x, -1)
        logp = torch.where(targets < 0, 0.0, logs[torch.arange(len(x), device=x.device), targets.clamp(min=0)])
        possible = torch.where(torch.isinf(logs), 0.0, logs)
        entropy = -(torch.exp(logs) * possible).sum(-1)
        if case["kind"] == "logprob_top":
            order = torch.argsort(x, dim=-1, descending=True, stable=True)[:, :case["top"]]
            parts.append((logp, entropy, torch.gather(logs, 1, order), order))
            continue
        p = torch.exp(logs)
        dx = -p * torch.where(targets < 0, 0.0, s["dlogp"][k:k + few].double())[:, None]
        rows = torch.nonzero(targets >= 0)[:, 0]
        dx[rows, targets[rows]] += s["dlogp"][k:k + few].double()[rows]
        if case["entropy"]:
            dx -= s["dentropy"][k:k + few].double()[:, None] * p * (possible + entropy[:, None])
        parts.append((logp, entropy, dx))
    return [torch.cat(v) for v in zip(*parts)]


def _exact_codes(x, top, index, step, phase):
    """What x, in units of its block's largest magnitude, is held as."""
    b = x.reshape(-1, _BLOCK)
    most = b.abs().amax(1, keepdim=True)
    unit = torch.where(most < _LEAST_STATE, 0.0, b / most)
    y = unit.abs() * top ** 2
    low = torch.sqrt(y).floor()
    share = (y - low ** 2) / (2 * low + 1)
    turn = torch.remainder(index * phase[0] + step * phase[1], 2 ** 32).div(256, rounding_mode="floor").double().reshape(b.shape) / 2 ** 24
    q = torch.minimum(low + (share > turn).double(), torch.tensor(float(top), device=x.device, dtype=torch.float64))
    if top == 255:
        q = torch.where(unit > 0, torch.maximum(q, torch.ones_like(q)), 0.0)
    return ((q / top) ** 2 * torch.sign(unit) * most).reshape(-1)


def _exact_adamw(case, s):
    step = int(s["count"][0]) + 1
    beta1, beta2 = float(torch.tensor(_BETA1)), float(torch.tensor(_BETA2))   # the moments' factors are held in 32 bits
    res = []
    for arena in s["arenas"]:
        w = arena["all"]
        g = w["grad"].double()
        if arena["index"] is None:
            m, v = w["m"].double(), w["v"].double()
        else:
            blocks = lambda k: w[k].double().reshape(-1, _BLOCK)  # noqa: E731
            m = (torch.sign(blocks("m")) * (blocks("m") / 127) ** 2 * w["m_scale"].double()[:, None]).reshape(-1)
            v = ((blocks("v") / 255) ** 2 * w["v_scale"].double()[:, None]).reshape(-1) ** 2
        m = beta1 * m + (1 - beta1) * g
        v = beta2 * v + (1 - beta2) * g ** 2
        rates = _LR / (1 - _BETA1 ** step) * m / (torch.sqrt(v / (1 - _BETA2 ** step)) + _ADAM_EPS)
        p = w["master"].double() * (1 - _LR * _DECAY) - rates
        if arena["low"]:
            res.append(p)
        if arena["index"] is not None:
            m = _exact_codes(m, 127, arena["index"], step, _WEYL[:2])
            v = _exact_codes(torch.sqrt(v), 255, arena["index"], step, _WEYL[2:])
        res += [p, m, v]
    return res


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("rms"):
        return _exact_norm(case, s)
    if kind.startswith("embed"):
        return _exact_embed(case, s)
    return _exact_logprob(case, s) if kind.startswith("logprob") else _exact_adamw(case, s)
