"""The operators together, as a language model uses them: ids -> embedding -> blocks with RMS norm -> norm -> logits -> log probabilities, the gradients of
all of it against the same steps in float64 through torch's autograd on the CPU, AdamW's step on them, the whole of it captured and replayed, and the
served form of it."""
import numpy as np
import pytest
import torch

from oracle import model_oracle as mo
from paper_2312_00752_amd import autograd as ag
from paper_2312_00752_amd import binding as B
from paper_2312_00752_amd import block as bk
from paper_2312_00752_amd import optim
from tests import op_util as u

pytestmark = pytest.mark.gpu
VOCAB, SCALE = 37, 3.0


def _block_reference(p, x, residual, reset):
    """The block with RMS norm in float64, step after step, differentiable."""
    s = x + residual
    h = s / torch.sqrt((s * s).mean(-1, keepdim=True) + 1e-5) * p["norm_weight"]
    xs, f, i, z = (h @ p["W_in"].t()).transpose(1, 2).chunk(4, 1)
    sg = torch.sigmoid(f + p["f_bias"][:, None])
    la = -torch.nn.functional.softplus(p["rate_raw"])[:, None] * sg
    keep = (~reset)[:, None].double()
    a, m = torch.exp(la) * keep, torch.sqrt(1 - torch.exp(2 * la) * keep)
    b = m * torch.sigmoid(i + p["i_bias"][:, None]) * xs
    state, hs = torch.zeros_like(b[..., 0]), []
    for t in range(b.shape[-1]):
        state = a[..., t] * state + b[..., t]
        hs.append(state)
    y = torch.stack(hs, -1) * z * torch.sigmoid(z)
    return y.transpose(1, 2) @ p["W_out"].t(), s


class Model(torch.nn.Module):
    def __init__(self, width, inner, layers=2):
        super().__init__()
        self.table = torch.nn.Parameter(0.3 * torch.randn(VOCAB, width, device="cuda"))
        self.blocks = torch.nn.ModuleList(bk.GatedBlock(width, inner, norm="rms") for _ in range(layers))
        self.norm_weight = torch.nn.Parameter(torch.ones(width, device="cuda"))
        self.head = torch.nn.Parameter(torch.randn(VOCAB, width, device="cuda") * width ** -0.5)

    def forward(self, ids, targets, reset):
        x, residual = ag.embedding(ids, self.table, scale=SCALE), None
        for b in self.blocks:
            x, residual = b(x, residual, reset)
        h, _ = ag.rms_norm(x, self.norm_weight, residual=residual)
        logp, entropy = ag.token_logprobs(h @ self.head.t(), targets)
        return logp.sum() + 0.1 * entropy.sum()


def _reference(p, ids, targets, reset):
    """Model.forward in float64 on the CPU: p by name."""
    there = (ids >= 0)[..., None]
    x = torch.where(there, SCALE * p["table"][ids.clamp(min=0)], 0.0)
    residual = torch.zeros_like(x)
    for k in range(2):
        x, residual = _block_reference({n.split(".", 2)[2]: v for n, v in p.items() if n.startswith("blocks.%d." % k)}, x, residual, reset)
    s = x + residual
    h = s / torch.sqrt((s * s).mean(-1, keepdim=True) + 1e-5) * p["norm_weight"]
    logs = torch.log_softmax(h @ p["head"].t(), -1)
    logp = torch.where(targets >= 0, logs.gather(-1, targets.clamp(min=0)[..., None])[..., 0], 0.0)
    return logp.sum() - 0.1 * (logs.exp() * logs).sum()


def _data(nb, nl, seed=0):
    """Documents packed into rows, padded at their ends."""
    g = torch.Generator().manual_seed(seed)
    ids, targets = torch.randint(0, VOCAB, (nb, nl), generator=g), torch.randint(0, VOCAB, (nb, nl), generator=g)
    for k in range(nb):
        ids[k, nl - 3 * k:] = -1
        targets[k, nl - 3 * k - 1:] = -1
    reset = torch.rand(nb, nl, generator=g) < 0.05
    return [t.cuda() for t in (ids, targets, reset)]


@pytest.mark.parametrize("nb,nl,width,inner", [(3, 40, 24, 33), (1, 300, 64, 16), (2, 1, 16, 8)])
def test_gradients(nb, nl, width, inner):
    """Float32 throughout, sums of up to some thousand terms through a dozen operators: 2e-4 of the largest magnitude, twice what one block is held to."""
    torch.manual_seed(nl)
    model = Model(width, inner)
    data = _data(nb, nl)
    loss = model(*data)
    names = [n for n, _ in model.named_parameters()]
    grads = torch.autograd.grad(loss, list(model.parameters()))
    p = {n: v.detach().double().cpu().requires_grad_(True) for n, v in model.named_parameters()}
    ref = _reference(p, *(t.cpu() for t in data))
    rg = torch.autograd.grad(ref, [p[n] for n in names])
    assert abs(loss.item() - ref.item()) < 1e-4 * abs(ref.item())
    for name, got, want in zip(names, grads, rg):
        err = (got.double().cpu() - want).abs().max() / want.abs().max().clamp(min=1e-6)
        assert err < 2e-4, (name, float(err))


@pytest.mark.parametrize("bits", [8, 32])
def test_step(bits):
    """The optimiser's step on the model's gradients: that of the definition, on the gradients as they are."""
    torch.manual_seed(1)
    model = Model(24, 33)
    opt = optim.AdamW(model.parameters(), lr=1e-2, weight_decay=0.1, state_bits=bits)
    before = [p.detach().double().cpu().numpy() for p in model.parameters()]
    (-model(*_data(3, 40))).backward()
    opt.step()
    for p, x in zip(model.parameters(), before):
        g = p.grad.double().cpu().numpy()
        zero = np.zeros_like(g)
        ref, _, _, size = mo.adamw(x, g, zero, zero, 1, 1e-2, 0.9, 0.999, 1e-8, 0.1)
        u.close(p, ref, 24, "param", size=np.abs(x) / 8 + size)


def test_captured_training_step():
    """Forward, backward and the optimiser in one graph: each replay is a step, as an eager one is."""
    torch.manual_seed(2)
    eager, graphed = Model(24, 33), Model(24, 33)
    with torch.no_grad():
        for p, q in zip(eager.parameters(), graphed.parameters()):
            q.copy_(p)
    a, b = (optim.AdamW(m.parameters(), lr=1e-2, state_bits=8) for m in (eager, graphed))
    ids, targets, reset = _data(3, 40)

    def step(model, opt):
        params = list(model.parameters())
        for p, g in zip(params, torch.autograd.grad(-model(ids, targets, reset), params)):
            p.grad = g
        opt.step()

    # the graph's memory is warmed up on another model, on a stream of its own
    warm = Model(24, 33)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(warm, optim.AdamW(warm.parameters(), state_bits=8))
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed, b)
    for k in range(4):
        for t, new in zip((ids, targets, reset), _data(3, 40, seed=k)):
            t.copy_(new)
        step(eager, a)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for (name, p), q in zip(eager.named_parameters(), graphed.named_parameters()):
            assert torch.equal(p, q[1]), (k, name)
    assert b.param_groups[0]["count"].tolist() == [4, 0]


def test_served():
    """Prompt and tokens through the served blocks with RMS norm, and what is said of the tokens taken."""
    torch.manual_seed(3)
    model = Model(96, 130)
    served = [b.serving() for b in model.blocks]
    ids = torch.randint(0, VOCAB, (3, 50), device="cuda")
    with torch.no_grad():
        def tail(x, residual, next_ids):
            h, _, _ = B.ss_norm_fwd(x, model.norm_weight, residual=residual, rms=True)
            return B.ss_logprob_fwd(h @ model.head.t(), next_ids, top=5)
        x, residual, states = B.ss_embed_fwd(ids[:, :37].contiguous(), model.table, scale=SCALE), None, []
        for b in served:
            x, residual, state = b.prompt(x, residual)
            states.append(state)
        logp, entropy, _, top_logp, top_ids = tail(x, residual, ids[:, 1:38].contiguous())
        # against the model in float32: two 8-bit products a block cost some percent of the activations, so of logits of a size of 3 some tenths
        y, r = ag.embedding(ids[:, :37].contiguous(), model.table, scale=SCALE), None
        for b in model.blocks:
            y, r = b(y, r)
        want, wanted_entropy = ag.token_logprobs(ag.rms_norm(y, model.norm_weight, residual=r)[0] @ model.head.t(), ids[:, 1:38].contiguous())
        assert (logp - want).abs().mean() < 0.1 and (entropy - wanted_entropy).abs().mean() < 0.1
        assert (top_logp[..., :-1] >= top_logp[..., 1:]).all() and (top_logp[..., 0] >= logp - 1e-5).all()
        # token by token from the prompt's states: the same as a longer prompt, to what its 8-bit rounding gives where a value lies between two codes
        x, residual = B.ss_embed_fwd(ids, model.table, scale=SCALE), None
        for b in served:
            x, residual, _ = b.prompt(x, residual)
        whole = tail(x, residual, ids.roll(-1, 1).contiguous())[0]
        for t in range(37, 50):
            x, residual = B.ss_embed_fwd(ids[:, t].contiguous(), model.table, scale=SCALE), None
            for b, state in zip(served, states):
                x, residual = b.step(x, state, residual)
            one = tail(x, residual, ids.roll(-1, 1)[:, t].contiguous())[0]
            assert (one - whole[:, t]).abs().max() < 0.05


@pytest.mark.parametrize("norm,bits", [("rms", 32), ("layer", 8)])
def test_example(norm, bits):
    loss, right = bk.main(steps=3, norm=norm, state_bits=bits)
    assert np.isfinite(loss) and 0 <= right <= 16


def test_block_refuses_other_norms():
    with pytest.raises(ValueError):
        bk.GatedBlock(8, 8, norm="batch")
