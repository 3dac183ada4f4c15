"""A block made of the library's operators: layer or RMS norm with the residual stream, a projection, the gated linear recurrence, a
projection back (the homogeneous block of arXiv 2312.00752, Section 3.4, with the recurrence of its Theorem 1 in the scan's place).

    h, residual = norm(x + residual)
    [x; f; i; z] = W_in h            (4 inner, L): the sequence comes last, as the recurrence reads it
    y            = gated_recurrence(x, f, rate, i, z)
    out          = W_out y           tokens first again

``GatedBlock`` trains: every step is differentiable, and documents packed into rows are kept apart by ``reset``.  ``serving()`` gives the
same block with both projections in 8-bit integers, for prompts and single tokens.  ``python -m paper_2312_00752_amd.block`` trains one on
a recall task, with the library's embedding before it, its log probabilities behind it and its optimiser, and serves it.
"""
import torch

from . import autograd, binding as B, optim


def _sum_like(W, terms):
    """Float32 memory for a sum of products, the first of which overwrites it; 0 where there is none."""
    return (torch.empty if terms else torch.zeros)(W.shape, dtype=torch.float32, device=W.device)


class _Projection(torch.autograd.Function):
    """W (M,K) times tokens h (B,L,K): (B,M,L), on the library's projection kernels (include/ss_layer.h)."""

    @staticmethod
    def forward(ctx, W, h):
        ctx.save_for_backward(W, h)
        out = torch.empty((h.shape[0], W.shape[0], h.shape[1]), dtype=h.dtype, device=h.device)
        return B.ss_proj_gemm(W, h, out, trans_b=True)

    @staticmethod
    @autograd.last_derivative
    def backward(ctx, dout):
        W, h = ctx.saved_tensors
        dout = dout.contiguous()
        dh = B.ss_proj_gemm(dout, W, torch.empty_like(h), trans_a=True)
        dW = _sum_like(W, len(h))
        for b in range(h.shape[0]):
            B.ss_proj_gemm(dout[b], h[b], dW, accumulate=b > 0)
        return dW.to(W.dtype), dh


class _ProjectionBack(torch.autograd.Function):
    """The transpose of W (M,K) times y (B,K,L): tokens (B,L,M)."""

    @staticmethod
    def forward(ctx, W, y):
        ctx.save_for_backward(W, y)
        out = torch.empty((y.shape[0], y.shape[2], W.shape[0]), dtype=y.dtype, device=y.device)
        return B.ss_proj_gemm(y, W, out, trans_a=True, trans_b=True)

    @staticmethod
    @autograd.last_derivative
    def backward(ctx, dout):
        W, y = ctx.saved_tensors
        dout = dout.contiguous()
        dy = B.ss_proj_gemm(W, dout, torch.empty_like(y), trans_a=True, trans_b=True)
        dW = _sum_like(W, len(y))
        for b in range(y.shape[0]):
            B.ss_proj_gemm(dout[b], y[b], dW, trans_a=True, trans_b=True, accumulate=b > 0)
        return dW.to(W.dtype), dy


class GatedBlock(torch.nn.Module):
    """x (B,L,width) of ``dtype``; the residual stream is float32 or of that type.  ``norm`` is "layer" or "rms" (which has no bias).
    Calls give (out, residual)."""

    rms = False   # of blocks that were pickled before there was a choice

    def __init__(self, width, inner, dtype=torch.float32, device="cuda", eps=1e-5, norm="layer"):
        super().__init__()
        if norm not in ("layer", "rms"):
            raise ValueError("norm must be \"layer\" or \"rms\", got %r" % (norm,))
        self.inner, self.eps, self.rms = inner, eps, norm == "rms"
        f32 = {"dtype": torch.float32, "device": device}
        self.norm_weight = torch.nn.Parameter(torch.ones(width, **f32))
        self.norm_bias = None if self.rms else torch.nn.Parameter(torch.zeros(width, **f32))
        self.W_in = torch.nn.Parameter((torch.randn(4 * inner, width, **f32) * width ** -0.5).to(dtype))
        self.W_out = torch.nn.Parameter((torch.randn(width, inner, **f32) * inner ** -0.5).to(dtype))
        # decays at a logit of 0 between 0.9 and 0.999, as rate sigmoid(f_bias) = -log a
        half = -torch.log(torch.empty(inner, **f32).uniform_(0.9, 0.999))
        self.rate_raw = torch.nn.Parameter(torch.full((inner,), 0.5413, **f32))   # softplus of it is 1
        self.f_bias = torch.nn.Parameter(torch.logit(half))
        self.i_bias = torch.nn.Parameter(torch.zeros(inner, **f32))

    def rate(self):
        return torch.nn.functional.softplus(self.rate_raw)

    def forward(self, x, residual=None, reset=None):
        if residual is None:
            residual = torch.zeros_like(x)
        norm = autograd.rms_norm if self.rms else autograd.layer_norm
        h, residual = norm(x, self.norm_weight, self.norm_bias, residual=residual, eps=self.eps)
        xs, f, i, z = _Projection.apply(self.W_in, h).chunk(4, 1)
        y = autograd.gated_recurrence(xs, f, self.rate(), i=i, z=z, f_bias=self.f_bias, i_bias=self.i_bias, reset=reset)
        return _ProjectionBack.apply(self.W_out, y), residual

    def serving(self):
        return ServedBlock(self)


class ServedBlock:
    """A block as it stands, with its projections in 8-bit integers: ``prompt`` gives (out, residual, state), ``step`` continues from
    the state, which it updates in place."""

    rms = False   # as GatedBlock's

    @torch.no_grad()
    def __init__(self, block):
        own = lambda v: v if v is None else v.detach().clone()   # as the 8-bit weights and the rate are: training goes on without this block
        self.norm_weight, self.norm_bias, self.eps, self.rms = own(block.norm_weight), own(block.norm_bias), block.eps, block.rms
        self.rate, self.f_bias, self.i_bias = block.rate(), own(block.f_bias), own(block.i_bias)
        self.W_in, self.in_scale = B.ss_quant_rows(block.W_in.detach())
        self.W_out, self.out_scale = B.ss_quant_rows(block.W_out.detach())

    def prompt(self, x, residual=None, reset=None, state=None):
        if residual is None:
            residual = torch.zeros_like(x)
        if x.shape[1] == 1 and x.shape[0] <= 4:
            # as in step: the same bits and launches, and less for the host (9.4 us against 11.0; of 8 rows of 1024 columns, which the product does not
            # bring to 8 bits in its own launch, 11.8 against 11.3)
            h, residual, _ = B.ss_norm_fwd(x, self.norm_weight, self.norm_bias, residual=residual, eps=self.eps, rms=self.rms)
            gates = B.ss_qlinear(h, self.W_in, self.in_scale, out_seq_last=True)
        else:
            q, scale, residual = B.ss_norm_quant(x, self.norm_weight, self.norm_bias, residual=residual, eps=self.eps, rms=self.rms)
            gates = B.ss_qlinear(q.view(*x.shape[:2], q.shape[1]), self.W_in, self.in_scale, x_scale=scale, dim=x.shape[2], out_dtype=x.dtype, out_seq_last=True)
        xs, f, i, z = gates.chunk(4, 1)
        y, state = B.ss_gate_fwd(xs, f, self.rate, i=i, z=z, f_bias=self.f_bias, i_bias=self.i_bias, reset=reset, h0=state,
                                 return_last_state=True)
        return B.ss_qlinear(y, self.W_out, self.out_scale, x_seq_last=True), residual, state

    def step(self, x_t, state, residual_t=None, reset_t=None):
        """One token: x_t (B,width).  Returns (out_t, residual_t)."""
        if residual_t is None:
            residual_t = torch.zeros_like(x_t)
        # the product of a few tokens brings them to 8 bits in its own launch
        h, residual_t, _ = B.ss_norm_fwd(x_t, self.norm_weight, self.norm_bias, residual=residual_t, eps=self.eps, rms=self.rms)
        xs, f, i, z = B.ss_qlinear(h, self.W_in, self.in_scale).chunk(4, 1)
        y = B.ss_gate_step(state, xs, f, self.rate, i_t=i, z_t=z, f_bias=self.f_bias, i_bias=self.i_bias, reset_t=reset_t)
        return B.ss_qlinear(y, self.W_out, self.out_scale), residual_t


def main(steps=60, batch=16, length=64, width=128, inner=256, symbols=16, norm="layer", state_bits=32):
    """Recall: the symbol shown at the start of a document is asked for at its end; two documents a row, kept apart by reset."""
    torch.manual_seed(0)
    dev = "cuda"
    block = GatedBlock(width, inner, device=dev, norm=norm)
    embed = torch.nn.Parameter(torch.randn(symbols + 1, width, device=dev) * 0.5)
    read = torch.nn.Parameter(torch.randn(symbols, width, device=dev) * width ** -0.5)
    params = list(block.parameters()) + [embed, read]
    opt = optim.AdamW(params, lr=3e-3, weight_decay=0.0, state_bits=state_bits)
    reset = torch.zeros(batch, length, dtype=torch.bool, device=dev)
    reset[:, [0, length // 2]] = True

    def task():
        seq = torch.full((batch, length), symbols, device=dev)
        seq[:, 0::length // 2] = torch.randint(0, symbols, (batch, 2), device=dev)
        return seq, seq[:, 0::length // 2].contiguous()

    for step in range(steps):
        seq, want = task()
        out, residual = block(autograd.embedding(seq, embed), reset=reset)
        logits = (out + residual)[:, length // 2 - 1::length // 2] @ read.t()
        loss = -autograd.token_logprobs(logits, want)[0].mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        if step % 10 == 0 or step == steps - 1:
            print("step %d: loss %.3f" % (step, loss.item()), flush=True)
    with torch.no_grad():   # the first document token by token, in 8 bits
        served = block.serving()
        seq, want = task()
        x = B.ss_embed_fwd(seq, embed)
        _, _, state = served.prompt(x[:, :4].contiguous())
        for t in range(4, length // 2):
            out, residual = served.step(x[:, t].contiguous(), state)
        logp, entropy, _, _, best = B.ss_logprob_fwd((out + residual) @ read.t(), want[:, 0].contiguous(), top=1)
        right = best[:, 0] == want[:, 0]
        print("served in 8 bits: %d of %d recalled, log probability %.3f, entropy %.3f" % (int(right.sum()), batch, logp.mean().item(), entropy.mean().item()), flush=True)
    return loss.item(), int(right.sum())


if __name__ == "__main__":
    main()
