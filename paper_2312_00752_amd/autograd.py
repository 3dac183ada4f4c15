"""``torch.autograd`` front-ends of the library: the selective scan, the layer around it, layer norm and the gated recurrence.

Still marshalling only: ``forward`` enqueues ``ss_scan_fwd`` / ``ss_layer_fwd`` and keeps the
workspace the library filled, ``backward`` enqueues ``ss_scan_bwd`` / ``ss_layer_bwd``; all
arithmetic happens in the HIP kernels.  Tensors use the library's layouts (sequence axis
last): u, delta, z (B,D,L); B, C (B,N,L) or a time-invariant (D,N) float32; A (D,N) float32.
"""
import functools

import torch

from . import binding as B


def _code(t):
    return B.SS_BF16 if t.dtype == torch.bfloat16 else B.SS_F32


class _NoGradient(torch.autograd.Function):
    """Gradients as results of what they were computed from; differentiating them is an error."""

    @staticmethod
    def forward(ctx, grads, *sources):
        return tuple(g.detach() for g in grads)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the gradients of this operator cannot be differentiated again")


def last_derivative(backward):
    """Of a backward function that computes its gradients outside of torch's graph: where a graph of them is being built, they are
    connected to everything that they depend on through an error, so that a second derivative is refused whichever way it
    is asked for (an error without connections is passed over where torch looks for the way to given inputs)."""
    @functools.wraps(backward)
    def call(ctx, *douts):
        with torch.no_grad():
            grads = backward(ctx, *douts)
        sources = [t for t in (*ctx.saved_tensors, *douts) if t is not None and t.requires_grad] if torch.is_grad_enabled() else []
        if not sources:
            return grads
        some = [k for k, g in enumerate(grads) if g is not None]
        grads = list(grads)
        for k, g in zip(some, _NoGradient.apply([grads[k] for k in some], *sources)):
            grads[k] = g
        return tuple(grads)
    return call


class _SelectiveScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, u, delta, A, Bm, Cm, Dskip, z, delta_bias, h0, delta_softplus, exact_zoh, return_last_state):
        nb, nd, nl = u.shape
        nn = A.shape[1]
        ws = torch.empty(max(256, B.ss_workspace_bytes(nb, nd, nl, nn, True, _code(u), z is not None,
                                                       Bm.dim() == 2, Cm.dim() == 2)),
                         dtype=torch.uint8, device=u.device)
        out, h_last = B.ss_scan_fwd(u, delta, A, Bm, Cm, Dskip=Dskip, z=z, delta_bias=delta_bias, h0=h0,
                                    delta_softplus=delta_softplus, return_last_state=return_last_state,
                                    workspace=ws, save_for_bwd=True, exact_zoh=exact_zoh)
        ctx.save_for_backward(u, delta, A, Bm, Cm, Dskip, z, delta_bias, h0, ws)
        ctx.opts = (delta_softplus, exact_zoh)
        if return_last_state:
            return out, h_last
        return out

    @staticmethod
    def backward(ctx, dout, *rest):
        u, delta, A, Bm, Cm, Dskip, z, delta_bias, h0, ws = ctx.saved_tensors
        delta_softplus, exact_zoh = ctx.opts
        dh_last = rest[0] if rest and rest[0] is not None else None
        g = B.ss_scan_bwd(dout.contiguous(), u, delta, A, Bm, Cm, ws, Dskip=Dskip, z=z, delta_bias=delta_bias,
                          h0=h0, delta_softplus=delta_softplus,
                          dh_last=None if dh_last is None else dh_last.contiguous(),
                          want_dh0=h0 is not None, exact_zoh=exact_zoh)
        dB = g["dB"] if Bm.dim() == 2 else g["dB"].to(Bm.dtype)
        dC = g["dC"] if Cm.dim() == 2 else g["dC"].to(Cm.dtype)
        return (g["du"], g["ddelta"], g["dA"], dB, dC, g["dD"], g["dz"], g["ddelta_bias"], g["dh0"],
                None, None, None)


def selective_scan(u, delta, A, Bm, Cm, Dskip=None, z=None, delta_bias=None, h0=None, delta_softplus=False,
                   exact_zoh=False, return_last_state=False):
    """Differentiable selective scan (Algorithm 2, steps 5-6, with the gate of Section 3.4).
    Returns out, or (out, h_last) with ``return_last_state``."""
    return _SelectiveScan.apply(u, delta, A, Bm, Cm, Dskip, z, delta_bias, h0, delta_softplus, exact_zoh,
                                return_last_state)


class _SelectiveSSMLayer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, z, conv_w, conv_b, W_x, W_dt, dt_bias, A, Dskip):
        nb, nd, nl = x.shape
        nn, rank, width = A.shape[1], W_dt.shape[1], conv_w.shape[1]
        code = _code(x)
        saved = torch.empty(B.ss_layer_saved_bytes(nb, nd, nl, nn, rank, width, code), dtype=torch.uint8, device=x.device)
        scratch = torch.empty(B.ss_layer_scratch_bytes(nb, nd, nl, nn, rank, width, code, False), dtype=torch.uint8,
                              device=x.device)
        out = B.ss_layer_fwd(x, z, conv_w, conv_b, W_x, W_dt, dt_bias, A, Dskip, scratch=scratch, saved=saved)
        ctx.save_for_backward(x, z, conv_w, conv_b, W_x, W_dt, dt_bias, A, Dskip, saved)
        return out

    @staticmethod
    def backward(ctx, dout):
        x, z, conv_w, conv_b, W_x, W_dt, dt_bias, A, Dskip, saved = ctx.saved_tensors
        nb, nd, nl = x.shape
        nn, rank, width = A.shape[1], W_dt.shape[1], conv_w.shape[1]
        scratch = torch.empty(B.ss_layer_scratch_bytes(nb, nd, nl, nn, rank, width, _code(x), True), dtype=torch.uint8,
                              device=x.device)
        g = B.ss_layer_bwd(dout.contiguous(), x, z, conv_w, conv_b, W_x, W_dt, dt_bias, A, Dskip, scratch=scratch,
                           saved=saved)
        return (g["dx"], g["dz"], g["dconv_w"], g["dconv_b"], g["dW_x"].to(W_x.dtype), g["dW_dt"].to(W_dt.dtype),
                g["ddt_bias"], g["dA"], g["dD"])


def selective_ssm_layer(x, z, conv_w, conv_b, W_x, W_dt, dt_bias, A, Dskip):
    """Differentiable layer around the scan: conv + SiLU, Delta/B/C projections, scan, gate (Section 3.4,
    Algorithm 2); only x, z, the small projection output and the scan's checkpoints are kept for backward."""
    return _SelectiveSSMLayer.apply(x, z, conv_w, conv_b, W_x, W_dt, dt_bias, A, Dskip)


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, eps):
        out, summed, stats = B.ss_norm_fwd(x, weight, bias, residual=residual, eps=eps, save_stats=True)
        ctx.save_for_backward(x if summed is None else summed, weight, stats)
        ctx.opts = (bias is not None, None if residual is None else residual.dtype, eps, x.dtype)
        ctx.set_materialize_grads(False)
        return out if summed is None else (out, summed)

    @staticmethod
    @last_derivative
    def backward(ctx, dout, dsummed=None):
        s, weight, stats = ctx.saved_tensors
        has_bias, held, eps, io = ctx.opts
        if dout is None:   # only the sum was used
            return (None if dsummed is None else dsummed.to(io)), None, None, dsummed, None
        g = B.ss_norm_bwd(dout.contiguous(), s, stats, weight, has_bias=has_bias, residual_dtype=held, eps=eps,
                          dsummed=None if dsummed is None else dsummed.contiguous())
        return g["dx"], g["dweight"], g["dbias"], g["dresidual"], None


def layer_norm(x, weight=None, bias=None, residual=None, eps=1e-5):
    """Differentiable layer norm over the last axis.  With ``residual`` (float32 or x's dtype) the sum of the two is normalised
    and returned as well, in residual's dtype: (out, summed), the residual stream that the next block continues."""
    if x.is_cuda:
        r = B.layer_norm_node(x, weight, bias, residual, eps)
        if r is not None:
            return r if residual is not None else r[0]
    return _LayerNorm.apply(x, weight, bias, residual, eps)


class _GatedRecurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, f, rate, i, z, f_bias, i_bias, reset, h0, return_last_state):
        ws = torch.empty(max(256, B.ss_gate_workspace_bytes(*x.shape)), dtype=torch.uint8, device=x.device)
        out, h_last = B.ss_gate_fwd(x, f, rate, i=i, z=z, f_bias=f_bias, i_bias=i_bias, reset=reset, h0=h0,
                                    return_last_state=return_last_state, workspace=ws, save_for_bwd=True)
        ctx.save_for_backward(x, f, rate, i, z, f_bias, i_bias, reset, h0, ws)
        return (out, h_last) if return_last_state else out

    @staticmethod
    @last_derivative
    def backward(ctx, dout, dh_last=None):
        x, f, rate, i, z, f_bias, i_bias, reset, h0, ws = ctx.saved_tensors
        g = B.ss_gate_bwd(dout.contiguous(), x, f, rate, ws, i=i, z=z, f_bias=f_bias, i_bias=i_bias, reset=reset, h0=h0,
                          dh_last=None if dh_last is None else dh_last.contiguous(), want_dh0=h0 is not None)
        return g["dx"], g["df"], g["drate"], g["di"], g["dz"], g["df_bias"], g["di_bias"], None, g["dh0"], None


def gated_recurrence(x, f, rate, i=None, z=None, f_bias=None, i_bias=None, reset=None, h0=None, return_last_state=False):
    """Differentiable gated linear recurrence (include/ss_gate.h): h <- a h + sqrt(1 - a^2) sigmoid(i) x with
    a = exp(-rate sigmoid(f)), gated by SiLU(z).  Returns out, or (out, h_last) with ``return_last_state``."""
    if x.is_cuda:
        r = B.gated_recurrence_node(x, f, i, z, rate, f_bias, i_bias, reset, h0, return_last_state)
        if r is not None:
            return r if return_last_state else r[0]
    return _GatedRecurrence.apply(x, f, rate, i, z, f_bias, i_bias, reset, h0, return_last_state)
