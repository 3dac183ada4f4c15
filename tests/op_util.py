"""Comparison of the block's operators with their float64 oracles.

A result held in bf16 is off by its rounding, at most half the distance of two neighbours (8 significant bits: 2^-8 of the power of
two below it), and by the float32 arithmetic before that; a float32 result by the latter alone.  The float32 part is given per tensor as a multiple of
2^-24 of a size: of the largest magnitude of the result, or of what the test names (terms of a sum).
"""
import numpy as np
import torch

EPS = 2.0 ** -24


def host(t):
    return t.detach().double().cpu().numpy()


def rounded(a, io):
    """float64 copy of ``a`` as a tensor of this type holds it."""
    return torch.from_numpy(np.asarray(a, np.float32)).to(TYPES[io]).double().numpy()


TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def close(got, ref, steps, name, size=None):
    """|got - ref| <= (half a unit in bf16's last place) + steps 2^-24 size, element by element."""
    g, ref = host(got), np.asarray(ref, np.float64)
    assert g.shape == ref.shape, (name, g.shape, ref.shape)
    if ref.size == 0:
        return
    if size is None:
        size = np.max(np.abs(ref[np.isfinite(ref)]), initial=0.0)
    assert np.array_equal(np.isnan(g), np.isnan(ref)), name + ": NaN elsewhere"
    limit = steps * EPS * np.asarray(size, np.float64)
    if got.dtype == torch.bfloat16:   # of the larger of the two: the float32 value may lie across a power of two
        limit = limit + 2.0 ** (np.frexp(np.maximum(np.abs(ref), np.where(np.isfinite(g), np.abs(g), 0.0)))[1] - 9.0)
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(g - ref) <= limit) & ~np.isnan(ref) & ~((g == ref))
    if bad.any():
        at = np.unravel_index(np.argmax(np.where(bad, np.abs(g - ref) / np.maximum(limit, 1e-300), 0.0)), ref.shape)
        raise AssertionError("%s: %d of %d off, the worst at %s: %r, not %r (limit %.2e)"
                             % (name, bad.sum(), ref.size, at, g[at], ref[at], np.broadcast_to(limit, ref.shape)[at]))


def upload(a, io):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to("cuda").to(TYPES[io])
