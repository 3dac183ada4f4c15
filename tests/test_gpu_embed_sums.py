"""Sums of the embedding's gradient against the float64 oracle, within what their division allows: every addition that a term passes may be off by half a step
of the sum of magnitudes so far, 2^-24 of the whole sum at most, and so may the product (tests/embed_plan.py counts them)."""
import numpy as np
import pytest
import torch

from paper_2312_00752_amd import binding as B
from tests import embed_plan, op_util as u

pytestmark = pytest.mark.gpu


def reference(ids, vocab, dout, scale):
    """The oracle's sums, and those of magnitudes, by whole rows."""
    grad, size = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1]))
    np.add.at(grad, ids, dout * scale)
    np.add.at(size, ids, np.abs(dout * scale))
    return grad, size


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,dim", [(100, 7, 40), (5199, 257, 1021), (8193, 300, 513), (16384, 500, 2048), (40000, 1000, 8), (65536, 256, 64)])
@pytest.mark.parametrize("kind", ["even", "text", "one", "ones"])
def test_sums(kind, n, vocab, dim, io):
    rng = np.random.default_rng(n)
    ids = {"even": lambda: rng.integers(0, vocab, n), "text": lambda: np.minimum((vocab * rng.uniform(size=n) ** 4).astype(np.int64), vocab - 1),
           "one": lambda: np.full(n, vocab - 1), "ones": lambda: np.where(rng.uniform(size=n) < 0.9, 3, rng.integers(0, vocab, n))}[kind]()
    # of one sign and of like sizes, whose roundings add up more than those of mixed ones
    dout = u.rounded(rng.uniform(0.5, 1.0, (n, dim)), io)
    got = B.ss_embed_bwd(u.upload(dout, io), torch.from_numpy(ids).cuda(), vocab, scale=0.7, dtype=torch.float32)
    grad, size = reference(ids, vocab, dout, float(np.float32(0.7)))
    u.close(got, grad, embed_plan.roundings(n, dim), "dtable", size=size)
