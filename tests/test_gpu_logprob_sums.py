"""Sums over long rows of logits that one column outweighs: what is added to it does not vanish, term by term, in the rounding.

Tolerance in multiples of 2^-24 of op_util.close's sizes, from the longest chain that a term of S = sum exp(x - max) passes: its exponential, 4 (an argument
of |d| rounded twice, which the size counts, and a unit in the last place); the sum of a lane's 32 values of a step, eight one after another and their sums as a tree, 9; a step's
correction for a new maximum and its addition, 4 a step of 8192 columns (of 1024 in rows of one wave, two at most); a wave's lanes, 3 and 6; four waves one after another, 12; the
pieces' parts, 4 for every 64 of them and 9 more; the logarithm or the reciprocal, 5.  52 + 4 ceil(vocab / 8192).  A sum that takes its terms one by one loses
vocab / 256 of the terms here, each by nearly a whole step of 2^-24: 195 at 50021 columns where 80 are allowed."""
import numpy as np
import pytest
import torch

from oracle import model_oracle as mo
from paper_2312_00752_amd import binding as B
from tests import op_util as u

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("rows", [5, 300])
@pytest.mark.parametrize("vocab", [2048, 50021, 131077])
def test_a_row_with_one_large_logit(vocab, rows, top):
    rng = np.random.default_rng(vocab)
    if rows * vocab > 20e6:
        rows = 256   # the least that are not cut into pieces
    # exp of it is 0.98 of half a step of 1: lost beside 1, alone
    x = np.full((rows, vocab), np.float32(np.log(0.98 * 2.0 ** -24)), np.float32)
    at = rng.integers(0, 300, rows)   # early: what follows in its lane comes onto it
    x[np.arange(rows), at] = 0.0
    x = (x + rng.integers(-3, 4, (rows, 1))).astype(np.float32)
    some = np.r_[:3, rows - 2:rows]   # the oracle is slow
    t = rng.integers(0, vocab, rows)
    t[some[::2]] = at[some[::2]]
    dl, dh = rng.standard_normal(rows).astype(np.float32), rng.standard_normal(rows).astype(np.float32)
    tx, tt = torch.from_numpy(x).cuda(), torch.from_numpy(t).cuda()
    logp, entropy, stats, _, _ = B.ss_logprob_fwd(tx, tt, top=top)
    steps = 52 + 4 * -(-vocab // 8192)
    ref = mo.logprob_fwd(x[some], t[some])
    u.close(logp[some], ref["logp"], steps, "logp", size=ref["logp_size"])
    u.close(entropy[some], ref["entropy"], steps, "entropy", size=ref["entropy_size"])
    u.close(stats[1][some], 1.0 / ref["total"], steps, "1 / S", size=(1.0 - (ref["p"] * ref["d"]).sum(1)) / ref["total"])
    for de in (None, dh):
        dx = B.ss_logprob_bwd(tx, stats, tt, dlogp=torch.from_numpy(dl).cuda(), entropy=entropy, dentropy=None if de is None else torch.from_numpy(de).cuda())
        g = mo.logprob_bwd(ref, t[some], dl[some], None if de is None else de[some])
        u.close(dx[some], g["dlogits"], steps, "dlogits", size=g["dlogits_size"])
