"""8-bit moments over thousands of steps against moments that are not rounded: what the rounding adds in the mean.

A rounding is right in the mean, and m is linear in it.  v is the square of sqrt(v) as held, a code q, so a rounding over a distance D = (2 q + 1) / 255^2 a of neighbours adds
its variance: from a code the next value lies |g^2 / v - 1| (1 - beta2) / 2 sqrt(v) away, d, and a rounding of d to 0 or D has the variance d (D - d).  With
D = 2 / q sqrt(v) and a mean of |g^2 / v - 1| of 0.97 (normal gradients) that is 0.97 (1 - beta2) / q of v in every step, and in balance v is 1 / (1 - 0.97 / q) of
what it should be: 0.97 / (q - 0.97) too large, q = 255 sqrt(sqrt(v) / a).  Allowed: a third more, and 0.02 to either side for what is drawn (12000 elements a
size; an element's v strays by its rounding's variance over 1 / (1 - beta2) steps, up to about itself at the smallest size)."""
import numpy as np
import pytest
import torch

from paper_2312_00752_amd import binding as B

pytestmark = pytest.mark.gpu
SHARES = [1.0, 1e-1, 1e-2, 1e-3, 1e-4]


@pytest.mark.parametrize("beta2", [0.95, 0.99, 0.999])
def test_thousands_of_steps(beta2):
    blocks, steps = 256, 4000
    gen = torch.Generator(device="cuda").manual_seed(0)
    sizes = torch.tensor(SHARES, device="cuda").repeat_interleave(52)[:256].repeat(blocks)
    n = sizes.numel()
    p, m, v = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs, count = torch.zeros(blocks, device="cuda"), torch.zeros(blocks, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    m_exact, v_exact = torch.zeros(n, device="cuda", dtype=torch.float64), torch.zeros(n, device="cuda", dtype=torch.float64)
    for _ in range(steps):
        g = torch.randn(n, generator=gen, device="cuda") * sizes
        B.ss_adamw_step([p], [g], [m], [v], count, 0.0, betas=(0.9, beta2), m_scale=[ms], v_scale=[vs])
        m_exact.lerp_(g.double(), 0.1)
        v_exact.lerp_(g.double() ** 2, 1 - beta2)
    got_m, got_v = B.ss_adamw_values(m, ms).double(), B.ss_adamw_values(v, vs).double() ** 2
    top = vs.double().repeat_interleave(256)
    for share in SHARES:
        at = sizes == sizes.new_tensor(share)
        q = 255 * (v_exact[at].sqrt() / top[at]).sqrt().mean().item()
        excess = (got_v[at].mean() / v_exact[at].mean()).item() - 1
        off = ((got_m - m_exact)[at].mean() / m_exact[at].square().mean().sqrt()).item()
        print("beta2 %g, %g of the largest: code %.1f, v %+.4f, sqrt(v) %+.4f, m %+.4f"
              % (beta2, share, q, excess, (got_v[at].sqrt().mean() / v_exact[at].sqrt().mean()).item() - 1, off))
        assert -0.02 <= excess <= 1.33 * 0.97 / (q - 0.97) + 0.02, share
        assert abs(off) <= 0.05, share
