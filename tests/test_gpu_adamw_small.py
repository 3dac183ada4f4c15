"""AdamW where second moments are too small for a normal float32: their root, and with it the step, is that of the number held.

The step's tolerance is the one of test_gpu_adamw.py, 24 roundings of it, with the second moment as float32 holds it."""
import numpy as np
import pytest
import torch

from paper_2312_00752_amd import binding as B
from tests.test_gpu_adamw import F, codes_in_f32, values_in_f32

pytestmark = pytest.mark.gpu
LR, B1, B2 = 1e-2, 0.9, 0.999


def one_step(g, bits, eps, dtype=torch.float32):
    n = len(g)
    tg, p = torch.from_numpy(g).cuda(), torch.zeros(n, device="cuda")
    eight = bits == 8
    m, v = (torch.zeros(n, device="cuda").to(t) for t in ((torch.int8, torch.uint8) if eight else (torch.float32, torch.float32)))
    scales = [torch.zeros(-(-n // 256), device="cuda") for _ in range(2)]
    count = torch.zeros(2, dtype=torch.int32, device="cuda")
    B.ss_adamw_step([p], [tg], [m], [v], count, LR, betas=(B1, B2), eps=eps, **(dict(m_scale=[scales[0]], v_scale=[scales[1]]) if eight else {}))
    return p.double().cpu().numpy(), v, scales[1]


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -126, 1e-30, 1e-20, 1e-8])
def test_step(eps, bits):
    # second moments from 2^-149, the least number, to 2^-80, and a cut-off block
    g = np.exp(np.linspace(np.log(1.3e-21), np.log(1e-11), 1027)).astype(F) * np.where(np.arange(1027) % 2, 1, -1).astype(F)
    moment = g * g * F(1 - B2)
    assert moment.min() > 0 and (moment < 2.0 ** -126).sum() > 200
    p, v, scale = one_step(g, bits, eps)
    m = (g * F(1 - B1)).astype(np.float64)
    want = -LR / (1 - B1) * m / (np.sqrt(moment.astype(np.float64)) / np.sqrt(1 - B2) + eps)
    assert np.isfinite(p).all()
    assert (np.abs(p - want) <= 24 * 2.0 ** -24 * np.abs(want)).all()
    if bits == 32:
        assert np.array_equal(v.cpu().numpy(), moment)
    else:
        codes, a = codes_in_f32(np.sqrt(moment), 1, False)
        assert np.array_equal(scale.cpu().numpy(), a) and np.array_equal(v.cpu().numpy(), codes)
        assert (a > 0).all()


@pytest.mark.parametrize("bits", [8, 32])
def test_one_small_element_among_others(bits):
    """Lanes whose four elements are of all sizes, zeros among them: the others' bits are those of a step without it."""
    rng = np.random.default_rng(0)
    g = rng.standard_normal(512).astype(F)
    plain, v, _ = one_step(g, 32, 1e-8)
    h = g.copy()
    h[5::37], h[11::41] = 1e-19, 0.0
    got, w, _ = one_step(h, 32, 1e-8)
    same = h == g
    assert np.array_equal(got[same], plain[same]) and torch.equal(w[torch.from_numpy(same)], v[torch.from_numpy(same)])
    assert (got[11::41] == 0).all()
    small = one_step(h, bits, 1e-30)[0]
    assert np.isfinite(small).all() and (np.abs(small) <= LR * 1.01).all()
