"""AdamW's groups: a rate on the device through a file, groups that are refused leave the optimiser as it was."""
import io

import pytest
import torch

from paper_2312_00752_amd import optim

pytestmark = pytest.mark.gpu


def made(lr, shape=(300,), **options):
    torch.manual_seed(0)
    p = torch.nn.Parameter(torch.randn(shape, device="cuda"))
    p.grad = torch.randn_like(p)
    return p, optim.AdamW([p], lr=lr, **options)


def through_a_file(state, device):
    file = io.BytesIO()
    torch.save(state, file)
    file.seek(0)
    return torch.load(file, map_location=device, weights_only=True)


@pytest.mark.parametrize("device", ["cpu", "cuda"])
@pytest.mark.parametrize("mine", ["number", "tensor"])
@pytest.mark.parametrize("theirs", ["number", "tensor", "float64", "scheduled"])
def test_rate_through_a_file(theirs, mine, device):
    """A number or a tensor, saved or to be replaced, read onto either device: the next steps are those of the saved run."""
    rate = {"number": lambda v: v, "tensor": lambda v: torch.tensor([v], device="cuda"), "scheduled": lambda v: torch.tensor(v, device="cuda")}
    p, a = made(rate.get(theirs, rate["number"])(3e-3))
    if theirs == "scheduled":
        schedule = torch.optim.lr_scheduler.StepLR(a, 1, gamma=1.0)
    a.step()
    saved = through_a_file(a.state_dict(), device)
    if theirs == "float64":   # as another program may have written it
        saved["param_groups"][0]["lr"] = torch.tensor(3e-3, dtype=torch.float64, device=device)
    q, b = made(rate[mine](7.0))
    with torch.no_grad():
        q.copy_(p)
    own = b.param_groups[0]["lr"]
    b.load_state_dict(saved)
    lr = b.param_groups[0]["lr"]
    assert float(lr) == pytest.approx(3e-3, rel=2.0 ** -23)
    if mine == "tensor":
        assert lr is own   # what a captured step reads
    elif theirs != "number":
        assert lr.dtype == torch.float32 and lr.is_cuda and lr is not a.param_groups[0]["lr"]
    for _ in range(3):
        a.step()
        b.step()
    assert torch.equal(p, q)


def test_a_refused_group_is_not_added():
    p, opt = made(1e-3)
    more = torch.nn.Parameter(torch.ones(5, device="cuda"))
    bad = [torch.nn.Parameter(torch.ones(3)), torch.nn.Parameter(torch.ones(3, device="cuda").half()), torch.nn.Parameter(torch.ones(4, 6, device="cuda")[:, ::2])]
    for group in [{"params": [more, b]} for b in bad] + [{"params": [more], "state_bits": 16}, {"params": [more], "state_bits": 0}]:
        with pytest.raises(ValueError):
            opt.add_param_group(group)
        assert len(opt.param_groups) == 1 and more not in opt.state
    opt.step()
    opt.add_param_group({"params": [more], "state_bits": 8})
    more.grad = torch.ones_like(more)
    opt.step()
    assert opt.state[more]["m"].dtype == torch.int8
    assert [g["count"].tolist() for g in opt.param_groups] == [[2, 0], [1, 0]]
