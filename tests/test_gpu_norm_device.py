"""The norms' calls with tensors on another device than the current one, which their launch would not be ordered with: refused on either path, before anything is launched.

There is one device: the binding is told that the current one is another, with the stream left as it is."""
import pytest
import torch

from paper_2312_00752_amd import autograd as ag
from paper_2312_00752_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[False, True], ids=["compiled", "python"])
def elsewhere(request, monkeypatch):
    B._marshal()
    stream = torch.cuda.current_stream().cuda_stream
    B._stream(None)
    if request.param:
        monkeypatch.setattr(B, "_native", B._NoMarshal)
    monkeypatch.setattr(B, "_raw_stream", lambda _: stream)
    monkeypatch.setattr(B, "_device_index", lambda: 1)


X = lambda: torch.randn(4, 40, device="cuda")
CALLS = {
    "layer": lambda x: B.ss_norm_fwd(x),
    "rms": lambda x: B.ss_norm_fwd(x, rms=True),
    "into": lambda x: B.ss_norm_fwd(x, out=torch.empty_like(x)),
    "quant": lambda x: B.ss_norm_quant(x),
    "rms quant": lambda x: B.ss_norm_quant(x, residual=x.clone(), rms=True),
    "backward": lambda x: B.ss_norm_bwd(x, x, torch.ones(2, 4, device="cuda")),
    "rms backward": lambda x: B.ss_norm_bwd(x, x, torch.ones(4, device="cuda"), rms=True),
    "layer_norm": lambda x: ag.layer_norm(x.requires_grad_(True)),
    "rms_norm": lambda x: ag.rms_norm(x.requires_grad_(True), residual=x),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_refused(name, elsewhere):
    with pytest.raises(ValueError, match="current device is cuda:1"):
        CALLS[name](X())


@pytest.mark.parametrize("name", sorted(CALLS))
def test_served_on_the_current_device(name):
    CALLS[name](X())
