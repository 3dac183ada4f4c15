"""Each of the norms' tensors is looked at for its device: one alone elsewhere is refused, whichever it is."""
import pytest
import torch

from paper_2312_00752_amd import binding as B


class On(torch.Tensor):
    """A tensor that says that it lies on a GPU."""
    index = 0
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.index))

    def get_device(self):
        return self.index


def on(index, *shape):
    t = torch.zeros(shape).as_subclass(On)
    t.index = index
    return t


FWD = dict(x=(4, 40), weight=(40,), bias=(40,), residual=(4, 40), summed=(4, 40))
CALLS = {
    "fwd": (lambda **t: B.ss_norm_fwd(t.pop("x"), **t), dict(FWD, out=(4, 40))),
    "rms fwd": (lambda **t: B.ss_norm_fwd(t.pop("x"), rms=True, **t), dict(FWD, out=(4, 40))),
    "quant": (lambda **t: B.ss_norm_quant(t.pop("x"), **t), FWD),
    "bwd": (lambda **t: B.ss_norm_bwd(t.pop("dout"), t.pop("s"), t.pop("stats"), residual_dtype=torch.float32, **t),
            dict(dout=(4, 40), s=(4, 40), stats=(2, 4), weight=(40,), dsummed=(4, 40), workspace=(1 << 20,))),
}


@pytest.fixture
def first_device(monkeypatch):
    monkeypatch.setattr(B, "_native", B._NoMarshal)
    monkeypatch.setattr(B, "_raw_stream", lambda _: 0)
    monkeypatch.setattr(B, "_device_index", lambda: 0)
    monkeypatch.setattr(B, "lib", lambda: pytest.fail("the call went on"))


@pytest.mark.parametrize("call,name", [(c, n) for c in sorted(CALLS) for n in CALLS[c][1]])
def test_one_tensor_elsewhere(call, name, first_device):
    f, shapes = CALLS[call]
    with pytest.raises(ValueError, match="lies on cuda:1, the current device is cuda:0"):
        f(**{n: on(int(n == name), *s) for n, s in shapes.items()})
