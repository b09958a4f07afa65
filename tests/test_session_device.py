"""Which device a session lives on."""
import pytest
import torch

import decoder_util as D
from paper_2312_10351_amd import runtime
from paper_2312_10351_amd.runtime import Session


def test_a_device_without_a_number_is_the_current_one(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    assert str(runtime._placed("cuda")) == "cuda:3"
    assert str(runtime._placed("cuda:1")) == "cuda:1"
    assert str(runtime._placed(torch.device("cuda", 2))) == "cuda:2"


@pytest.mark.parametrize("current", [0, 1])
def test_tensors_of_another_device_are_refused(monkeypatch, current):
    """A session on "cuda" takes tensors of the device that was current when it was built, and of no other."""
    class Tensor(torch.Tensor):
        device = torch.device("cuda", 1)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
    s = Session.__new__(Session)
    s.device = str(runtime._placed("cuda"))
    t = torch.zeros(4).as_subclass(Tensor)
    if current == 1:
        assert s._upload(t) is t
    else:
        with pytest.raises(ValueError):
            s._upload(t)


@pytest.mark.gpu
@pytest.mark.parametrize("device", ["cuda", "cuda:0", torch.device("cuda")])
def test_a_session_on_the_current_device(device):
    x = D.normal(torch.Generator().manual_seed(1), (3, 128), "f16")
    s = D.bind(lambda b, e: b.rotary(e[0], 2, 64), [x], device=device)
    assert s.device == "cuda:0"
    s.launch()
    torch.cuda.synchronize()
    D.within(s.result(0), *D.rotary(x, 2, 64, 64, False, range(3)), "f16")
    s.close()
