"""Weights that Precc.adapted_weights refuses before it packs anything (no GPU)."""
import pytest
import torch

from paper_2609_34054_b200.binding import Precc, PreccError


class _Library:
    def __getattr__(self, name):
        raise AssertionError(f"{name} is called")


def _context(device):
    px = Precc.__new__(Precc)
    px.device, px.lib, px.h = device, _Library(), None
    return px


def _fake(*shape):
    """A tensor that says it lies on a GPU and has no storage."""
    from torch._subclasses import FakeTensorMode
    with FakeTensorMode():
        return torch.empty(shape, dtype=torch.bfloat16, device="cuda:0")


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("wrong", ["W on the host", "A on the host", "B on the host", "W strided", "A strided", "B strided"])
def test_weights_elsewhere(e4m3, wrong):
    t = dict(W=_fake(256, 64), A=_fake(3, 256, 8), B=_fake(3, 8, 64))
    name = wrong[0]
    if "host" in wrong:
        t[name] = torch.zeros(t[name].shape, dtype=torch.bfloat16)
    else:
        t[name] = _fake(*t[name].shape[:-1], 2 * t[name].shape[-1])[..., ::2]
    with pytest.raises(PreccError, match="contiguous tensors on the context's device 0"):
        _context(0).adapted_weights(t["W"], t["A"], t["B"], 1.0, e4m3=e4m3)


def test_a_context_on_another_device():
    with pytest.raises(PreccError, match="context's device 1"):
        _context(1).adapted_weights(_fake(256, 64), None, None, 1.0)


def test_another_current_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(PreccError, match="not the current one"):
        _context(0).adapted_weights(_fake(256, 64), None, None, 1.0)
