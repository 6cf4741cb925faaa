"""Argument checks of the norm's marshalling (no GPU: every case is refused before the library is called)."""
import pytest
import torch

from paper_2609_34054_b200 import binding


@pytest.fixture(scope="module")
def native():
    from paper_2609_34054_b200 import build
    build.build()
    binding.load_library()
    return binding._native


def _fake(shape, dtype=torch.bfloat16, device="cuda"):
    """A tensor that says it lies on a GPU and has no storage."""
    from torch._subclasses import FakeTensorMode
    with FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device=device)


def _call(**changed):
    a = dict(x=_fake((4, 64)), gain=_fake((64,)), eps=1e-5, out=_fake((4, 64)), residual=None, residual_out=None, q=None, scale=None)
    a.update(changed)
    return [0] + list(a.values())


@pytest.mark.parametrize("changed", [
    dict(x=None), dict(gain=None), dict(x=_fake((4, 64), torch.float32)), dict(gain=_fake((64,), torch.float32)),
    dict(out=_fake((4, 64), torch.float16)), dict(q=_fake((4, 64))), dict(scale=_fake((4,))), dict(x=[1.0]),
    dict(x=torch.zeros(4, 64, dtype=torch.bfloat16)), dict(x=_fake((4, 128))[:, :64])])
def test_wrong_tensors(native, changed):
    with pytest.raises(binding.PreccError):
        native.rms_norm(*_call(**changed))


def test_no_dimension_and_wrong_sizes(native):
    with pytest.raises(binding.PreccError, match="has no dimensions"):
        native.rms_norm(*_call(x=_fake(())))
    for changed in (dict(x=_fake((4, 32))), dict(x=_fake((8, 64)))):
        with pytest.raises(binding.PreccError):
            native.rms_norm(*_call(**changed))


def test_eps_and_argument_count(native):
    with pytest.raises(TypeError):
        native.rms_norm(*_call(eps="small"))
    with pytest.raises(TypeError):
        native.rms_norm(*_call()[:-1])
