"""Argument checks of the adapted projection's marshalling (no GPU: every case is refused before the library is called)."""
import ctypes

import pytest
import torch

from paper_2609_34054_b200 import binding
from paper_2609_34054_b200.binding import AdaptedWeights, ProjectionDesc

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def native():
    from paper_2609_34054_b200 import build
    build.build()
    binding.load_library()
    return binding._native


def _fake(shape, dtype=torch.bfloat16):
    """A tensor that says it lies on a GPU and has no storage."""
    from torch._subclasses import FakeTensorMode
    with FakeTensorMode():
        return torch.empty(shape, dtype=dtype, device="cuda")


def _weights(e4m3, **changed):
    k, n, agents, r = 256, 64, 3, 8
    w = dict(desc=ProjectionDesc(k, n, agents, r, 1.0), W=_fake((n, k), E4M3 if e4m3 else torch.bfloat16), w_scale=_fake((n,), torch.float32) if e4m3 else None,
             A=_fake((2 * agents * r, k), E4M3) if e4m3 else _fake((agents * r, k)), B=_fake((agents, r, n)),
             a_scale=_fake((agents * r,), torch.float32) if e4m3 else None)
    w.update(changed)
    return AdaptedWeights(**w)


def _call(e4m3, weights=None, **changed):
    a = dict(weights=weights or _weights(e4m3), x=_fake((4, 256), E4M3 if e4m3 else torch.bfloat16))
    if e4m3:
        a["x_scale"] = _fake((4,), torch.float32)
    a.update(out=_fake((4, 64)), agent_id=_fake((4,), torch.int32), workspace=_fake((256,), torch.uint8))
    a.update(changed)
    return [0] + list(a.values())


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("changed,match", [
    (dict(x=None), "x is None"), (dict(x=_fake((4, 256), torch.float32)), "x must be"), (dict(out=None), "out is None"),
    (dict(out=_fake((4, 64), torch.float32)), "out must be"), (dict(out=_fake((4, 32))), "elements"), (dict(agent_id=_fake((4,), torch.int64)), "agent_id must be"),
    (dict(agent_id=_fake((5,), torch.int32)), "elements"), (dict(x=torch.zeros(4, 256)), "contiguous CUDA")])
def test_wrong_tensors(native, e4m3, changed, match):
    with pytest.raises(binding.PreccError, match=match):
        (native.adapted_project_e4m3 if e4m3 else native.adapted_project)(*_call(e4m3, **changed))


@pytest.mark.parametrize("e4m3", [False, True])
def test_wrong_width_and_no_dimension(native, e4m3):
    call = native.adapted_project_e4m3 if e4m3 else native.adapted_project
    dtype = E4M3 if e4m3 else torch.bfloat16
    with pytest.raises(binding.PreccError, match="has 128 columns, the projection takes 256"):
        call(*_call(e4m3, x=_fake((4, 128), dtype)))
    with pytest.raises(binding.PreccError, match="has no dimensions"):
        call(*_call(e4m3, x=_fake((), dtype)))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("changed,match", [
    (dict(W=None), "weights.W is None"), (dict(W=_fake((64, 128))), "weights.W"), (dict(A=None), "weights.A is None"), (dict(A=_fake((8, 256))), "weights.A"),
    (dict(B=None), "weights.B is None"), (dict(B=_fake((3, 8, 32))), "weights.B"), (dict(desc=b"short"), "ProjectionDesc")])
def test_wrong_weights(native, e4m3, changed, match):
    with pytest.raises(binding.PreccError, match=match):
        (native.adapted_project_e4m3 if e4m3 else native.adapted_project)(*_call(e4m3, weights=_weights(e4m3, **changed)))


@pytest.mark.parametrize("changed,match", [(dict(w_scale=None), "w_scale is None"), (dict(w_scale=_fake((32,), torch.float32)), "w_scale has 32"),
                                           (dict(a_scale=None), "a_scale is None"), (dict(a_scale=_fake((24,))), "a_scale must be")])
def test_wrong_scales(native, changed, match):
    with pytest.raises(binding.PreccError, match=match):
        native.adapted_project_e4m3(*_call(True, weights=_weights(True, **changed)))
    with pytest.raises(binding.PreccError, match="x_scale is None"):
        native.adapted_project_e4m3(*_call(True, x_scale=None))


def test_not_weights_at_all(native):
    with pytest.raises(AttributeError):
        native.adapted_project(*_call(False, weights=object()))
    with pytest.raises(TypeError):
        native.adapted_project(*_call(False)[:-1])


def test_workspace_sizes(native):
    lib = binding.load_library()
    d = ProjectionDesc(256, 64, 3, 8, 1.0)
    assert lib.precc_adapted_ws_bytes(ctypes.byref(d), 1) == 256
    assert lib.precc_adapted_ws_bytes(ctypes.byref(d), 100) == 3328            # 16 coordinates a row at least, whole 256 bytes
    assert lib.precc_adapted_ws_bytes(ctypes.byref(ProjectionDesc(256, 64, 3, 64, 1.0)), 100) == 12800
    assert lib.precc_adapted_ws_bytes(ctypes.byref(ProjectionDesc(256, 64, 0, 0, 1.0)), 100) == 0
    assert lib.precc_adapted_ws_bytes(ctypes.byref(d), 0) == 0 and lib.precc_adapted_ws_bytes(None, 5) == 0
