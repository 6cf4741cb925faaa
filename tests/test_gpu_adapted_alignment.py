"""Pointers of the adapted projection on the smallest boundary that the call accepts, such as scales of several layers in one buffer."""
import pytest
import torch

from paper_2609_34054_b200.binding import AdaptedWeights, PreccError
from test_gpu_adapted import E4M3, _draw, _ids, forced, px  # noqa: F401

pytestmark = pytest.mark.gpu


def _moved(t, offset):
    """The same values, `offset` elements behind the start of an allocation."""
    flat = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
    flat[offset:] = t.reshape(-1)
    return flat[offset:].view(t.shape)


def _same_bits(px, rows, k, n, rank, agents, offset):
    x, w, A, B = _draw(k, n, rank, agents, rows, seed=offset)
    ids = _ids(rows, agents, "runs")
    wt = px.adapted_weights(w, A, B, 1.5, e4m3=True)
    xs = x.float().abs().amax(1) / 448
    xq = (x.float() / xs[:, None]).to(E4M3)
    ws = px.adapted_workspace(wt, rows)
    want, got = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda"), torch.full((rows, n), 7.0, dtype=torch.bfloat16, device="cuda")
    px.adapted_project_e4m3(wt, xq, xs, want, ids, ws)
    moved = AdaptedWeights(wt.desc, wt.W, wt.w_scale, wt.A, wt.B, _moved(wt.a_scale, offset))
    px.adapted_project_e4m3(moved, xq, _moved(xs, offset), got, _moved(ids, offset), ws)
    assert torch.equal(got, want)


@pytest.mark.parametrize("offset", [1, 2, 3])
@pytest.mark.parametrize("rows,rank", [(5, 16), (100, 64), (300, 64), (2300, 8), (1100, 16), (700, 32)])
def test_scales_and_ids_on_4_byte_boundaries(px, rows, rank, offset):  # noqa: F811
    _same_bits(px, rows, 512, 264, rank, 6, offset)


@pytest.mark.parametrize("rows,rank", [(3, 8), (16, 64), (200, 16), (513, 32)])
def test_every_kernel_takes_4_byte_boundaries(forced, rows, rank):  # noqa: F811
    _same_bits(forced, rows, 384, 136, rank, 5, 1)


@pytest.mark.parametrize("offset", [1, 2, 3])
def test_adapters_packed_to_4_byte_boundaries(px, offset):  # noqa: F811
    _, w, A, _ = _draw(256, 8, 16, 3, 4)
    wt = px.adapted_weights(w, A, torch.zeros((3, 16, 8), dtype=torch.bfloat16, device="cuda"), 1.0, e4m3=True)
    packed, scale = torch.zeros_like(wt.A), _moved(torch.zeros_like(wt.a_scale), offset)
    st = torch.cuda.current_stream().cuda_stream
    for a in range(3):
        px._check(px.lib.precc_pack_adapter_e4m3(px.h, A[a].data_ptr(), 256, 16, a, 3, packed.data_ptr(), scale.data_ptr(), st), "pack")
    assert torch.equal(packed.view(torch.uint8), wt.A.view(torch.uint8)) and torch.equal(scale, wt.a_scale)


def test_scales_of_columns_off_a_16_byte_boundary_are_refused(px):  # noqa: F811
    x, w, A, B = _draw(256, 64, 8, 2, 4)
    wt = px.adapted_weights(w, A, B, 1.0, e4m3=True)
    out = torch.full((4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    moved = AdaptedWeights(wt.desc, wt.W, _moved(wt.w_scale, 1), wt.A, wt.B, wt.a_scale)
    with pytest.raises(PreccError, match="16-byte aligned"):
        px.adapted_project_e4m3(moved, x.to(E4M3), torch.ones(4, device="cuda"), out, _ids(4, 2, "rows"), px.adapted_workspace(wt, 4))
    torch.cuda.synchronize()
    assert (out == 7).all()
