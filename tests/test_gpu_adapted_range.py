"""The adapted projections at the ends of the range: row and column scales of 8 bits whose product leaves fp32's, rows with infinities."""
import pytest
import torch

from test_gpu_adapted import E4M3, _draw, _ids, _quantised, _reference, forced, px  # noqa: F401

pytestmark = pytest.mark.gpu
LEAST = 2.0**-134                                # half of bf16's least step


def _scaled(px, rows, rank, row_scale, w_std):
    """Rows with scales around row_scale, columns around w_std.  The bound is that of ordinary sizes, taken in units of the two."""
    k, n, agents = 256, 264, 4
    x, w, A, B = _draw(k, n, rank, agents, rows, seed=7)
    w, B = ((t.double() * (w_std / 0.02)).to(torch.bfloat16) if t is not None else None for t in (w, B))
    ids = _ids(rows, agents, "rows")
    wt = px.adapted_weights(w, A, B, 1.5, e4m3=True)
    xq = (x.float() * 100).clamp(-448, 448).to(E4M3)
    if rows > 1:
        xq[rows // 8] = 0
    xs = (row_scale * (1 + torch.arange(rows, device="cuda") % 4)).float()
    out = torch.full((rows, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    px.adapted_project_e4m3(wt, xq, xs, out, ids, px.adapted_workspace(wt, rows))
    wq, s = _quantised(w)
    y, bound = _reference(xq.double(), wq.double() * s, A, B, ids, 1.5, True)
    y, bound = y * xs.double()[:, None], (bound - 1e-30) * xs.double()[:, None]
    assert rows == 1 or (out[rows // 8] == 0).all()
    assert ((out.double() - y).abs() <= bound * (1 + 2.0**-20) + LEAST).all()


# the least scale that the norm leaves, and one that a product with the columns' takes out of fp32; then the large side
SIZES = [(2.0**-126, 0.02), (2.0**-100, 2.0**-40), (2.0**-122, 2.0**-10), (2.0**-60, 2.0**-70), (2.0**70, 2.0**30), (2.0**-120, 2.0**90), (2.0**80, 2.0**-90)]


@pytest.mark.parametrize("row_scale,w_std", SIZES)
@pytest.mark.parametrize("rows,rank", [(1, 16), (7, 8), (30, 0), (100, 32), (600, 16), (2500, 64)])
def test_scales_whose_product_leaves_the_range(px, rows, rank, row_scale, w_std):  # noqa: F811
    _scaled(px, rows, rank, row_scale, w_std)


@pytest.mark.parametrize("row_scale,w_std", SIZES[:2])
@pytest.mark.parametrize("rows", [3, 70, 300])
def test_every_kernel_keeps_small_scales(forced, rows, row_scale, w_std):  # noqa: F811
    _scaled(forced, rows, 16, row_scale, w_std)


@pytest.mark.parametrize("row_scale,w_std", [(2.0**100, 2.0**38)])
@pytest.mark.parametrize("rows", [3, 70, 700])
def test_zeros_under_scales_whose_product_overflows(px, rows, row_scale, w_std):  # noqa: F811
    k, n = 256, 64
    _, w, _, _ = _draw(k, n, 0, 0, rows)
    wt = px.adapted_weights((w.double() * w_std / 0.02).to(torch.bfloat16), None, None, 1.0, e4m3=True)
    xq = torch.zeros((rows, k), dtype=E4M3, device="cuda")
    out = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    px.adapted_project_e4m3(wt, xq, torch.full((rows,), row_scale, device="cuda"), out)
    assert (out == 0).all()


def _infinite_row(px, rows, rank):
    """Weights and adapters above zero: a row with an infinity is infinite in every column, and no padding of the rank makes it NaN."""
    k, n, agents = 256, 72, 3
    x, w, A, B = (t.abs() + 0.01 for t in _draw(k, n, rank, agents, rows))
    ids = _ids(rows, agents, "one")
    ws = px.adapted_workspace(px.adapted_weights(w, A, B, 1.0), rows).fill_(255)
    x[rows // 2, 3] = float("inf")
    out = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    px.adapted_project(px.adapted_weights(w, A, B, 1.0), x, out, ids, ws)
    assert (out[rows // 2] == float("inf")).all()
    others = torch.arange(rows, device="cuda") != rows // 2
    assert torch.isfinite(out[others]).all()


@pytest.mark.parametrize("rank", [8, 16, 64])
@pytest.mark.parametrize("rows", [1, 9, 30, 70, 700, 2500])
def test_a_row_with_an_infinity(px, rows, rank):  # noqa: F811
    _infinite_row(px, rows, rank)


@pytest.mark.parametrize("rank", [8, 32])
@pytest.mark.parametrize("rows", [5, 70, 300])
def test_a_row_with_an_infinity_in_every_kernel(forced, rows, rank):  # noqa: F811
    _infinite_row(forced, rows, rank)
