"""precc_rms_norm against the definition in 64 bits: widths from one piece to the widest row, both outputs, in place, rows that
hold zeros, infinities and NaN, captured and on another stream, and what it refuses."""
import pytest
import torch

from paper_2609_34054_b200 import inputs as I
from paper_2609_34054_b200.binding import Precc, PreccError

pytestmark = pytest.mark.gpu
EPS = 1e-5
E4M3 = torch.float8_e4m3fn
# relative error of y in fp32: the sum of squares adds at most 32768 terms, in partial sums of at most 32 x 8 and a tree (2^-24 each
# of at most 300 additions, halved by the root), the fast root and reciprocal 2^-21, three products
Y_REL = 150 * 2.0**-24 + 2.0**-21 + 3 * 2.0**-24


@pytest.fixture(scope="module")
def px():
    p = Precc(0)
    yield p
    torch.cuda.synchronize()
    assert p.poll_status() == 0
    p.close()


def _inputs(rows, width, seed=0, residual=True):
    x = I.normal_bf16((rows, width), 3.0, seed, "norm.x").cuda()
    r = I.normal_bf16((rows, width), 5.0, seed, "norm.r").cuda() if residual else None
    g = I.normal_bf16((width,), 1.0, seed, "norm.g").cuda()
    return x, r, g


def _reference(x, r, g, eps=EPS):
    s = x.double() + (r.double() if r is not None else 0)
    return s, s / (s.square().mean(-1, keepdim=True) + eps).sqrt() * g.double()


def _check(x, r, g, out, res_out, q, scale, eps=EPS):
    s, y = _reference(x, r, g, eps)
    if res_out is not None:
        # (the sum of two bf16 in fp32 is off by 2^-24, then one rounding to bf16)
        assert ((res_out.double() - s).abs() <= (2.0**-8 + 2.0**-23) * s.abs()).all()
    if out is not None:
        assert ((out.double() - y).abs() <= (2.0**-8 + 2 * Y_REL) * y.abs() + 1e-37).all()
    if q is not None:
        top = y.abs().amax(-1)
        want = torch.where(top == 0, torch.ones_like(top), top / 448)
        assert ((scale.double().view(top.shape) - want).abs() <= 2 * Y_REL * want).all()
        z = y / want.unsqueeze(-1)
        # half a step of e4m3: 2^-4 of the value, 2^-10 among the subnormals
        assert ((q.double() - z).abs() <= torch.maximum(z.abs() * (2.0**-4 + 4 * Y_REL), torch.full_like(z, 2.0**-10 + 2.0**-18))).all()
        assert (q.double().abs().amax(-1)[top > 0] == 448).all()


@pytest.mark.parametrize("width", [8, 16, 24, 64, 120, 128, 256, 264, 1000, 2048, 3584, 4096, 8192, 8200, 16384, 32768])
@pytest.mark.parametrize("rows", [1, 3, 37, 700, 2001])
def test_norm_matches_the_definition(px, rows, width):
    x, r, g = _inputs(rows, width, seed=width + rows)
    out, res_out = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    q, scale = torch.zeros(x.shape, dtype=E4M3, device="cuda"), torch.full((rows,), -1.0, device="cuda")
    px.rms_norm(x, g, EPS, out=out, residual=r, residual_out=res_out, out_e4m3=q, out_scale=scale)
    _check(x, r, g, out, res_out, q, scale)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("outputs", ["bf16", "e4m3"])
@pytest.mark.parametrize("width", [128, 520, 4096, 16000])
@pytest.mark.parametrize("rows", [301, 5003])
def test_norm_forms(px, rows, width, outputs, residual):
    x, r, g = _inputs(rows, width, seed=5, residual=residual)
    out = torch.empty_like(x) if outputs == "bf16" else None
    q = torch.empty(x.shape, dtype=E4M3, device="cuda") if outputs == "e4m3" else None
    scale = torch.empty(rows, device="cuda") if outputs == "e4m3" else None
    px.rms_norm(x, g, EPS, out=out, residual=r, out_e4m3=q, out_scale=scale)
    _check(x, r, g, out, None, q, scale)


@pytest.mark.parametrize("width", [16384, 16392, 24000, 32768])
@pytest.mark.parametrize("rows", [1, 148, 149, 300])
def test_widest_rows_without_residual(px, rows, width):
    x, _, g = _inputs(rows, width, seed=width, residual=False)
    out = torch.full_like(x, float("nan"))
    px.rms_norm(x, g, EPS, out=out)
    _check(x, None, g, out, None, None, None)


@pytest.mark.parametrize("width", [64, 4096])
def test_norm_in_place(px, width):
    x, r, g = _inputs(65, width, seed=9)
    want, want_res = torch.empty_like(x), torch.empty_like(x)
    px.rms_norm(x, g, EPS, out=want, residual=r, residual_out=want_res)
    px.rms_norm(x, g, EPS, out=x, residual=r, residual_out=r)
    assert torch.equal(x, want) and torch.equal(r, want_res)


def test_norm_of_query_heads(px):
    """Per-head norm: the last dimension is the width, the others are rows."""
    q = I.queries(7, I.C4, 3).cuda()
    g = I.normal_bf16((I.C4.hd,), 1.0, 3, "norm.head").cuda()
    out = torch.empty_like(q)
    px.rms_norm(q, g, EPS, out=out)
    _check(q, None, g, out, None, None, None)


def test_rows_behind_the_last_one_stay(px):
    x, r, g = _inputs(10, 96, seed=1)
    q, scale = torch.full((10, 96), 3.0, device="cuda").to(E4M3), torch.full((10,), 7.0, device="cuda")
    out, res_out = torch.full_like(x, 5.0), torch.full_like(x, 6.0)
    px.rms_norm(x[:7], g, EPS, out=out[:7], residual=r[:7], residual_out=res_out[:7], out_e4m3=q[:7], out_scale=scale[:7])
    _check(x[:7], r[:7], g, out[:7], res_out[:7], q[:7], scale[:7])
    assert (out[7:] == 5).all() and (res_out[7:] == 6).all() and (q[7:].float() == 3).all() and (scale[7:] == 7).all()


@pytest.mark.parametrize("width", [64, 2048])
def test_rows_of_zeros_and_non_finite_rows(px, width):
    x, _, g = _inputs(9, width, seed=2, residual=False)
    x[1] = 0
    x[3, 5] = float("inf")
    x[5, 7] = float("nan")
    x[7] = 1e30
    out = torch.empty_like(x)
    q, scale = torch.empty(x.shape, dtype=E4M3, device="cuda"), torch.empty(9, device="cuda")
    px.rms_norm(x, g, EPS, out=out, out_e4m3=q, out_scale=scale)
    fine = [0, 2, 4, 6, 8]
    _check(x[fine], None, g, out[fine], None, q[fine], scale[fine])
    assert (out[1] == 0).all() and (q[1].float() == 0).all() and scale[1] == 1
    assert torch.isnan(out[3, 5]) and not torch.isfinite(scale[3])
    assert torch.isnan(out[5]).all() and torch.isnan(scale[5]) and torch.isnan(q[5].float()).all()


@pytest.mark.parametrize("rows", [5, 200, 1500])
@pytest.mark.parametrize("width", [8, 64, 264, 1000, 4096, 32768])
def test_rows_whose_squares_overflow(px, rows, width):
    """Rows around the square root of fp32's largest number and up to bf16's own, between ordinary ones."""
    x, r, g = _inputs(rows, width, seed=rows + width)
    x[1::3] = (x[1::3].double() * 2.0**63).to(torch.bfloat16)
    x[2, -1] = torch.finfo(torch.bfloat16).min
    x[4] = torch.finfo(torch.bfloat16).max
    r[4] = 0
    out, res_out = torch.empty_like(x), torch.empty_like(x)
    q, scale = torch.empty(x.shape, dtype=E4M3, device="cuda"), torch.empty(rows, device="cuda")
    px.rms_norm(x, g, EPS, out=out, residual=r, residual_out=res_out, out_e4m3=q, out_scale=scale)
    _check(x, r, g, out, res_out, q, scale)
    if rows == 5:                                 # ordinary rows are the same bits alone
        alone = torch.empty_like(x[3:4])
        px.rms_norm(x[3:4], g, EPS, out=alone, residual=r[3:4])
        assert torch.equal(alone, out[3:4])


@pytest.mark.parametrize("size", [1e-18, 1e-30])
def test_tiny_rows(px, size):
    """Values whose squares vanish beside eps; the scale stays a normal number with a finite reciprocal."""
    g = torch.ones(256, dtype=torch.bfloat16, device="cuda")
    x = (I.normal_bf16((4, 256), 1.0, 4, "norm.tiny").double().cuda() * size).to(torch.bfloat16)
    out, q, scale = torch.empty_like(x), torch.empty(x.shape, dtype=E4M3, device="cuda"), torch.empty(4, device="cuda")
    px.rms_norm(x, g, EPS, out=out, out_e4m3=q, out_scale=scale)
    _check(x, None, g, out, None, q, scale)


def test_norm_without_eps(px):
    x, r, g = _inputs(5, 640, seed=6)
    out = torch.empty_like(x)
    px.rms_norm(x, g, 0.0, out=out, residual=r)
    _check(x, r, g, out, None, None, None, eps=0.0)


def test_more_than_2_to_the_31_elements(px):
    """Offsets past 32 bits: the last rows of a tensor of 4.3 GB."""
    rows, width = 65537, 32768
    x = torch.zeros((rows, width), dtype=torch.bfloat16, device="cuda")
    x[-3:] = I.normal_bf16((3, width), 2.0, 8, "norm.far").cuda()
    g = I.normal_bf16((width,), 1.0, 8, "norm.far.g").cuda()
    px.rms_norm(x, g, EPS, out=x, residual=None)
    want = _reference(I.normal_bf16((3, width), 2.0, 8, "norm.far").cuda(), None, g)[1]
    assert ((x[-3:].double() - want).abs() <= (2.0**-8 + 2 * Y_REL) * want.abs() + 1e-37).all()
    assert (x[:-3].abs().amax() == 0)


def test_captured_and_on_another_stream(px):
    x, r, g = _inputs(33, 2048, seed=12)
    out, acc = torch.empty_like(x), r.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        px.rms_norm(x, g, EPS, out=out, residual=acc, residual_out=acc)
    side.synchronize()
    _check(x, r, g, out, acc, None, None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        px.rms_norm(x, g, EPS, out=out, residual=acc, residual_out=acc)      # the stream grows by x with every replay
        px.rms_norm(out, g, EPS, out=out)
    now = acc.clone()
    graph.replay()
    torch.cuda.synchronize()
    first = torch.empty_like(x)
    px.rms_norm(x, g, EPS, out=first, residual=now, residual_out=now)
    px.rms_norm(first, g, EPS, out=first)
    assert torch.equal(acc, now) and torch.equal(out, first)


def test_refusals(px):
    x, r, g = _inputs(4, 64)
    q, scale = torch.empty(x.shape, dtype=E4M3, device="cuda"), torch.empty(4, device="cuda")
    out = torch.full_like(x, 7.0)

    def refused(match, *a, **k):
        with pytest.raises(PreccError, match=match):
            px.rms_norm(*a, **k)

    refused("neither", x, g, EPS)
    refused("come together", x, g, EPS, out=out, out_e4m3=q)
    refused("come together", x, g, EPS, out=out, out_scale=scale)
    refused("eps", x, g, -1.0, out=out)
    refused("eps", x, g, float("nan"), out=out)
    refused("not a multiple of 8", x[:, :63].contiguous(), g[:63].contiguous(), EPS, out=out[:, :63].contiguous())
    refused("contiguous", x[:, :32], g[:32], EPS, out=out[:, :32])
    refused("elements", x, g[:32], EPS, out=out)
    refused("elements", x, g, EPS, out=out[:2])
    refused("elements", x, g, EPS, out=out, residual=r[:1])
    refused("must be", x.float(), g, EPS, out=out)
    refused("must be", x, g, EPS, out=out, residual=r.float())
    refused("must be", x, g, EPS, out_e4m3=out, out_scale=scale)
    flat = torch.empty(4 * 64 + 4, dtype=torch.bfloat16, device="cuda")
    refused("16-byte aligned", flat[1:257].view(4, 64), g, EPS, out=out)
    wide = torch.empty((1, 32776), dtype=torch.bfloat16, device="cuda")
    refused("up to 32768", wide, wide[0], EPS, out=wide)
    px.rms_norm(x[:0], g, EPS, out=out[:0])
    torch.cuda.synchronize()
    assert (out == 7).all()


def test_device_of_the_context(px):
    """Tensors on the host are refused before anything is launched."""
    x, _, g = _inputs(4, 64)
    with pytest.raises(PreccError, match="CUDA"):
        px.rms_norm(x.cpu(), g, EPS, out=torch.empty_like(x))
