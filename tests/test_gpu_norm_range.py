"""precc_rms_norm at the ends of bf16's range: no eps or a tiny one under rows whose squares vanish, sums past fp32's largest number, subnormal
values among ordinary ones."""
import pytest
import torch

from paper_2609_34054_b200 import inputs as I
from test_gpu_norm import E4M3, Y_REL, _reference, px  # noqa: F401

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
TOP = torch.finfo(BF16).max
# half of bf16's least step, 2^-133: what a rounding among the subnormals may be off
LEAST = 2.0**-134


def _rows(rows, width, size, seed):
    """Rows of N(0, size^2), rounded to bf16 (subnormals included), as x and residual."""
    draw = lambda tag: (I.normal_bf16((rows, width), 1.0, seed, tag).cuda().double() * size).to(BF16)  # noqa: E731
    return draw("range.x"), draw("range.r")


def _check(px, x, r, g, eps):  # noqa: F811
    """All four outputs against 64 bits.  eps: as fp32 holds it."""
    eps = torch.tensor(eps, dtype=torch.float32).item()
    rows = x.shape[0]
    out, res_out = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    q, scale = torch.zeros(x.shape, dtype=E4M3, device="cuda"), torch.full((rows,), -1.0, device="cuda")
    px.rms_norm(x, g, eps, out=out, residual=r, residual_out=res_out, out_e4m3=q, out_scale=scale)
    s, y = _reference(x, r, g, eps)
    # one addition in fp32 (2^-24), one rounding to bf16; from bf16's largest number and half a step on it is infinite
    edge = TOP + 2.0**119
    over, fine = s.abs() >= edge * (1 + 2.0**-23), s.abs() < edge * (1 - 2.0**-23)
    assert torch.equal(res_out[over].double(), torch.sign(s[over]) * float("inf"))
    assert ((res_out.double() - s).abs() <= (2.0**-8 + 2.0**-23) * s.abs() + LEAST)[fine].all()
    assert ((out.double() - y).abs() <= (2.0**-8 + 2 * Y_REL) * y.abs() + LEAST).all()
    top = y.abs().amax(-1)
    want = torch.where(top == 0, torch.ones_like(top), (top / 448).clamp_min(2.0**-126))
    assert ((scale.double() - want).abs() <= 2 * Y_REL * want).all()
    z = y / want[:, None]
    assert ((q.double() - z).abs() <= torch.maximum(z.abs() * (2.0**-4 + 4 * Y_REL), torch.full_like(z, 2.0**-10 + 2.0**-18))).all()


def _gain(width):
    return I.normal_bf16((width,), 1.0, 3, "range.g").cuda()


SHAPES = [(1, 8), (5, 64), (300, 264), (1500, 128), (1300, 1000), (200, 4096), (3, 32768)]


@pytest.mark.parametrize("size", [1e-17, 1e-19, 1e-21, 1e-25, 1e-32, 1e-37, 1e-39])
@pytest.mark.parametrize("rows,width", SHAPES)
def test_tiny_rows_without_eps(px, rows, width, size):  # noqa: F811
    x, r = _rows(rows, width, size, seed=width)
    x[:, 0] = size                               # (no row of zeros: without eps that is 0 / 0)
    r[:, 0] = 0
    x[rows // 2] = (I.normal_bf16((width,), 1.0, 1, "range.mid").cuda())
    r[rows // 2] = 0
    _check(px, x, r, _gain(width), 0.0)


@pytest.mark.parametrize("eps", [1e-45, 1e-41, 1e-38, 1e-34, 1e-30, 1e-24])
@pytest.mark.parametrize("size", [1e-12, 1e-17, 1e-19, 1e-22, 1e-30, 1e-39])
def test_tiny_rows_with_a_tiny_eps(px, eps, size):  # noqa: F811
    x, r = _rows(37, 520, size, seed=4)
    x[3], r[3] = 0, 0
    _check(px, x, r, _gain(520), eps)


@pytest.mark.parametrize("rows,width", SHAPES)
def test_sums_past_fp32(px, rows, width):  # noqa: F811
    """x + residual passes fp32's largest number where both are near bf16's."""
    x, r = _rows(rows, width, 1.0, seed=width)
    x[0] = r[0] = TOP
    m = rows // 2
    x[m, ::2] = r[m, ::2] = -TOP
    x[m, 1::4], r[m, 1::4] = TOP, -TOP
    if rows > 1:                                 # (a row of its own: the one above times 2^125 would hold infinities)
        x[rows - 1] = (x[rows - 1].double() * 2.0**125).to(BF16)
        r[rows - 1, -1] = TOP
    _check(px, x, r, _gain(width), 1e-5)


@pytest.mark.parametrize("rows,width", SHAPES)
def test_subnormals_among_ordinary_values(px, rows, width):  # noqa: F811
    x, r = _rows(rows, width, 1.0, seed=width)
    small, small_r = _rows(rows, width, 1e-39, seed=width + 1)
    x[:, 1::3], r[:, 1::3] = small[:, 1::3], small_r[:, 1::3]
    _check(px, x, r, torch.ones(width, dtype=BF16, device="cuda"), 1e-5)


@pytest.mark.parametrize("size", [1e-36, 1e-39])
def test_outputs_among_the_subnormals(px, size):  # noqa: F811
    """An eps that outweighs the row leaves y where it is, and the 8-bit scale at the least normal number."""
    x, r = _rows(9, 264, size, seed=8)
    _check(px, x, r, torch.ones(264, dtype=BF16, device="cuda"), 1.0)
