"""precc_adapted_project / _e4m3 against the definition in 64 bits: one row to thousands, odd sizes, every rank, agents in runs and row by row,
rows without an adapter, adapters and rows that hold NaN, packing, captured calls, and what is refused."""
import math
import os

import pytest
import torch

from paper_2609_34054_b200 import inputs as I
from paper_2609_34054_b200.binding import AdaptedWeights, Precc, PreccError, ProjectionDesc

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def px():
    p = Precc(0)
    yield p
    torch.cuda.synchronize()
    assert p.poll_status() == 0
    p.close()


@pytest.fixture(scope="module", params=[("turn", "mma"), ("turn", "tc"), ("pair", "mma"), ("pair", "tc"), ("few", "tc")], ids="-".join)
def forced(request):
    """A context that takes one pair of kernels wherever they can take the call."""
    old = {k: os.environ.get(k) for k in ("PRECC_ADAPTED", "PRECC_ADAPTED_SHRINK")}
    os.environ["PRECC_ADAPTED"], os.environ["PRECC_ADAPTED_SHRINK"] = request.param
    try:
        p = Precc(0)
    finally:
        for k, v in old.items():
            os.environ.pop(k) if v is None else os.environ.__setitem__(k, v)
    yield p
    torch.cuda.synchronize()
    assert p.poll_status() == 0
    p.close()


def _ids(rows, agents, mix, seed=0):
    if mix == "none":
        return None
    if mix == "one":
        return torch.full((rows,), agents - 1, dtype=torch.int32, device="cuda")
    if mix == "neutral":
        return torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    if mix == "runs":
        return ((torch.arange(rows) * (agents + 1) // rows + 1) % (agents + 1) - 1).to(torch.int32).cuda()
    return (I.uniform_int(-1, agents - 1, rows, seed, "adapted.ids")).cuda()


def _draw(k, n, r, agents, rows, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 * seed + k + n + rows)
    t = lambda *s, std=1.0: (torch.randn(s, device="cuda", generator=g) * std).to(torch.bfloat16)  # noqa: E731
    return (t(rows, k), t(k, n, std=0.02), t(agents, k, r, std=k ** -0.5) if r else None, t(agents, r, n, std=0.05) if r else None)


def _quantised(w):
    """The definition of the packed 8-bit weights, in 64 bits."""
    top = w.double().abs().amax(0)
    s = torch.ones_like(top)
    on = top > 0
    s[on] = torch.exp2(torch.ceil(torch.log2(top[on] / 448)))
    return (w.double() / s).to(E4M3), s


def _reference(x, w, A, B, ids, scale, e4m3=False):
    """Y in 64 bits, and the bound on what the kernels may be off: x, w in double.  In 8 bits A is the sum of two e4m3 values, off by at most
    2^-17 of the coordinate's largest."""
    k = x.shape[1]
    y = x @ w
    # sums of K products in fp32, at most 2^-23 of the magnitudes a step (tensor cores may truncate); T: one rounding to bf16 (2^-8)
    off = k * 2.0**-23 * (x.abs() @ w.abs())
    if A is not None and ids is not None:
        for a in range(A.shape[0]):
            rows = (ids == a).nonzero()[:, 0]
            if rows.numel():
                Aa, Ba = A[a].double(), B[a].double()
                t = x[rows] @ Aa
                y[rows] += scale * t @ Ba
                a_off = 2.0**-17 * Aa.abs().amax(0) * x[rows].abs().sum(1, keepdim=True) if e4m3 else 0
                off[rows] += abs(scale) * ((2.0**-8 * t.abs() + (k + 64) * 2.0**-23 * (x[rows].abs() @ Aa.abs()) + a_off) @ Ba.abs())
    return y, off + 2.0**-8 * y.abs() + 1e-30


def _run(px, rows, k, n, r, agents, mix, e4m3, scale=1.5, seed=0, ids=None, check=True):
    x, w, A, B = _draw(k, n, r, agents, rows, seed)
    ids = _ids(rows, agents, mix, seed) if ids is None else ids
    wt = px.adapted_weights(w, A, B, scale, e4m3=e4m3)
    ws = px.adapted_workspace(wt, rows)
    if ws is not None:
        ws.fill_(255)                       # NaN as bf16: whatever the scratch holds must not matter
    out = torch.full((rows + 3, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    if e4m3:
        xs = x.float().abs().amax(1) / 448
        xq = (x.float() / xs[:, None]).to(E4M3)
        px.adapted_project_e4m3(wt, xq, xs, out[:rows], ids, ws)
        wq, s = _quantised(w)
        xd, wd = xq.double() * xs.double()[:, None], wq.double() * s
    else:
        px.adapted_project(wt, x, out[:rows], ids, ws)
        xd, wd = x.double(), w.double()
    assert torch.isnan(out[rows:]).all()    # rows behind the last one stay
    y, bound = _reference(xd, wd, A, B, ids, scale, e4m3)
    if check:
        err = (out[:rows].double() - y).abs()
        assert torch.isfinite(out[:rows]).all()
        assert (err <= bound).all(), f"{(err > bound).sum().item()} of {err.numel()} off, by up to {(err / bound).max().item():.3g} bounds"
        # all errors together: the roundings of Y and T, both below 2^-8 of what they round
        low = (y - xd @ wd).norm()
        assert err.norm() <= 2.0**-8 * (y.norm() + 2 * low) + 1e-30
    return out[:rows], y, bound


SIZES = [(1, 64, 8), (1, 2048, 2048), (2, 128, 24), (7, 1024, 1000), (16, 3584, 3584), (17, 256, 136), (40, 4096, 2304), (64, 512, 64), (65, 1024, 520),
         (127, 192, 264), (128, 256, 256), (129, 2048, 128), (200, 3584, 1280), (256, 1024, 1024), (257, 640, 200), (333, 1024, 1000),
         (511, 128, 2048), (700, 4096, 512), (1500, 256, 4096), (3001, 320, 328), (9000, 128, 136)]


@pytest.mark.parametrize("rank", [0, 8, 16, 32, 64])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_bf16_matches_the_definition(px, rows, k, n, rank):
    _run(px, rows, k, n, rank, 5, "rows", False, seed=rank)


@pytest.mark.parametrize("rank", [0, 8, 16, 32, 64])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_8_bits_match_the_definition(px, rows, k, n, rank):
    _run(px, rows, max(128, k // 128 * 128), n, rank, 5, "rows", True, seed=rank)


def _far(px, rows, k, n, r, e4m3, tail_rows, tail_cols):
    """A call whose last rows and columns lie past 2^31 elements; everything but those is zero.  Only the corner is compared."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + k + n)
    t = lambda *s, std=1.0: (torch.randn(s, device="cuda", generator=g) * std).to(torch.bfloat16)  # noqa: E731
    x = torch.zeros((rows, k), dtype=torch.bfloat16, device="cuda")
    x[-tail_rows:] = t(tail_rows, k)
    w = torch.zeros((k, n), dtype=torch.bfloat16, device="cuda")
    w[:, -tail_cols:] = t(k, tail_cols, std=0.02)
    A, B = t(2, k, r, std=k ** -0.5), t(2, r, n, std=0.05)
    wt = px.adapted_weights(w, A, B, 1.5, e4m3=e4m3)
    ids = (torch.arange(rows, device="cuda") % 3 - 1).to(torch.int32)
    out = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    ws = px.adapted_workspace(wt, rows)
    xt, wc = x[-tail_rows:], w[:, -tail_cols:].contiguous()
    if e4m3:
        xs = torch.ones(rows, device="cuda")
        xq = torch.zeros((rows, k), dtype=E4M3, device="cuda")
        xq[-tail_rows:] = xt.to(E4M3)
        px.adapted_project_e4m3(wt, xq, xs, out, ids, ws)
        wq, s = _quantised(wc)
        xd, wd = xq[-tail_rows:].double(), wq.double() * s
    else:
        px.adapted_project(wt, x, out, ids, ws)
        xd, wd = xt.double(), wc.double()
    y, bound = _reference(xd, wd, A, B[:, :, -tail_cols:], ids[-tail_rows:], 1.5, e4m3)
    assert ((out[-tail_rows:, -tail_cols:].double() - y).abs() <= bound).all()
    assert (out[0, :-tail_cols] == 0).all()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows,k,n", [(270001, 128, 8192), (65601, 32768, 136)])
def test_rows_past_32_bits(px, rows, k, n, e4m3):
    _far(px, rows, k, n, 16, e4m3, 300, 64)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows", [4, 16, 100, 1000])
def test_weights_past_32_bits(px, rows, e4m3):
    _far(px, rows, 262144, 9472, 16, e4m3, min(rows, 50), 64)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("mix", ["none", "neutral", "one", "runs", "rows"])
@pytest.mark.parametrize("rows", [1, 5, 31, 96, 300, 2200])
def test_agents(px, rows, mix, e4m3):
    _run(px, rows, 384, 272, 16, 7, mix, e4m3)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rank", [8, 64])
@pytest.mark.parametrize("rows", [3, 61, 256, 900, 2500, 40000])
def test_64_agents(px, rows, rank, e4m3):
    _run(px, rows, 512, 328, rank, 64, "rows", e4m3)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rank", [0, 8, 16, 32, 64])
@pytest.mark.parametrize("rows,k,n", [(1, 128, 40), (16, 1024, 520), (17, 256, 136), (64, 512, 64), (129, 2048, 128), (300, 384, 1000), (1500, 256, 264), (4097, 640, 72)])
def test_every_kernel_takes_every_size(forced, rows, k, n, rank, e4m3):
    _run(forced, rows, k, n, rank, 5, "rows", e4m3, seed=rank)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rank", [8, 64])
@pytest.mark.parametrize("rows", [3, 100, 700])
def test_every_kernel_takes_64_agents(forced, rows, rank, e4m3):
    _run(forced, rows, 512, 328, rank, 64, "rows", e4m3)


@pytest.mark.parametrize("rows", [4, 50, 200, 1000])
def test_the_largest_width_and_depth(px, rows):
    _run(px, rows, 14336, 4096, 32, 3, "rows", False)
    _run(px, rows, 4096, 14336, 32, 3, "runs", True)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows", [1, 6, 24, 70, 150, 400, 1300, 2600])
def test_other_adapters_and_rows_do_not_reach_a_row(px, rows, e4m3):
    _isolation(px, rows, e4m3)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows", [6, 70, 400])
def test_no_kernel_lets_other_adapters_reach_a_row(forced, rows, e4m3):
    _isolation(forced, rows, e4m3)


def _isolation(px, rows, e4m3):
    """Bit for bit the same whatever the other agents' adapters and the other rows hold, infinities and NaN among them."""
    k, n, r, agents = 512, 264, 16, 6
    x, w, A, B = _draw(k, n, r, agents, rows, seed=3)
    ids = _ids(rows, agents, "rows", seed=3)
    mine = ids == 2
    mine[0], ids[0] = True, 2
    xs = x.float().abs().amax(1) / 448
    xq = (x.float() / xs[:, None]).to(E4M3)

    def run(A, B, xq, xs, x):
        wt = px.adapted_weights(w, A, B, 2.0, e4m3=e4m3)
        out, ws = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda"), px.adapted_workspace(wt, rows)
        if e4m3:
            px.adapted_project_e4m3(wt, xq, xs, out, ids, ws)
        else:
            px.adapted_project(wt, x, out, ids, ws)
        return out

    want = run(A, B, xq, xs, x)
    A2, B2 = A.clone(), B.clone()
    others = [a for a in range(agents) if a != 2]
    A2[others], B2[others] = float("nan"), float("inf")
    x2, xq2, xs2 = x.clone(), xq.clone(), xs.clone()
    x2[~mine], xs2[~mine] = float("nan"), float("inf")
    xq2.view(torch.uint8)[~mine] = 0x7f                  # NaN
    got = run(A2, B2, xq2, xs2, x2)
    assert torch.isfinite(got[mine]).all() and torch.equal(got[mine], want[mine])
    # a row's own NaN does reach it
    x3, xs3 = x.clone(), xs.clone()
    x3[0, 5], xs3[0] = float("nan"), float("nan")
    got = run(A, B, xq, xs3, x3)
    assert torch.isnan(got[0]).all() and torch.equal(got[1:], want[1:])
    B3 = B.clone()
    B3[2, 1] = float("inf")
    got = run(A, B3, xq, xs, x)
    assert not torch.isfinite(got[0]).any() and torch.equal(got[~mine], want[~mine])


@pytest.mark.parametrize("rows", [2, 30, 100, 600, 2300])
def test_bad_agent_ids_are_reported_and_skipped(px, rows):
    ids = _ids(rows, 4, "rows")
    good = ids.clone()
    ids[0], good[0] = 4, -1
    ids[1], good[1] = -2, -1
    if rows > 2:
        ids[2], good[2] = 2**31 - 1, -1
        ids[3], good[3] = -2**31, -1
    got = _run(px, rows, 256, 136, 8, 4, "rows", False, ids=ids)[0]
    with pytest.raises(PreccError, match="bad-index"):
        px._check(px.lib.precc_poll_status(px.h, torch.cuda.current_stream().cuda_stream, None), "status")
    want = _run(px, rows, 256, 136, 8, 4, "rows", False, ids=good)[0]
    assert torch.equal(got, want)


@pytest.mark.parametrize("k,n", [(128, 8), (256, 33), (384, 100), (4096, 1000)])
def test_packed_8_bit_weights(px, k, n):
    """Bit for bit the quantisation of the definition, maxima on both sides of a power of two among them."""
    w = I.normal_bf16((k, n), 0.02, 1, "adapted.pack").cuda()
    w[:, 0] = 0
    w[0, 1], w[1:, 1] = 448 * 2.0**-9, 0.001                # exactly 448 * 2^s: the scale is that power of two
    w[0, 2], w[1:, 2] = 450 * 2.0**-9, 0.001                # the next bf16 above it
    w[0, 3], w[1:, 3] = 1e-37, 0                            # below the least scale
    w[0, 4], w[1:, 4] = 3e38, 1.0
    packed, scale = torch.empty((k // 128, n, 128), dtype=E4M3, device="cuda"), torch.empty(n, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    px._check(px.lib.precc_pack_kmajor_e4m3(px.h, w.data_ptr(), k, n, packed.data_ptr(), scale.data_ptr(), st), "pack")
    q, s = _quantised(w)
    s[3] = 2.0**-100
    q[:, 3] = (w[:, 3].double() / s[3]).to(E4M3)
    assert torch.equal(scale.double(), s)
    assert torch.equal(packed.permute(0, 2, 1).reshape(k, n).view(torch.uint8), q.view(torch.uint8))
    B = I.normal_bf16((6, n), 0.05, 2, "adapted.packB").cuda()
    dst = torch.empty_like(B)
    px._check(px.lib.precc_pack_expand_e4m3(px.h, B.data_ptr(), 6, n, scale.data_ptr(), dst.data_ptr(), st), "pack")
    keep = [i for i in range(n) if i not in (3, 4)]          # (B / 2^-100 and B / 2^120 leave bf16's range)
    assert torch.equal(dst.double()[:, keep], (B.double() / s)[:, keep])


@pytest.mark.parametrize("k,r", [(128, 8), (384, 64), (4096, 16)])
def test_packed_8_bit_adapters(px, k, r):
    """Value and rest sum up to A: exactly down to 2^-9 of a coordinate's largest value, within 2^-17 of that below."""
    A = (I.normal_bf16((3, k, r), 1.0, 1, "adapted.packA").double() * torch.exp2(torch.randint(-24, 1, (3, k, r), generator=torch.Generator().manual_seed(3)))).to(torch.bfloat16).cuda()
    A[1, :, 0] = 0
    wt = px.adapted_weights(torch.zeros((k, 8), dtype=torch.bfloat16, device="cuda"), A, torch.zeros((3, r, 8), dtype=torch.bfloat16, device="cuda"), 1.0, e4m3=True)
    parts = wt.A.view(k // 128, 2, 3, r, 128).double().permute(1, 2, 0, 4, 3).reshape(2, 3, k, r)
    got = parts.sum(0) * wt.a_scale.double().view(3, 1, r)
    top = A.double().abs().amax(1, keepdim=True)
    s = torch.where(top > 0, torch.exp2(torch.ceil(torch.log2(top / 448))), torch.ones_like(top))
    assert torch.equal(wt.a_scale.double().view(3, 1, r), s)
    err = (got - A.double()).abs()
    assert (err <= 2.0**-17 * top).all() and (err[A.double().abs() >= 2.0**-9 * top] == 0).all()


@pytest.mark.parametrize("rows", [1, 9, 64, 300, 1100])
def test_the_same_call_gives_the_same_bits(px, rows):
    a = _run(px, rows, 1024, 520, 32, 4, "rows", False, seed=8)[0]
    b = _run(px, rows, 1024, 520, 32, 4, "rows", False, seed=8)[0]
    assert torch.equal(a, b)


@pytest.mark.parametrize("rows", [1, 8, 48, 300, 1100])
def test_back_to_back_calls_on_one_workspace(px, rows):
    """A chain in which every call reads what the one before it wrote, through one scratch."""
    k = 512
    x, w, A, B = _draw(k, k, 16, 3, rows, seed=4)
    w = (w.float() * (50 / math.sqrt(k))).to(torch.bfloat16)
    ids = _ids(rows, 3, "rows")
    wt = px.adapted_weights(w, A, B, 1.0)
    ws = px.adapted_workspace(wt, rows)
    buf = [x.clone()] + [torch.empty_like(x) for _ in range(8)]
    torch.cuda.synchronize()
    for i in range(8):
        px.adapted_project(wt, buf[i], buf[i + 1], ids, ws)
    torch.cuda.synchronize()
    for i in range(8):
        out = torch.empty_like(x)
        px.adapted_project(wt, buf[i], out, ids, ws)
        torch.cuda.synchronize()
        assert torch.equal(out, buf[i + 1]), i


@pytest.mark.parametrize("rows", [1, 12, 64, 300])
def test_captured_replayed_and_on_another_stream(px, rows):
    x, w, A, B = _draw(1024, 264, 16, 3, rows, seed=5)
    ids = _ids(rows, 3, "rows")
    wt = px.adapted_weights(w, A, B, 1.0)
    ws = [px.adapted_workspace(wt, rows) for _ in range(2)]
    out = [torch.empty((rows, 264), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    px.adapted_project(wt, x, out[0], ids, ws[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.mul_(2)
        px.adapted_project(wt, x, out[1], ids, ws[1])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[1].float(), out[0].float() * 2)          # a power of two passes through every rounding
    ids.fill_(1)
    B[1] = 0                                                        # bf16 takes B where it lies
    graph.replay()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        px.adapted_project(wt, x, out[0], None, None)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(out[1], out[0])


def test_two_streams_at_once(px):
    """Calls of two streams, each with its own scratch, overlapping as they like."""
    cases = []
    for i, rows in enumerate((700, 40)):
        x, w, A, B = _draw(1024, 1024, 32, 4, rows, seed=20 + i)
        ids = _ids(rows, 4, "rows", seed=i)
        wt = px.adapted_weights(w, A, B, 1.0)
        out = torch.empty((rows, 1024), dtype=torch.bfloat16, device="cuda")
        px.adapted_project(wt, x, out, ids, px.adapted_workspace(wt, rows))
        cases.append((x, wt, ids, out, px.adapted_workspace(wt, rows), [torch.empty_like(out) for _ in range(20)], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for i in range(20):
        for x, wt, ids, _, ws, outs, stream in cases:
            with torch.cuda.stream(stream):
                px.adapted_project(wt, x, outs[i], ids, ws)
    torch.cuda.synchronize()
    for _, _, _, want, _, outs, _ in cases:
        assert all(torch.equal(o, want) for o in outs)


def test_refusals(px):
    x, w, A, B = _draw(256, 64, 8, 2, 4)
    wt = px.adapted_weights(w, A, B, 1.0)
    w8 = px.adapted_weights(w, A, B, 1.0, e4m3=True)
    ids, ws = _ids(4, 2, "rows"), px.adapted_workspace(wt, 4)
    out = torch.full((4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    xq, xs = x.to(E4M3), torch.ones(4, device="cuda")

    def refused(match, call, *a):
        with pytest.raises(PreccError, match=match):
            call(*a)

    p, p8 = px.adapted_project, px.adapted_project_e4m3
    refused("columns", p, wt, x[:, :128].contiguous(), out, ids, ws)
    refused("elements", p, wt, x, out[:3], ids, ws)
    refused("elements", p, wt, x, out, ids[:3], ws)
    refused("must be", p, wt, x, out, ids.long(), ws)
    refused("must be", p, wt, x.half(), out, ids, ws)
    refused("must be", p, wt, x, out.float(), ids, ws)
    refused("must be", p, w8, x, out, ids, ws)
    refused("must be", p8, wt, xq, xs, out, ids, ws)
    refused("x_scale is None", p8, w8, xq, None, out, ids, ws)
    refused("elements", p8, w8, xq, xs[:2], out, ids, ws)
    refused("workspace: need", p, wt, x, out, ids, None)
    refused("workspace: need", p, wt, x, out, ids, ws[:-1])
    big = torch.empty(ws.numel() + 64, dtype=torch.uint8, device="cuda")
    refused("128-byte aligned", p, wt, x, out, ids, big[16:16 + ws.numel()])
    refused("contiguous", p, wt, x.t().contiguous().t(), out, ids, ws)
    flat = torch.empty(4 * 256 + 4, dtype=torch.bfloat16, device="cuda")
    refused("16-byte aligned", p, wt, flat[1:1025].view(4, 256), out, ids, ws)
    refused("out is None", p, wt, x, None, ids, ws)

    def with_desc(k, n, agents, r):
        mk = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        return AdaptedWeights(ProjectionDesc(k, n, agents, r, 1.0), mk(n, k), None, mk(agents * r, k), mk(agents, r, n))

    def shape(match, k, n, agents, r):
        refused(match, p, with_desc(k, n, agents, r), torch.zeros((4, k), dtype=torch.bfloat16, device="cuda"),
                torch.empty((4, n), dtype=torch.bfloat16, device="cuda"), ids, big)

    shape("k_dim", 96, 64, 2, 8)
    shape("n_out", 64, 60, 2, 8)
    shape("rank", 64, 64, 2, 24)
    shape("rank", 64, 64, 2, 128)
    shape("n_agents", 64, 64, 65, 8)
    refused("come together", px.adapted_weights, w, A, None, 1.0)
    refused("A must be", px.adapted_weights, w, A[:, :128].contiguous(), B, 1.0)
    refused("W must be", px.adapted_weights, w.float(), A, B, 1.0)
    refused("k_dim", px.adapted_weights, w[:192].contiguous(), None, None, 1.0, True)
    p(wt, x[:0], out[:0], ids[:0], ws)
    torch.cuda.synchronize()
    assert (out == 7).all()
