"""Attention blocks: norm, query projection, cached attention and output projection as they run together, against the definition in 64 bits,
and the trace replay through them."""
import numpy as np
import pytest
import torch

from harness import assert_close, f64

from paper_2609_34054_b200 import inputs as I
from paper_2609_34054_b200 import replay as R
from paper_2609_34054_b200.binding import Cache, Precc, layer_desc
from paper_2609_34054_b200.block import EPS, AttentionBlocks

pytestmark = pytest.mark.gpu
GEO = I.Geometry(d_model=256, n_q=4, n_kv=2, hd=64, n_agents=3, rank_k=16, rank_v=16, alpha=32.0)


@pytest.fixture(scope="module")
def px():
    p = Precc(0)
    yield p
    torch.cuda.synchronize()
    assert p.poll_status() == 0
    p.close()


def _layers(px, geo, n_layers, n_blocks):
    desc, out = layer_desc(geo), []
    for l in range(n_layers):
        w = {k: v.cuda() for k, v in I.layer_weights(geo, 0, f"L{l}").items()}
        out.append((w, px.pack_turn_weights(geo, w["W_k"], w["W_v"], w["A_k"], w["A_v"]), Cache(geo, n_blocks, fill=0.0)))
    return desc, out


def _norm64(r, gain):
    return r / np.sqrt((r * r).mean(-1, keepdims=True) + EPS) * gain


def _reference(geo, x, agent, n_layers):
    """The residual stream after n_layers blocks of one sequence of `agent` (None: adapter-free), float64."""
    r = f64(x)
    n, s = r.shape[0], geo.scale(geo.rank_v)
    causal = np.tril(np.ones((n, n), bool))
    for l in range(n_layers):
        w = {k: f64(v) for k, v in {**I.layer_weights(geo, 0, f"L{l}"), **I.block_weights(geo, 0, f"L{l}")}.items()}

        def adapted(a, name, scale):
            return a @ w["W_" + name] + (scale * (a @ w["A_" + name][agent]) @ w["B_" + name][agent] if agent is not None else 0)
        h = _norm64(r, w["gain"])
        q = adapted(h, "q", s).reshape(n, geo.n_q, geo.hd)
        k, v = (adapted(h, name, sc).reshape(n, geo.n_kv, geo.hd) for name, sc in (("k", geo.scale_k), ("v", geo.scale_v)))
        o = np.empty_like(q)
        for i in range(geo.n_q):
            z = q[:, i] @ k[:, i // geo.group].T / np.sqrt(geo.hd)
            z = np.where(causal, z, -np.inf)
            p = np.exp(z - z.max(1, keepdims=True))
            o[:, i] = p / p.sum(1, keepdims=True) @ v[:, i // geo.group]
        r = r + adapted(o.reshape(n, -1), "o", s)
    return r


@pytest.mark.parametrize("agent", [1, -1])
@pytest.mark.parametrize("n", [1, 37, 200])
def test_a_turn_and_a_decode_step_through_two_blocks(px, n, agent):
    """n tokens as a turn, and once more with the last one as a decode step, against the whole block in 64 bits."""
    layers = 2
    desc, lw = _layers(px, GEO, layers, (n + 15) // 16)
    blocks = AttentionBlocks(px, GEO, layers, max(n, 2))
    x = I.normal_bf16((n, GEO.d_model), 1.0, 5, "block.x").cuda()
    ws = px.decode_workspace(desc, 1, n)
    ids = torch.full((n,), agent, dtype=torch.int32, device="cuda")
    one = torch.tensor([n], dtype=torch.int32, device="cuda")

    def turn(rows):
        def attend(l, h, q, out):
            w, wa, cache = lw[l]
            px.turn_project(desc, h, wa, cache, 0)
            px.lr_attend_prefill(desc, q, agent, 0, w["B_k"], w["B_v"], cache, out)
        return blocks.forward(x[:rows], ids[:rows], attend).clone()

    want = _reference(GEO, x, None if agent < 0 else agent, layers)
    got = turn(n)
    # bf16 roundings of h, q, the caches, the attention's output and y in each of two layers, of a stream that is itself rounded each time
    assert_close(f64(got), want, f"turn of {n}", atol=2e-2, rtol=2e-2, norm_tol=2e-2)
    if n > 1:
        turn(n - 1)

        def attend(l, h, q, out):
            w, wa, cache = lw[l]
            px.turn_project(desc, h, wa, cache, n - 1)
            px.lr_attend_decode(desc, q, ids[:1], one, n, w["B_k"], w["B_v"], cache, out, ws)
        last = blocks.forward(x[n - 1:], ids[:1], attend)
        assert_close(f64(last), want[n - 1:], f"decode behind {n - 1}", atol=2e-2, rtol=2e-2, norm_tol=2e-2)


def test_8_bit_blocks_step_by_step(px):
    """Every step of an 8-bit block against the definition from what it was given: the quantised hidden states go into the query projection,
    the bf16 ones into the caches."""
    n = 150
    blocks = AttentionBlocks(px, GEO, 2, n, e4m3=True)
    x = I.normal_bf16((n, GEO.d_model), 1.0, 6, "block.x8").cuda()
    ids = I.uniform_int(-1, GEO.n_agents - 1, n, 6, "block.ids").cuda()
    seen = []

    def attend(l, h, q, out):
        out.copy_(I.normal_bf16(tuple(out.shape), 1.0, l, "block.o").cuda())
        seen.append((h.clone(), blocks.h8[:n].clone(), blocks.h_scale[:n].clone(), q.reshape(n, -1).clone(), out.reshape(n, -1).clone(), blocks.r[:n].clone()))

    final = blocks.forward(x, ids, attend)
    s = GEO.scale(GEO.rank_v)
    r = x.double()
    for l, (h, h8, hs, q, o, r_now) in enumerate(seen):
        w = {k: v.cuda().double() for k, v in I.block_weights(GEO, 0, f"L{l}").items()}
        assert ((r_now.double() - r).abs() <= off(r)).all() if l else torch.equal(r_now.double(), r)
        r = r_now.double()
        want_h = r / (r.square().mean(-1, keepdim=True) + EPS).sqrt() * w["gain"]
        assert ((h.double() - want_h).abs() <= (2.0**-8 + (2.0**-7 if l else 1e-5)) * want_h.abs() + (0.02 if l else 0)).all()
        x8 = h8.double() * hs.double()[:, None]
        assert ((x8 - want_h).norm() <= 2.0**-4 * want_h.norm())
        top = w["W_q"].abs().amax(0)
        step = torch.exp2(torch.ceil(torch.log2(top / 448)))
        wq = (w["W_q"] / step).to(torch.float8_e4m3fn).double() * step

        def adapted(a, W, A, B):
            y = a @ W
            for g in range(GEO.n_agents):
                rows = ids == g
                y[rows] += s * (a[rows] @ A[g]) @ B[g]
            return y
        want_q = adapted(x8, wq, w["A_q"], w["B_q"])
        assert ((q.double() - want_q).norm(dim=1) <= 2 * 2.0**-8 * want_q.norm(dim=1)).all()
        o = o.double()
        y = adapted(o, w["W_o"], w["A_o"], w["B_o"])
        r = r + y
        # y: its own rounding, s (o A) rounded to bf16 before it meets B, and 32-bit sums of K products; then the rounding of the stream
        low = torch.zeros_like(y)
        for g in range(GEO.n_agents):
            low[ids == g] = s * (o[ids == g] @ w["A_o"][g]).abs() @ w["B_o"][g].abs()
        y_off = 2.0**-8 * (y.abs() + 1.01 * low) + o.shape[1] * 2.0**-23 * (o.abs() @ w["W_o"].abs())
        off = lambda r, y_off=y_off: 2.0**-8 * r.abs() + 1.01 * y_off
    assert ((final.double() - r).abs() <= off(r)).all()


@pytest.mark.parametrize("block", ["bf16", "e4m3"])
@pytest.mark.parametrize("policy", R.POLICIES)
def test_replay_through_blocks(px, policy, block):
    turns = [R.Turn(0, 70, 5), R.Turn(1, 120, 4), R.Turn(2, 33, 3)]
    total = R.trace_tokens(turns)
    st = R.Stack(px, GEO, n_layers=2, max_tokens=total + 16, max_rows=2 * total, private_tokens=220, block=block)
    r = R.replay(st, turns, policy)
    assert r["tokens"] == total and r["ttft_ms"] > 0 and r["decode_ms"] > 0
    torch.cuda.synchronize()
    rows = 2 if policy == "rebase_db" else 1
    first = st.blocks.r[:rows].clone()
    assert torch.isfinite(first.float()).all() and torch.isfinite(st.caches[1].k_base.float()).all()
    R.replay(st, turns, policy)                       # the same trace again: the same stream, bit for bit
    torch.cuda.synchronize()
    assert torch.equal(st.blocks.r[:rows], first)


def test_block_names():
    with pytest.raises(ValueError, match="block must be"):
        R.Stack.__init__(R.Stack.__new__(R.Stack), Precc(0), GEO, 1, 16, 16, block="fp4")
