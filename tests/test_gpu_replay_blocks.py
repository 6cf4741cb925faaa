"""The trace replay through attention blocks: the streams and caches that it leaves against a 64-bit replay, for every sharing policy, and
that nothing in its timed regions waits for the device."""
import numpy as np
import pytest
import torch

from block_oracle import BF16_OFF, E4M3_OFF, GEO, LAYERS, TURNS, Oracle, grown, off
from harness import base_rows, f64, lr_rows

from paper_2609_34054_b200 import inputs as I
from paper_2609_34054_b200 import replay as R
from paper_2609_34054_b200.binding import Precc

pytestmark = pytest.mark.gpu
TOTAL = R.trace_tokens(TURNS)


@pytest.fixture(scope="module")
def px():
    p = Precc(0)
    yield p
    torch.cuda.synchronize()
    assert p.poll_status() == 0
    p.close()


def _stack(px, block):
    return R.Stack(px, GEO, n_layers=LAYERS, max_tokens=TOTAL + I.PAGE, max_rows=2 * TOTAL, private_tokens=220, block=block)


@pytest.mark.parametrize("block", ["bf16", "e4m3"])
@pytest.mark.parametrize("policy", R.POLICIES)
def test_streams_and_caches_of_a_replay(px, monkeypatch, policy, block):
    want, rows = Oracle().replay(TURNS, policy)
    monkeypatch.setattr(I, "layer_weights", grown(I.layer_weights))
    monkeypatch.setattr(I, "block_weights", grown(I.block_weights))
    st = _stack(px, block)
    R.replay(st, TURNS, policy)
    torch.cuda.synchronize()
    tol = BF16_OFF if block == "bf16" else E4M3_OFF
    got = f64(st.blocks.r[:want.shape[0]])
    for i in ([0, 1] if policy == "rebase_db" else [slice(None)]):            # the adapted and the adapter-free token, each by itself
        assert off(got[i], want[i]) <= tol, (i, off(got[i], want[i]))
    for l, c in enumerate(st.caches):
        # (the first layer's rows come from inputs that 8-bit blocks hold in bf16 too)
        tol_l = tol if l else BF16_OFF
        pairs = [("k", base_rows(c.k_base)[:TOTAL], rows.k[l]), ("v", base_rows(c.v_base)[:TOTAL], rows.v[l])]
        for a in range(GEO.n_agents):
            pairs += [(f"lr_k {a}", lr_rows(c.lr_k, a)[:TOTAL], rows.lr_k[l, a]), (f"lr_v {a}", lr_rows(c.lr_v, a)[:TOTAL], rows.lr_v[l, a])]
        for name, g, w in pairs:
            w = w[:TOTAL]
            if not w.any():                              # rows that the policy never writes
                assert not g.any(), (name, l)
                continue
            at = np.cumsum([0] + [t.n_in + t.n_out for t in TURNS])
            for t, a, b in zip(TURNS, at, at[1:]):       # turn by turn: another one's rows do not hide it
                assert off(g[a:b], w[a:b]) <= tol_l, (name, l, t, off(g[a:b], w[a:b]))


@pytest.mark.parametrize("block", ["", "bf16", "e4m3"])
@pytest.mark.parametrize("policy", R.POLICIES)
def test_nothing_waits_in_a_timed_region(px, monkeypatch, policy, block):
    """Ids, masks and tables are on the device before a clock starts: a copy from pageable host memory would wait there for what the region times."""
    timed = R._timed

    def watched(fn):
        def run():
            torch.cuda.set_sync_debug_mode("error")
            try:
                fn()
            finally:
                torch.cuda.set_sync_debug_mode("default")
        return timed(run)
    monkeypatch.setattr(R, "_timed", watched)
    r = R.replay(_stack(px, block), TURNS, policy)
    assert r["ttft_ms"] > 0 and r["tokens"] == TOTAL
