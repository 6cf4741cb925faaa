"""The trace replay through attention blocks: nothing in its timed regions waits for the device."""
import pytest
import torch

from paper_2609_34054_b200 import inputs as I
from paper_2609_34054_b200 import replay as R
from paper_2609_34054_b200.binding import Precc

pytestmark = pytest.mark.gpu
GEO = I.Geometry(d_model=256, n_q=4, n_kv=2, hd=64, n_agents=3, rank_k=16, rank_v=16, alpha=32.0)
LAYERS = 2
TURNS = [R.Turn(0, 70, 5), R.Turn(1, 120, 4), R.Turn(2, 33, 3)]
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
