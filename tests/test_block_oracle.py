"""The 64-bit replay through attention blocks tells wrong routing apart from rounding (no GPU: the mistakes are planted in the oracle)."""
import numpy as np
import pytest

from block_oracle import BF16_OFF, E4M3_OFF, GEO, TURNS, Oracle, off, own_rows
from paper_2609_34054_b200 import replay as R


def _replay(policy, plant=lambda o: None):
    o = Oracle()
    plant(o)
    return o.replay(TURNS, policy)


def _other_agent(name):
    def plant(o):
        for w in o.w:
            for m in ("A_", "B_"):
                w[m + name] = np.roll(w[m + name], 1, 0)
    return plant


def _swapped(o):
    o.adapted, o.neutral = o.neutral, o.adapted


@pytest.mark.parametrize("policy", R.POLICIES)
def test_swapped_sequences_show(policy):
    (last, rows), (wrong, wrong_rows) = _replay(policy), _replay(policy, _swapped)
    assert off(wrong, last) > 3 * E4M3_OFF and off(wrong_rows.k[1], rows.k[1]) > 3 * E4M3_OFF


@pytest.mark.parametrize("name", ["q", "o"])
@pytest.mark.parametrize("policy", ["prelr", "rebase_db", "rebase_lp"])
def test_another_agents_query_or_output_adapter_shows(policy, name):
    (last, rows), (wrong, wrong_rows) = _replay(policy), _replay(policy, _other_agent(name))
    if policy == "rebase_lp":                            # its last pass is adapter-free: the adapted one left its low-rank rows
        last, wrong = (own_rows(r.lr_k[1]) for r in (rows, wrong_rows))
    assert off(wrong, last) > 6 * BF16_OFF and off(wrong, last) > 1.5 * E4M3_OFF


def test_policies_without_agents_have_none():
    for policy in ("fullshared", "nonshared"):
        assert off(_replay(policy, _other_agent("q"))[0], _replay(policy)[0]) == 0
    assert GEO.n_agents == 3
