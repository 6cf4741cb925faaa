"""The trace replay through attention blocks in 64 bits: what the residual streams and the shared caches hold after a trace, per sharing policy.

One sequence at a time, from the definitions: hidden states are the norm of the stream, base rows h W, low-rank rows h A_a of the agents that a pass
writes, queries and the output with the agent's adapters, attention over base + s LR_a B_a."""
import numpy as np

from harness import f64

from paper_2609_34054_b200 import inputs as I
from paper_2609_34054_b200.block import EPS
from paper_2609_34054_b200.inputs import block_weights, layer_weights
from paper_2609_34054_b200.replay import Turn, trace_tokens

GEO = I.Geometry(d_model=256, n_q=4, n_kv=2, hd=64, n_agents=3, rank_k=16, rank_v=16, alpha=32.0)
LAYERS = 2
TURNS = [Turn(0, 70, 5), Turn(1, 120, 4), Turn(2, 33, 3)]
# Weights large enough that a wrong agent, row or cache shows in the stream: scores of standard deviation 2 to 3, a block that adds as much as the stream
# holds.  (Both sides take them rounded to bf16.)
GROWN = {"W_q": 4, "B_q": 12, "W_k": 4, "B_k": 4, "W_v": 2, "B_v": 2, "W_o": 8, "B_o": 12}
# What roundings leave of a tensor's norm.  bf16: 2^-9 each on average (half a step is 2^-8 at most), of h, q, k, v, the low-rank rows and their products,
# the probabilities, o, y and the stream, those of q and k three times over as they pass through the scores: 14 in each of two layers, taken as if they added up.
# 8 bits: also the queries' two factors, each off by half a step, 2^-4, at most, on average over a step and a binade by 2^-4 / sqrt(3) * 0.71 = 0.026, independent of
# one another and from layer to layer (a root of two each), times the scores' factor 3.
BF16_OFF = 2 * 14 * 2.0**-9
E4M3_OFF = BF16_OFF + 2 * 3 * 0.026


def grown(fn):
    """layer_weights / block_weights with the factors above."""
    def weights(*a, **k):
        return {name: (t.float() * GROWN.get(name, 1)).to(t.dtype) for name, t in fn(*a, **k).items()}
    return weights


class Rows:
    """The rows of all layers' caches, by position: base keys and values, and the low-rank rows of every agent."""

    def __init__(self, geo, layers, tokens):
        self.k = np.zeros((layers, tokens, geo.n_kv * geo.hd))
        self.v = np.zeros((layers, tokens, geo.n_kv * geo.hd))
        self.lr_k = np.zeros((layers, geo.n_agents, tokens, geo.rank_k))
        self.lr_v = np.zeros((layers, geo.n_agents, tokens, geo.rank_v))

    def copy(self):
        c = Rows.__new__(Rows)
        c.k, c.v, c.lr_k, c.lr_v = (t.copy() for t in (self.k, self.v, self.lr_k, self.lr_v))
        return c


class Oracle:
    def __init__(self, geo=GEO, layers=LAYERS, tokens=trace_tokens(TURNS) + I.PAGE, seed=0):
        self.geo, self.layers = geo, layers
        weights = (grown(layer_weights), grown(block_weights))
        self.w = [{n: f64(t) for fn in weights for n, t in fn(geo, seed, f"L{l}").items()} for l in range(layers)]
        rows = (tokens + I.PAGE - 1) // I.PAGE * I.PAGE
        self.adapted, self.neutral = (f64(I.normal_bf16((rows, geo.d_model), 1.0, seed, f"replay.H_{n}")) for n in ("adpt", "neut"))
        self.tokens = tokens

    def step(self, rows, x, start, agent, writes):
        """Tokens x [n, d] at positions start.. of one sequence: writes base rows and the low-rank rows of the agents in `writes`, attends as
        `agent` (None: adapter-free), returns the stream."""
        geo, r, n = self.geo, x, x.shape[0]
        seen = slice(0, start + n)
        mask = np.arange(start + n)[None, :] > (start + np.arange(n))[:, None]
        for l, w in enumerate(self.w):
            def adapted(a, name, scale):
                y = a @ w["W_" + name]
                return y if agent is None else y + scale * (a @ w["A_" + name][agent]) @ w["B_" + name][agent]
            h = r / np.sqrt((r * r).mean(-1, keepdims=True) + EPS) * w["gain"]
            new = slice(start, start + n)
            rows.k[l, new], rows.v[l, new] = h @ w["W_k"], h @ w["W_v"]
            for a in writes:
                rows.lr_k[l, a, new], rows.lr_v[l, a, new] = h @ w["A_k"][a], h @ w["A_v"][a]
            k, v = rows.k[l, seen], rows.v[l, seen]
            if agent is not None:
                k = k + geo.scale_k * rows.lr_k[l, agent, seen] @ w["B_k"][agent]
                v = v + geo.scale_v * rows.lr_v[l, agent, seen] @ w["B_v"][agent]
            q = adapted(h, "q", geo.scale(geo.rank_v)).reshape(n, geo.n_q, geo.hd)
            k, v = k.reshape(-1, geo.n_kv, geo.hd), v.reshape(-1, geo.n_kv, geo.hd)
            o = np.empty_like(q)
            for i in range(geo.n_q):
                z = np.where(mask, -np.inf, q[:, i] @ k[:, i // geo.group].T / np.sqrt(geo.hd))
                p = np.exp(z - z.max(1, keepdims=True))
                o[:, i] = p / p.sum(1, keepdims=True) @ v[:, i // geo.group]
            r = r + adapted(o.reshape(n, -1), "o", geo.scale(geo.rank_v))
        return r

    def replay(self, turns, policy):
        """(stream of the last pass or decode step, shared rows)."""
        geo, rows, P, last = self.geo, Rows(self.geo, self.layers, self.tokens), 0, None
        everyone = range(geo.n_agents)
        covered = [0] * geo.n_agents
        for t in turns:
            j, end = t.agent, P + t.n_in + t.n_out
            others = [a for a in everyone if a != j]
            if policy == "rebase_db":
                own = rows.copy()                        # the adapted sequence: the shared context, then rows of its own
                for at, n in [(P, t.n_in)] + [(p, 1) for p in range(P + t.n_in, end)]:
                    last = np.concatenate([self.step(own, self.adapted[at:at + n], at, j, [j]), self.step(rows, self.neutral[at:at + n], at, None, others)])
                    rows.lr_k[:, j, at:at + n], rows.lr_v[:, j, at:at + n] = own.lr_k[:, j, at:at + n], own.lr_v[:, j, at:at + n]
            else:
                agent, writes = {"prelr": (j, everyone), "rebase_lp": (j, [j]), "fullshared": (None, []), "nonshared": (None, [])}[policy]
                start = covered[j] if policy == "nonshared" else P
                for at, n in [(start, P + t.n_in - start)] + [(p, 1) for p in range(P + t.n_in, end)]:
                    last = self.step(rows, self.adapted[at:at + n], at, agent, writes)
                if policy == "rebase_lp":
                    last = self.step(rows, self.neutral[P:end], P, None, others)
            P = end
            covered[j] = P
        return last, rows


def own_rows(lr, turns=TURNS):
    """Of low-rank rows [agents, tokens, r]: those of each turn's agent at the turn's tokens."""
    at = np.cumsum([0] + [t.n_in + t.n_out for t in turns])
    return np.concatenate([lr[t.agent, a:b] for t, a, b in zip(turns, at, at[1:])])


def off(got, want):
    """Distance of two arrays, relative to the second's norm."""
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))
