"""The operators around the cached attention, as cases that can be timed and compared.

* ``norm``     root-mean-square norm of the hidden states with the residual's addition; bf16 output, 8-bit output (e4m3) with
               one scale per row, or both
* ``project``  the query / output projection of a batch whose rows belong to many agents: the shared weights, plus
               the low-rank adapter of each row's own agent; bf16, or 8-bit inputs and weights with scales

Layer shapes are those of the repository's workloads (d_model 1024 / 2048 / 3584 / 4096).  Everything is drawn on the device
from the seed.
"""
import math

import torch

own = False

EPS = 1e-5
E4M3_MAX = 448.0
LORA_SCALE = 2.0


def _norm(rows, width, residual, bf16, e4m3, **more):
    return dict(op="norm", rows=rows, width=width, residual=residual, bf16=bf16, e4m3=e4m3, **more)


def _project(rows, k, n, rank, agents, mix, e4m3, **more):
    return dict(op="project", rows=rows, k=k, n=n, rank=rank, agents=agents, mix=mix, e4m3=e4m3, **more)


def listed():
    return [
        # one decoded token of the 16-layer benchmark model: the smallest call, where only latency counts
        _norm(1, 2048, True, True, False, name="norm-decode-token"),
        # norm of every query head of a 64-request decode step (28 heads of 128 columns): many short rows
        _norm(64 * 28, 128, False, True, False, name="norm-query-heads"),
        # a ragged turn whose hidden states feed the bf16 cache projection and the 8-bit query projection
        _norm(1337, 3584, True, True, True, name="norm-turn-both-outputs"),
        # a whole 32k-token context on its way into 8-bit projections
        _norm(32768, 4096, True, False, True, name="norm-context-8bit"),
        # query projection of one decoded token
        _project(1, 2048, 2048, 16, 4, "one", False, name="project-decode-token"),
        # output projection of a serving step: 64 requests of 8 agents, some of them without an adapter
        _project(64, 3584, 3584, 16, 8, "rows", False, name="project-serving-step"),
        # eight requests in 8 bits, every one of another agent
        _project(8, 4096, 4096, 32, 8, "rows", True, name="project-decode-8bit"),
        # a step in which nearly every request has an adapter of its own: the adapters weigh as much as the shared weights
        _project(61, 4096, 4096, 64, 64, "rows", False, name="project-many-agents"),
        # a turn's new tokens, one agent
        _project(512, 4096, 4096, 32, 4, "one", False, name="project-turn"),
        # turns of several agents in one batch, odd sizes, onto a slice of the heads
        _project(777, 1024, 1000, 8, 3, "runs", True, name="project-ragged-8bit"),
        # chunks of eight requests' contexts in one batch
        _project(8192, 4096, 4096, 32, 8, "runs", False, name="project-context"),
        # the same, longer and in 8 bits
        _project(16384, 4096, 4096, 64, 8, "runs", True, name="project-context-8bit"),
    ]


def _spread(rng, low, high):
    """An integer of [low, high], uniform in its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    if rng.random() < 0.4:
        width = 8 * _spread(rng, 8, 512)
        rows = _spread(rng, 1, min(32768 * 4, 32768 * 4096 // width))
        outputs = rng.choice([(True, False), (False, True), (True, True)])
        return _norm(rows, width, rng.random() < 0.7, *outputs)
    e4m3 = rng.random() < 0.4
    k = 128 * rng.randint(1, 32) if e4m3 else 64 * rng.randint(1, 64)
    n = 8 * _spread(rng, 4, 512)
    rows = _spread(rng, 1, 8192)
    return _project(rows, k, n, rng.choice([0, 8, 16, 32, 64]), rng.randint(1, 16) if rng.random() < 0.8 else 64,
                    rng.choice(["one", "runs", "rows"]), e4m3)


def _segments(case):
    """Length of a run of rows that belong to one request, where the rows of a request follow one another."""
    return max(1, -(-case["rows"] // (case["agents"] + 1)))


def _agent_ids(case, g):
    """One agent per row; -1 is a request without an adapter."""
    rows, n = case["rows"], case["agents"]
    if case["mix"] == "one":
        return torch.randint(0, n, (1,), device="cuda", generator=g, dtype=torch.int32).expand(rows).contiguous()
    if case["mix"] == "runs":
        request = torch.arange(rows, device="cuda") // _segments(case)
        return ((torch.randperm(n + 1, device="cuda", generator=g) - 1)[request]).to(torch.int32)
    if rows <= n:
        return torch.randperm(n, device="cuda", generator=g)[:rows].to(torch.int32)
    return torch.randint(-1, n, (rows,), device="cuda", generator=g, dtype=torch.int32)


def _draw_inputs(case, seed):
    """The inputs alone, on the device, from the seed."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 11)

    def normal(shape, std=1.0):
        return torch.randn(shape, device="cuda", generator=g).mul_(std).to(torch.bfloat16)

    if case["op"] == "norm":
        shape = (case["rows"], case["width"])
        # hidden states grow with depth, and a few coordinates of every row are far larger than the rest
        x = normal(shape, 3.0)
        x[:, :: 61] *= 8
        return {"x": x, "residual": normal(shape, 4.0) if case["residual"] else None,
                "gain": (1 + 0.2 * torch.randn(case["width"], device="cuda", generator=g)).to(torch.bfloat16)}
    rows, k, n, r, agents = (case[f] for f in ("rows", "k", "n", "rank", "agents"))
    s = {"x": normal((rows, k)), "w": normal((k, n), 0.02), "agent_id": _agent_ids(case, g),
         "a": normal((agents, k, r), k ** -0.5) if r else None, "b": normal((agents, r, n), 0.02) if r else None}
    if case["e4m3"]:
        x = s["x"].float()
        s["x_scale"] = x.abs().amax(1) / E4M3_MAX
        s["x"] = (x / s["x_scale"][:, None]).to(torch.float8_e4m3fn)
    return s


def _quantised_weights(w):
    """Weights in 8 bits: one power of two per output column, so that the largest value of the column fits."""
    top = w.abs().amax(0)
    scale = torch.where(top > 0, torch.exp2(torch.ceil(torch.log2(top.double() / E4M3_MAX))), 1.0).to(torch.float32)
    return (w / scale).to(torch.float8_e4m3fn), scale


_px = None


def _context():
    """One library context for the process, as a program keeps it."""
    global _px
    if _px is None:
        from paper_2609_34054_b200.binding import Precc
        _px = Precc(0)
    return _px


def prepare(case, seed):
    s = _draw_inputs(case, seed)
    s["case"] = dict(case)
    if case["op"] == "norm":
        rows, width = case["rows"], case["width"]
        s["residual_out"] = torch.empty_like(s["x"]) if case["residual"] else None
        s["out"] = torch.empty_like(s["x"]) if case["bf16"] else None
        s["out_e4m3"] = torch.empty((rows, width), dtype=torch.float8_e4m3fn, device="cuda") if case["e4m3"] else None
        s["out_scale"] = torch.empty(rows, dtype=torch.float32, device="cuda") if case["e4m3"] else None
        if own:
            s["px"] = _context()
        return s
    s["out"] = torch.empty((case["rows"], case["n"]), dtype=torch.bfloat16, device="cuda")
    if own:
        s["px"] = px = _context()
        s["weights"] = px.adapted_weights(s["w"], s["a"], s["b"], LORA_SCALE, e4m3=case["e4m3"])
        s["workspace"] = px.adapted_workspace(s["weights"], case["rows"])
    elif case["e4m3"]:
        s["wq"], s["w_scale"] = _quantised_weights(s["w"].float())
    return s


def _run_norm(s):
    case = s["case"]
    if own:
        s["px"].rms_norm(s["x"], s["gain"], EPS, out=s["out"], residual=s["residual"], residual_out=s["residual_out"],
                         out_e4m3=s["out_e4m3"], out_scale=s["out_scale"])
        return {"residual": s["residual_out"], "out": s["out"], "q": s["out_e4m3"], "scale": s["out_scale"]}
    x = s["x"].float()
    if case["residual"]:
        x = x + s["residual"].float()
        s["residual_out"].copy_(x)
    y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * s["gain"].float()
    if case["bf16"]:
        s["out"].copy_(y)
    if case["e4m3"]:
        top = y.abs().amax(1)
        scale = torch.where(top == 0, 1.0, top / E4M3_MAX)
        s["out_scale"].copy_(scale)
        s["out_e4m3"].copy_((y / scale[:, None]).to(torch.float8_e4m3fn))
    return {"residual": s["residual_out"], "out": s["out"], "q": s["out_e4m3"], "scale": s["out_scale"]}


def _run_project(s):
    case = s["case"]
    if own:
        if case["e4m3"]:
            s["px"].adapted_project_e4m3(s["weights"], s["x"], s["x_scale"], s["out"], s["agent_id"], s["workspace"])
        else:
            s["px"].adapted_project(s["weights"], s["x"], s["out"], s["agent_id"], s["workspace"])
        return s["out"]
    x = s["x"].float()
    y = x @ (s["wq"].float() * s["w_scale"] if case["e4m3"] else s["w"].float())
    if case["rank"]:
        rows, k, n, r, agents = (case[f] for f in ("rows", "k", "n", "rank", "agents"))
        t = (x @ s["a"].float().transpose(0, 1).reshape(k, agents * r)).view(rows, agents, r)
        mine = torch.arange(agents, device="cuda")[None, :] == s["agent_id"][:, None]
        y = y + LORA_SCALE * (t * mine[:, :, None]).view(rows, agents * r) @ s["b"].float().view(agents * r, n)
    s["out"].copy_(y * s["x_scale"][:, None] if case["e4m3"] else y)
    return s["out"]


def run(state):
    return _run_norm(state) if state["case"]["op"] == "norm" else _run_project(state)


def work(case):
    if case["op"] == "norm":
        values = case["rows"] * case["width"]
        moved = 2 * (1 + 2 * case["residual"]) + 2 * case["bf16"] + case["e4m3"]
        return {"bytes": values * moved + 2 * case["width"] + 4 * case["rows"] * case["e4m3"], "flops": 5 * values}
    rows, k, n, r, agents = (case[f] for f in ("rows", "k", "n", "rank", "agents"))
    size = 1 if case["e4m3"] else 2
    if case["mix"] == "one":
        present = 1
    elif case["mix"] == "runs":
        present = min(agents, -(-rows // _segments(case)))
    else:                      # as many different ones as so many draws are expected to hit
        present = rows if rows <= agents else agents * (1 - (1 - 1 / (agents + 1)) ** rows)
    moved = size * (rows * k + k * n) + 2 * rows * n + 4 * rows + 2 * present * r * (k + n) + (4 * (rows + n) if case["e4m3"] else 0)
    return {"bytes": moved, "flops": 2 * rows * (k * n + r * (k + n))}


def exact(case, seed):
    """The outputs from the definition in 64 bits."""
    s = _draw_inputs(case, seed)
    if case["op"] == "norm":
        total = s["x"].double()
        if case["residual"]:
            total += s["residual"].double()
        root = (torch.linalg.vector_norm(total, dim=1).square() / case["width"] + EPS).sqrt()
        y = total / root[:, None] * s["gain"].double()
        out = {"residual": total if case["residual"] else None, "out": y if case["bf16"] else None, "q": None, "scale": None}
        if case["e4m3"]:
            peak = torch.linalg.vector_norm(y, ord=math.inf, dim=1)
            peak[peak == 0] = E4M3_MAX
            out["scale"] = peak / E4M3_MAX
            out["q"] = y / out["scale"][:, None]
        return out
    x, w = s["x"].double(), s["w"].double()
    if case["e4m3"]:
        peak = w.abs().max(dim=0).values
        mantissa, exponent = torch.frexp(peak / E4M3_MAX)
        exponent -= (mantissa == 0.5).to(exponent.dtype)
        step = torch.ldexp(torch.ones_like(peak), exponent)
        step[peak == 0] = 1
        w = (w / step).to(torch.float8_e4m3fn).double() * step
        x = x * s["x_scale"].double()[:, None]
    y = x @ w
    if case["rank"]:
        for agent in range(case["agents"]):
            rows = (s["agent_id"] == agent).nonzero()[:, 0]
            if rows.numel():
                y[rows] += LORA_SCALE * (x[rows] @ s["a"][agent].double()) @ s["b"][agent].double()
    return y
