"""Operators at the boundary of the quantised layer, as cases that can be timed and compared.

A case is one pass through one operator:

* ``norm``      the residual's addition and the root-mean-square norm in front of a layer (``add_rms_norm``);
* ``gate``      the gated activation in front of the down projection (``gated_activation``);
* ``adapters``  the low-rank adapters of the requests of a batch beside a shared projection (``apply_adapters``).

Shapes are those of bench.py and of the test configurations: hidden 4096 / feed-forward 11008, hidden 5120 / feed-forward 13824,
1 to 4096 tokens, sizes that are no multiple of any tile; activations in fp32, bf16 and MXINT8.  An MXINT8 output is read
back as the values that it stands for (``dequantize_activations``; exact in bf16), which is part of such a pass.

Each operator has a plain form in torch (``own`` False) next to the call of the library (``own`` True).  What an 8-bit output
holds is decided in 64 bits in the plain form too: a value next to a rounding border goes to the side on which it lies.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5
BLOCK = 16
EXP_MIN, EXP_MAX = -56, 55
_FLOAT = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4.0, "bf16": 2.0, "mxint8": 17.0 / 16.0}


def _norm(rows, K, x="bf16", res="bf16", y="mxint8", bits=8):
    return {"op": "norm", "rows": rows, "K": K, "x": x, "res": res, "y": y, "bits": bits}


def _gate(rows, N, x="bf16", y="mxint8", act="silu", joined=False, bits=8):
    """joined: gate and up are the halves of one [rows, 2 N] tensor."""
    return {"op": "gate", "rows": rows, "N": N, "x": x, "y": y, "act": act, "joined": joined, "bits": bits}


def _adapters(rows, K, N, rank, slots, requests, used, x="bf16", y0="bf16", y="bf16", mixed=False, bare=0, plan=False):
    """slots: adapters loaded.  requests: the rows belong to that many requests, in runs of uneven length.  used: different
    adapters among them.  bare: requests without one.  mixed: ranks of rank, rank / 2, rank / 4 and rank / 8 in turn.
    plan: the batch is a new one, so its rows are sorted by adapter within the pass."""
    return {"op": "adapters", "rows": rows, "K": K, "N": N, "rank": rank, "slots": slots, "requests": requests, "used": used,
            "x": x, "y0": y0, "y": y, "mixed": mixed, "bare": bare, "plan": plan}


def listed():
    cases = {
        # one token in front of q, k, v: latency
        "norm_m1": _norm(1, 4096, y="bf16"),
        # a ragged batch on a hidden size that fits no tile, the layer's fp32 output and an fp32 residual
        "norm_m201": _norm(201, 4112, x="f32", res="f32"),
        # a prompt of 2048 tokens, handed on quantised
        "norm_m2048": _norm(2048, 4096),
        # one token between gate / up and down
        "gate_m1": _gate(1, 11008, y="bf16"),
        # a serving batch of 64 sequences, fp32 from the layers before, handed on quantised
        "gate_m64": _gate(64, 13824, x="f32"),
        # a prompt through a fused gate-and-up projection
        "gate_m2048": _gate(2048, 11008, joined=True),
        # one sequence with its adapter on an attention projection: latency
        "adapters_m1": _adapters(1, 4096, 4096, 16, 4, 1, 1),
        # sixteen sequences, sixteen adapters of different ranks, quantised activations, fp32 sums
        "adapters_m16": _adapters(16, 4096, 11008, 64, 16, 16, 16, x="mxint8", y0="f32", y="f32", mixed=True),
        # a serving batch of 64 sequences that share 24 adapters, eight of them on the base model
        "adapters_m64": _adapters(64, 5120, 5120, 16, 32, 64, 24, bare=8),
        # a chunk of six short prompts, sizes that fit no tile, an odd rank, the batch's first projection
        "adapters_m201": _adapters(201, 4112, 10992, 20, 8, 6, 4, x="f32", y0="f32", bare=1, plan=True),
        # prompts of four requests, bf16 activations
        "adapters_m2048": _adapters(2048, 4096, 11008, 64, 8, 4, 4),
        # a long prompt on the larger model, fp32 activations in and out
        "adapters_m4096": _adapters(4096, 5120, 13824, 64, 4, 2, 2, x="f32", y0="f32", y="f32"),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def draw(rng):
    """One more case of the same ranges."""
    def log_uniform(lo, hi):
        return lo * (hi / lo) ** rng.random()

    op = rng.choice(("norm", "gate", "adapters", "adapters"))
    rows = max(1, min(4096, int(round(log_uniform(0.7, 4096)))))
    kind = ("f32", "bf16")
    if op == "norm":
        K = 16 * int(log_uniform(16, 865))
        rows = min(rows, 20_000_000 // K)
        return _norm(rows, K, rng.choice(kind), rng.choice(kind), rng.choice(kind + ("mxint8", "mxint8")), rng.choice((8, 8, 8, 6)))
    if op == "gate":
        N = 16 * int(log_uniform(16, 865))
        rows = min(rows, 28_000_000 // N)
        return _gate(rows, N, rng.choice(kind), rng.choice(kind + ("mxint8", "mxint8")), rng.choice(("silu", "silu", "gelu")), rng.random() < 0.5,
                     rng.choice((8, 8, 8, 6)))
    K, N = 16 * int(log_uniform(16, 690)), 8 * int(log_uniform(32, 1729))
    rank = rng.choice((5, 8, 16, 16, 20, 32, 64))
    if rows <= 256:      # decoding: a row is a request of its own, or one of a few of a short prompt
        rank = rng.choice((rank, 100, 128))
        slots = rng.choice((1, 4, 16, 32, 64))
        requests = rows if rng.random() < 0.7 else max(1, min(rows, int(log_uniform(1, 32))))
    else:
        slots = rng.choice((1, 2, 4, 8))
        requests = int(log_uniform(1, 17))
    bare = rng.choice((0, 0, requests // 4))
    used = min(slots, requests - bare, max(1, int(log_uniform(1, slots + 1))))
    return _adapters(rows, K, N, rank, slots, requests, used, rng.choice(kind + ("mxint8",)), rng.choice(kind), rng.choice(kind), rng.random() < 0.3,
                     bare, rng.random() < 0.25)


def _ranks(case):
    return [max(1, case["rank"] >> (s % 4)) if case["mixed"] else case["rank"] for s in range(case["slots"])]


def _generator(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 8 + stream)
    return g


def _activations(rows, cols, kind, g, spread=1.0):
    """Normal values with a few outlier channels."""
    x = torch.randn((rows, cols), generator=g, device=DEV) * spread
    at = torch.randint(0, cols, (max(1, cols // 200),), generator=g, device=DEV)
    x[:, at] *= 20.0
    return x.to(_FLOAT[kind])


def _inputs(case, seed):
    """What the program has in hand, as plain tensors."""
    g = _generator(seed, {"norm": 0, "gate": 1, "adapters": 2}[case["op"]])
    rows = case["rows"]
    if case["op"] == "norm":
        return {"x": _activations(rows, case["K"], case["x"], g), "res": _activations(rows, case["K"], case["res"], g, 2.0),
                "w": 1.0 + 0.2 * torch.randn(case["K"], generator=g, device=DEV)}
    if case["op"] == "gate":
        N = case["N"]
        if case["joined"]:
            both = _activations(rows, 2 * N, case["x"], g)
            return {"gate": both[:, :N], "up": both[:, N:]}
        return {"gate": _activations(rows, N, case["x"], g), "up": _activations(rows, N, case["x"], g)}
    K, N, S, R = case["K"], case["N"], case["slots"], case["rank"]
    s = {"A": (torch.randn((S, K, R), generator=g, device=DEV) / K ** 0.5).bfloat16(),
         "B": (torch.randn((S, R, N), generator=g, device=DEV) * 0.5 / R ** 0.5).bfloat16(),
         "scale": 0.5 + torch.rand(S, generator=g, device=DEV)}
    for j, r in enumerate(_ranks(case)):
        s["A"][j, :, r:] = 0
        s["B"][j, r:] = 0
    x = _activations(rows, K, "f32" if case["x"] == "mxint8" else case["x"], g)
    s["x"] = _pack(*_quantised(x.double(), 8)) if case["x"] == "mxint8" else x
    s["y0"] = _activations(rows, N, case["y0"], g)
    # requests of uneven length, each with a slot; `used` different slots among those that have one
    picks = torch.randperm(S, generator=g, device=DEV)[:max(1, case["used"])]
    of = picks[torch.arange(case["requests"], device=DEV) % len(picks)]
    of[case["requests"] - case["bare"]:] = -1
    of = of[torch.randperm(case["requests"], generator=g, device=DEV)]
    if case["requests"] == rows:
        request = torch.arange(rows, device=DEV)
    else:
        cuts = 1 + torch.randperm(rows - 1, generator=g, device=DEV)[:case["requests"] - 1]
        request = torch.zeros(rows, dtype=torch.int64, device=DEV).index_fill_(0, cuts, 1).cumsum(0)
    s["slots"] = of[request].to(torch.int32)
    return s


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=dict(case))
    if own:
        import paper_2402_02446_b200 as L
        state["cfg"] = L.default_config()
        state["cfg"].a_bits = case.get("bits", 8)
        if case["op"] == "adapters":
            pool = L.new_adapter_pool(case["K"], case["N"], case["rank"], case["slots"])
            for j, r in enumerate(_ranks(case)):
                L.load_adapter(pool, j, state["A"][j, :, :r].contiguous(), state["B"][j, :r].contiguous(), float(state["scale"][j]))
            state["pool"], state["plan"] = pool, L.adapter_plan(state["slots"], pool)
    return state


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the calls of the library ----------------------------------------------------------------------------------------------------

def _run_own(s):
    import paper_2402_02446_b200 as L
    c = s["case"]
    if c["op"] == "adapters":
        plan = L.adapter_plan(s["slots"], s["pool"], plan=s["plan"]) if c["plan"] else s["plan"]
        return {"y": L.apply_adapters(s["x"], s["pool"], plan, s["y0"], out_dtype=_FLOAT[c["y"]], cfg=s["cfg"])}
    out_dtype = L.MXINT8 if c["y"] == "mxint8" else _FLOAT[c["y"]]
    if c["op"] == "norm":
        y, res = L.add_rms_norm(s["x"], s["w"], EPS, residual=s["res"], out_dtype=out_dtype, cfg=s["cfg"])
        out = {"res": res}
    else:
        y, out = L.gated_activation(s["gate"], s["up"], act=c["act"], out_dtype=out_dtype, cfg=s["cfg"]), {}
    if c["y"] == "mxint8":
        y = L.dequantize_activations(y, c["rows"], c["K"] if c["op"] == "norm" else c["N"], out_dtype=torch.bfloat16, cfg=s["cfg"])
    return dict(out, y=y)


# ---- the plain forms -------------------------------------------------------------------------------------------------------------

def _quantised(v, bits):
    """Mantissas and exponents (blocks of 16 along the row) of fp64 values."""
    b = v.unflatten(-1, (-1, BLOCK))
    e = (torch.frexp(b.abs().amax(-1, keepdim=True))[1] - 1).clamp(EXP_MIN, EXP_MAX)
    top = 2 ** (bits - 1) - 1
    m = torch.round(torch.ldexp(b, bits - 2 - e)).clamp(-top, top)
    return m.flatten(-2), e.squeeze(-1)


def _values(m, e, bits):
    step = torch.ldexp(torch.ones_like(e, dtype=m.dtype), e - (bits - 2))
    return (m.unflatten(-1, (-1, BLOCK)) * step[..., None]).flatten(-2)


def _pack(m, e):
    """The library's MXINT8 buffer: mantissas, then exponent bytes."""
    return torch.cat([m.to(torch.int8).view(torch.uint8).flatten(), (e + 127).to(torch.uint8).flatten()])


def _unpacked(buf, rows, cols, bits=8):
    m = buf[:rows * cols].view(torch.int8).view(rows, cols).float()
    return _values(m, buf[rows * cols:].view(rows, cols // BLOCK).int() - 127, bits)


def _act(g, act):
    if act == "silu":
        return g / (1.0 + torch.exp(-g))
    return g / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g)))


def _run_plain(s):
    c = s["case"]
    wide = torch.float64 if c["y"] == "mxint8" else torch.float32
    if c["op"] == "adapters":
        x = _unpacked(s["x"], c["rows"], c["K"]) if c["x"] == "mxint8" else s["x"].float()
        t = torch.matmul(x, s["A"].float()) * s["scale"][:, None, None]
        mine = s["slots"] == torch.arange(c["slots"], device=x.device)[:, None]
        t = torch.where(mine[..., None], t, 0.0)
        y = torch.matmul(t.transpose(0, 1).flatten(1), s["B"].float().flatten(0, 1))
        return {"y": (s["y0"].float() + y).to(_FLOAT[c["y"]])}
    if c["op"] == "norm":
        res = (s["x"].float() + s["res"].float()).to(_FLOAT[c["res"]])
        h = res.to(wide)
        y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * s["w"].to(wide)
        out = {"res": res}
    else:
        y, out = _act(s["gate"].to(wide), c["act"]) * s["up"].to(wide), {}
    if c["y"] == "mxint8":
        return dict(out, y=_values(*_quantised(y, c["bits"]), c["bits"]).bfloat16())
    return dict(out, y=y.to(_FLOAT[c["y"]]))


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "adapters":
        K, rows = case["K"], case["rows"]
        if case["x"] == "mxint8":
            step = torch.pow(2.0, s["x"][rows * K:].double() - 127 - 6).view(rows, K // BLOCK)
            x = s["x"][:rows * K].view(torch.int8).double().view(rows, K) * step.repeat_interleave(BLOCK, 1)
        else:
            x = s["x"].double()
        y = s["y0"].double()
        for j in range(case["slots"]):
            at = (s["slots"] == j).nonzero()[:, 0]
            if len(at):
                y[at] += s["scale"][j].double() * ((x[at] @ s["A"][j].double()) @ s["B"][j].double())
        return {"y": y}
    if case["op"] == "norm":
        total = s["x"].double() + s["res"].double()
        h = total.to(_FLOAT[case["res"]]).double()
        y = h / torch.sqrt((h * h).sum(-1, keepdim=True) / case["K"] + EPS) * s["w"].double()
        out = {"res": total}
    else:
        g, u = s["gate"].double(), s["up"].double()
        if case["act"] == "silu":
            y = g * torch.sigmoid(g) * u
        else:
            y = 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3))) * u
        out = {}
    if case["y"] == "mxint8":
        rows, n = y.shape
        b = y.view(rows, n // BLOCK, BLOCK)
        power = torch.floor(torch.log2(b.abs().amax(-1)))
        step = torch.pow(2.0, power.clamp(EXP_MIN, EXP_MAX) - (case["bits"] - 2))[..., None]
        top = 2.0 ** (case["bits"] - 1) - 1
        y = (torch.clamp(torch.round(b / step), -top, top) * step).view(rows, n)
    return dict(out, y=y)


def work(case):
    rows = case["rows"]
    if case["op"] == "norm":
        n = rows * case["K"]
        return {"bytes": n * (_BYTES[case["x"]] + 2 * _BYTES[case["res"]] + _BYTES[case["y"]]) + 4.0 * case["K"], "flops": 5.0 * n}
    if case["op"] == "gate":
        n = rows * case["N"]
        return {"bytes": n * (2 * _BYTES[case["x"]] + _BYTES[case["y"]]), "flops": 6.0 * n}
    K, N = case["K"], case["N"]
    # the adapters that are used, at the mean rank of those loaded; the rows that have one
    rank = sum(_ranks(case)) / case["slots"]
    mine = rows * (case["requests"] - case["bare"]) / case["requests"]
    return {"bytes": case["used"] * rank * (K + N) * 2.0 + mine * K * _BYTES[case["x"]] + rows * N * (_BYTES[case["y0"]] + _BYTES[case["y"]]),
            "flops": 2.0 * mine * rank * (K + N)}
