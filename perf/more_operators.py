"""Cases of the operators of a decoder layer's mixture of experts, and of the norms around its AllReduces.

Four operators, each with a plain form in elementary torch operations and the library's call:

* ``norm``     what follows an AllReduce: the block's result normed, gated, scaled and added to the residual stream, and
               the sum normed for the next block;
* ``route``    the experts of every token with their weights, and the lists that sort tokens by expert;
* ``experts``  one matrix product per expert over the tokens that chose it, ragged sizes, gated activation;
* ``combine``  the weighted sum of a token's rows, back in the tokens' order.

Norm.  a = after(x), r = residual_scale * residual + scale * act(gate) * a, y = before(r), where a norm of kind "rms" is
v / sqrt(mean(v^2) + eps) * w + b, one of kind "layer" (v - mean) / sqrt(var + eps) * w + b.

Route.  score = softmax(logits) or sigmoid(logits); a token's experts are the top_k with the largest logits (score + bias
where there is a bias), the lowest index first among equals; its weights are their scores, divided by their sum where
``renormalise`` is true, times ``scale``.  An expert whose logit (or bias) is -inf is nobody's: -1 and a weight of 0 stand
where a token has too few others.  Rows are sorted by expert, then by token: row_token names every row's token,
token_row every choice's row, expert_start[e] .. expert_start[e + 1] are expert e's rows.

Experts.  out[r] = act(x[token of r] w_e^T + b_e), or act(gate) * up where w_e holds first the gate's rows, then up's.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------
def _norm(name, m, n, heads=0, after="none", before="rms", gate="none", gate_act="none", residual=True, bias=False,
          dtype="bf16", stream="bf16", scale=1.0, residual_scale=1.0):
    return {"name": name, "op": "norm", "m": m, "n": n, "heads": heads, "after": after, "before": before, "gate": gate,
            "gate_act": gate_act, "residual": residual, "bias": bias, "dtype": dtype, "stream": stream, "scale": scale,
            "residual_scale": residual_scale}


def _route(name, tokens, experts, top_k, score="softmax", bias=False, renormalise=True, scale=1.0, dtype="f32", idle=0):
    return {"name": name, "op": "route", "tokens": tokens, "experts": experts, "top_k": top_k, "score": score,
            "bias": bias, "renormalise": renormalise, "scale": scale, "dtype": dtype, "idle": idle}


def _experts(name, tokens, experts, top_k, n, k, ranks=1, gated=False, act="none", bias=False, by_row=False, out="bf16",
             skew=0.5, idle=0):
    return {"name": name, "op": "experts", "tokens": tokens, "experts": experts, "top_k": top_k, "n": n, "k": k,
            "ranks": ranks, "gated": gated, "act": act, "bias": bias, "by_row": by_row, "out": out, "skew": skew,
            "idle": idle}


def _combine(name, tokens, experts, top_k, n, ranks=1, residual=False, root=-1, dtype="bf16", out="bf16", idle=0):
    return {"name": name, "op": "combine", "tokens": tokens, "experts": experts, "top_k": top_k, "n": n, "ranks": ranks,
            "residual": residual, "root": root, "dtype": dtype, "out": out, "idle": idle}


def listed():
    return [
        # one token after the AllReduce (hidden size 8192): residual and the next block's norm, latency
        _norm("norm_token", 1, 8192),
        # norm of every query and key head before the rotation, read out of the fused projection's result
        _norm("norm_heads", 4096, 128, heads=18, residual=False),
        # odd sizes, float32 residual stream, layer norms with bias, one gate a token
        _norm("norm_odd", 1501, 2049, after="layer", before="layer", gate="row", gate_act="sigmoid", bias=True,
              stream="f32"),
        # long prompts, norms on both sides of the block, a scale for every channel: bandwidth
        _norm("norm_prompt", 16384, 8192, after="rms", gate="channel", scale=0.5, residual_scale=1.25),
        # a decode batch with idle slots: latency
        _route("route_decode", 64, 128, 8, dtype="bf16", idle=5),
        # long prompts, sigmoid scores, experts balanced by a bias
        _route("route_prompt", 16384, 256, 8, score="sigmoid", bias=True, scale=2.5),
        # one token through eight of 128 experts: the weights of those eight
        _experts("experts_token", 1, 128, 8, 768, 2048, gated=True, act="silu"),
        # a decode batch of four ranks, idle slots among it, the way down: nearly every expert for a few tokens
        _experts("experts_decode", 64, 64, 6, 2048, 352, ranks=4, by_row=True, idle=5),
        # odd sizes, float32 partial sums, two ranks
        _experts("experts_odd", 333, 7, 3, 1003, 520, ranks=2, bias=True, act="gelu", out="f32"),
        # a prompt through the gated products: tensor cores
        _experts("experts_prompt", 4096, 32, 4, 1024, 4096, gated=True, act="silu"),
        # a decode batch back in order, partial sums of eight ranks; the residual joins on one
        _combine("combine_decode", 64, 128, 8, 2048, ranks=8, residual=True, root=0),
        # a prompt back in order: bandwidth
        _combine("combine_prompt", 8192, 32, 4, 4096, idle=100),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "route", "experts", "experts", "combine"])
    idle = rng.choice([0, 0, rng.randint(1, 8)])
    if op == "norm":
        while True:
            heads = rng.choice([0, 0, 0, 1, 2, 10, 18])
            m = _log(rng, 1, 16384)
            n = rng.choice([64, 128, 256]) if heads else _log(rng, 64, 16384)
            if not heads and rng.random() < 0.6:
                n = max(64, n // 64 * 64)
            if m * n * max(heads, 1) <= 1 << 27:
                break
        c = _norm("", m, n, heads=heads, after=rng.choice(["none", "rms", "layer"]), before=rng.choice(["none", "rms", "rms", "layer"]),
                  gate=rng.choice(["none", "none", "row", "channel", "all"]), gate_act=rng.choice(["none", "sigmoid", "tanh"]),
                  residual=rng.random() < 0.7, bias=rng.random() < 0.4, dtype=rng.choice(["bf16", "bf16", "f32"]),
                  stream=rng.choice(["bf16", "bf16", "f32"]), scale=rng.choice([1.0, 0.22]), residual_scale=rng.choice([1.0, 1.5]))
        if c["before"] == "none" and not c["residual"]:
            c["before"] = "rms"
        if c["m"] * c["n"] * max(heads, 1) > 1 << 26:               # not above the largest listed one's bytes
            c["dtype"], c["stream"] = "bf16", "bf16"
            c["gate"] = "channel" if c["gate"] == "all" else c["gate"]
    elif op == "route":
        while True:
            tokens, experts = _log(rng, 1, 16384), rng.choice([8, 16, 60, 64, 128, 160, 256, rng.randint(2, 512)])
            top_k = rng.choice([1, 2, 4, 6, 8])
            if top_k <= experts and tokens * experts <= 16384 * 256:
                break
        c = _route("", tokens, experts, top_k, score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.4,
                   renormalise=rng.random() < 0.6, scale=rng.choice([1.0, 2.5]), dtype=rng.choice(["f32", "bf16"]),
                   idle=min(idle, tokens - 1))
    elif op == "experts":
        while True:
            tokens, experts, top_k = _log(rng, 1, 8192), rng.choice([4, 8, 16, 32, 60, 64, 128]), rng.choice([1, 2, 4, 6, 8])
            n, k, ranks = _log(rng, 64, 4096), _log(rng, 64, 8192), rng.choice([1, 1, 2, 4, 8])
            k = max(8, k // 8 * 8)
            if rng.random() < 0.6:
                n, k = max(64, n // 64 * 64), max(64, k // 64 * 64)
            gated = rng.random() < 0.5
            wide = 2 if gated else 1
            rows = tokens * top_k
            if top_k <= experts and ranks * experts * wide * n * k <= 1 << 28 and ranks * rows * (n + k) <= 1 << 26 and \
                    ranks * rows * wide * n * k <= 1 << 37:
                break
        c = _experts("", tokens, experts, top_k, n, k, ranks=ranks, gated=gated,
                     act=rng.choice(["silu", "gelu_tanh"]) if gated else rng.choice(["none", "relu", "gelu", "silu"]),
                     bias=rng.random() < 0.3, by_row=rng.random() < 0.5, out=rng.choice(["bf16", "bf16", "f32"]),
                     skew=rng.choice([0.0, 0.5, 1.0, 3.0]), idle=min(idle, tokens - 1))
    else:
        while True:
            tokens, experts, top_k = _log(rng, 1, 8192), rng.choice([8, 32, 64, 128]), rng.choice([1, 2, 4, 6, 8])
            n, ranks = _log(rng, 64, 8192), rng.choice([1, 1, 2, 4, 8])
            if rng.random() < 0.6:
                n = max(64, n // 64 * 64)
            if ranks * tokens * n * (top_k + 1) <= 160 << 20:
                break
        c = _combine("", tokens, experts, top_k, n, ranks=ranks, residual=rng.random() < 0.5,
                     root=rng.choice([-1, 0, ranks - 1]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                     out=rng.choice(["bf16", "bf16", "f32"]), idle=min(idle, tokens - 1))
        if ranks * tokens * n * (top_k + 1) > 80 << 20:
            c["dtype"] = c["out"] = "bf16"
    del c["name"]
    return c


def _width(name):
    return 4 if name == "f32" else 2


def work(case):
    if case["op"] == "norm":
        n = case["n"]
        cells = case["m"] * max(case["heads"], 1) * n
        x, s = _width(case["dtype"]), _width(case["stream"])
        gate = {"none": 0, "row": cells // n, "channel": n, "all": cells}[case["gate"]]
        weights = (1 + case["bias"]) * ((case["after"] != "none") + (case["before"] != "none")) * n
        return {"bytes": cells * (x * (1 + (case["before"] != "none")) + 2 * s * case["residual"]) + x * (gate + weights),
                "flops": cells * (3 * case["residual"] + 4 * ((case["after"] != "none") + (case["before"] != "none")))}
    rows = (case["tokens"] - case["idle"]) * case["top_k"]
    slots = case["tokens"] * case["top_k"]
    if case["op"] == "route":
        cells = case["tokens"] * case["experts"]
        return {"bytes": cells * _width(case["dtype"]) + 4 * case["experts"] * case["bias"] + 16 * slots +
                4 * (case["experts"] + 1), "flops": 4 * cells}
    ranks, n, wide = case["ranks"], case["n"], _width(case["out"])
    if case["op"] == "experts":
        k, w_rows = case["k"], n * (2 if case["gated"] else 1)
        # experts that some token has chosen, were all of them liked alike
        used = round(case["experts"] * (1.0 - (1.0 - case["top_k"] / case["experts"]) ** (case["tokens"] - case["idle"])))
        x_rows = ranks * rows if case["by_row"] else case["tokens"] - case["idle"]
        return {"bytes": 2 * ranks * used * w_rows * (k + case["bias"]) + 2 * x_rows * k + wide * ranks * rows * n +
                4 * (rows + case["experts"] + 1), "flops": 2 * ranks * rows * w_rows * k}
    added = (ranks if case["root"] < 0 else 1) * case["tokens"] * n if case["residual"] else 0
    return {"bytes": _width(case["dtype"]) * ranks * rows * n + wide * (ranks * case["tokens"] * n + added) + 8 * slots,
            "flops": 2 * ranks * rows * n}


# ---------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------
def _sorted_by_expert(choice, experts):
    """(expert_start, row_token, token_row) int32 of the choices [tokens][top_k], -1 for none."""
    tokens, top_k = choice.shape
    mine = torch.where(choice < 0, experts, choice).flatten().long()
    order = torch.sort(mine, stable=True)
    start = torch.searchsorted(order.values, torch.arange(experts + 1, device=choice.device))
    row = torch.arange(tokens * top_k, device=choice.device)
    there = row < start[-1]
    row_token = torch.where(there, order.indices // top_k, -1)
    token_row = torch.empty_like(row)
    token_row[order.indices] = torch.where(there, row, -1)
    return start.to(torch.int32), row_token.to(torch.int32), token_row.view(tokens, top_k).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16, scale=1.0):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)

    state = {"case": dict(case)}
    if case["op"] == "norm":
        m, n, heads = case["m"], case["n"], case["heads"]
        dtype, stream = DTYPES[case["dtype"]], DTYPES[case["stream"]]
        shape = (m, heads, n) if heads else (m, n)
        # heads: the first ones of a wider row, as a fused projection leaves them; others: rows of their own, with the
        # few large channels that activations have
        x = normal(m, heads + 2 if heads else 1, n, dtype=torch.float32)
        x = x[:, :heads] if heads else x[:, 0]
        x[..., :: max(1, n // 5)] *= 20.0
        state["x"] = x.to(dtype) if not heads else x.to(dtype).contiguous()
        if heads:
            room = torch.zeros(m, heads + 2, n, dtype=dtype, device="cuda")
            room[:, :heads] = state["x"]
            state["x"] = room[:, :heads]
        state["residual"] = normal(*shape, dtype=stream, scale=3.0) if case["residual"] else None
        gate = {"none": None, "row": (*shape[:-1], 1), "channel": (n,), "all": shape}[case["gate"]]
        state["gate"] = normal(*gate, dtype=dtype) if gate else None
        for side in ("after", "before"):
            state[side + "_w"] = (1.0 + normal(n, dtype=torch.float32, scale=0.1)).to(dtype)
            state[side + "_b"] = normal(n, dtype=dtype, scale=0.1) if case["bias"] else None
        return state
    tokens, experts, top_k = case["tokens"], case["experts"], case["top_k"]
    active = torch.ones(tokens, dtype=torch.bool, device="cuda")
    if case["idle"]:
        active[torch.randperm(tokens, generator=gen, device="cuda")[:case["idle"]]] = False
    logits = normal(tokens, experts, dtype=torch.float32, scale=1.5)
    if case["op"] == "route":
        # some experts are liked more; the rows of idle slots are masked
        logits += normal(experts, dtype=torch.float32)
        logits[~active] = -math.inf
        state["logits"] = logits.to(DTYPES[case["dtype"]])
        state["bias"] = normal(experts, dtype=torch.float32, scale=0.05) if case["bias"] else None
        return state
    logits += normal(experts, dtype=torch.float32, scale=case.get("skew", 0.5))
    best = torch.sort(logits, dim=1, descending=True, stable=True)
    choice = torch.where(active[:, None], best.indices[:, :top_k], -1).to(torch.int32)
    weights = torch.softmax(best.values[:, :top_k], -1)
    state["choice"] = choice
    state["weights"] = torch.where(active[:, None], weights, 0.0).contiguous()
    state["expert_start"], state["row_token"], state["token_row"] = _sorted_by_expert(choice, experts)
    rows, ranks, n = tokens * top_k, case["ranks"], case["n"]
    if case["op"] == "experts":
        k, w_rows = case["k"], n * (2 if case["gated"] else 1)
        state["w"] = torch.empty(ranks, experts, w_rows, k, dtype=torch.bfloat16, device="cuda")
        for r in range(ranks):
            for e in range(experts):
                state["w"][r, e] = normal(w_rows, k, scale=k ** -0.5)
        # activations of tokens, which all ranks share, or of the ranks' rows, as the way up leaves them
        state["x"] = normal(ranks, rows, k) if case["by_row"] else normal(tokens, k)
        state["bias"] = normal(ranks, experts, w_rows) if case["bias"] else None
        # rows of nobody stay as they are
        state["out"] = torch.zeros(ranks, rows, n, dtype=DTYPES[case["out"]], device="cuda")
        state["counts"] = state["expert_start"].diff().tolist()
        return state
    state["y"] = normal(ranks, rows, n, dtype=DTYPES[case["dtype"]])
    state["residual"] = normal(tokens, n, dtype=DTYPES[case["out"]]) if case["residual"] else None
    return state


# ---------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


EPS = 1e-5


def _plain_normed(v, kind, w, b):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v * (1.0 / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)) * w.float()
    return v if b is None else v + b.float()


def _plain_norm(state):
    case = state["case"]
    r = _plain_normed(state["x"].float(), case["after"], state["after_w"], state["after_b"]) * case["scale"]
    if state["gate"] is not None:
        g = state["gate"].float()
        if case["gate_act"] == "sigmoid":
            g = 1.0 / (1.0 + torch.exp(-g))
        elif case["gate_act"] == "tanh":
            g = torch.tanh(g)
        r = r * g
    got = {}
    if state["residual"] is not None:
        r = r + state["residual"].float() * case["residual_scale"]
        got["residual"] = r.to(DTYPES[case["stream"]])
    if case["before"] != "none":
        got["y"] = _plain_normed(r, case["before"], state["before_w"], state["before_b"]).to(DTYPES[case["dtype"]])
    return got


def _plain_route(state):
    case = state["case"]
    wide = state["logits"].double()                     # choices next to a border
    there = wide > -math.inf
    if case["score"] == "sigmoid":
        score = 1.0 / (1.0 + torch.exp(-wide))
    else:
        top = wide.amax(-1, keepdim=True)
        score = torch.exp(wide - torch.where(there.any(-1, keepdim=True), top, 0.0))
        score = score / score.sum(-1, keepdim=True).clamp(min=1e-300)
    key = wide if state["bias"] is None else torch.where(there, score + state["bias"].double(), -math.inf)
    best = torch.sort(key, dim=1, descending=True, stable=True)
    found = best.values[:, :case["top_k"]] > -math.inf
    choice = torch.where(found, best.indices[:, :case["top_k"]], -1).to(torch.int32)
    weights = torch.where(found, torch.gather(score, 1, best.indices[:, :case["top_k"]]), 0.0)
    if case["renormalise"]:
        weights = weights / weights.sum(-1, keepdim=True).clamp(min=1e-300)
    start, row_token, token_row = _sorted_by_expert(choice, case["experts"])
    return {"choice": choice, "weights": (weights * case["scale"]).float(), "expert_start": start, "row_token": row_token,
            "token_row": token_row}


def _activate(x, act):
    if act == "relu":
        return x.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x * 0.7071067811865476))
    if act == "gelu_tanh":
        return 0.5 * x * (1.0 + torch.tanh(0.7978845608028654 * (x + 0.044715 * x * x * x)))
    if act == "silu":
        return x / (1.0 + torch.exp(-x))
    return x


def _plain_experts(state):
    case, n, out, first = state["case"], state["case"]["n"], state["out"], 0
    for e, count in enumerate(state["counts"]):
        if count:
            rows = slice(first, first + count)
            x = state["x"][:, rows] if case["by_row"] else state["x"][state["row_token"][rows].long()][None]
            y = torch.matmul(x.float(), state["w"][:, e].float().transpose(1, 2))
            if state["bias"] is not None:
                y = y + state["bias"][:, e, None].float()
            y = _activate(y[..., :n], case["act"]) * y[..., n:] if case["gated"] else _activate(y, case["act"])
            out[:, rows] = y.to(out.dtype)
            first += count
    return out


def _plain_combine(state):
    case = state["case"]
    at = state["token_row"].long()
    y = state["y"][:, at.clamp(min=0)].float()          # [ranks][tokens][top_k][n]
    w = torch.where(at < 0, 0.0, state["weights"])
    got = (y * w[..., None]).sum(2)
    if state["residual"] is not None:
        mine = slice(None) if case["root"] < 0 else slice(case["root"], case["root"] + 1)
        got[mine] += state["residual"].float()
    return got.to(DTYPES[case["out"]])


_plain = {"norm": _plain_norm, "route": _plain_route, "experts": _plain_experts, "combine": _plain_combine}


def _kept(state, name, make):
    """What a program makes once of its weights or lists and hands to every call."""
    if name not in state:
        state[name] = make()
    return state[name]


def _routes(state):
    from paper_2607_16100_b200 import symar
    return symar, _kept(state, "routes", lambda: symar.Routes(state["choice"], state["weights"], state["expert_start"],
                                                              state["row_token"], state["token_row"]))


def _own_norm(state):
    from paper_2607_16100_b200 import symar
    case = state["case"]

    def side(which):
        if case[which] == "none":
            return None
        return symar.Norm(case[which], state[which + "_w"], state[which + "_b"], eps=EPS)

    after, before = (_kept(state, which, lambda: side(which)) for which in ("after", "before"))
    y, residual = symar.norm(state["x"], state["residual"], after=after, before=before, gate=state["gate"],
                             gate_act=case["gate_act"], scale=case["scale"], residual_scale=case["residual_scale"])
    got = {}
    if residual is not None:
        got["residual"] = residual
    if y is not None:
        got["y"] = y
    return got


def _own_route(state):
    from paper_2607_16100_b200 import symar
    case = state["case"]
    r = symar.route(state["logits"], case["top_k"], bias=state["bias"], score=case["score"],
                    renormalise=case["renormalise"], scale=case["scale"])
    return {"choice": r.choice, "weights": r.weights, "expert_start": r.expert_start, "row_token": r.row_token,
            "token_row": r.token_row}


def _own_experts(state):
    symar, routes = _routes(state)
    case = state["case"]
    return symar.experts(state["x"], state["w"], routes, bias=state["bias"], act=case["act"], gated=case["gated"],
                         by_row=case["by_row"], out=state["out"])


def _own_combine(state):
    symar, routes = _routes(state)
    case = state["case"]
    return symar.combine(state["y"], routes, residual=state["residual"], root=case["root"],
                         out_dtype=DTYPES[case["out"]])


_own = {"norm": _own_norm, "route": _own_route, "experts": _own_experts, "combine": _own_combine}


# ---------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    return {"norm": _exact_norm, "route": _exact_route, "experts": _exact_experts, "combine": _exact_combine}[case["op"]](case, state)


def _exact_rows(v, kind, w, b):
    if kind == "rms":
        v = torch.nn.functional.normalize(v, dim=-1, eps=0.0) * (v.norm(dim=-1, keepdim=True) /
                                                                  (v.square().mean(-1, keepdim=True) + EPS).sqrt()) * w.double()
    elif kind == "layer":
        var, mean = torch.var_mean(v, -1, correction=0, keepdim=True)
        v = (v - mean) / (var + EPS).sqrt() * w.double()
    return v if kind == "none" or b is None else v + b.double()


def _exact_norm(case, state):
    got = {"residual": [], "y": []}
    for t in range(0, case["m"], 1024):                 # a few rows at a time
        rows = slice(t, t + 1024)
        r = _exact_rows(state["x"][rows].double(), case["after"], state["after_w"], state["after_b"])
        if state["gate"] is not None:
            g = (state["gate"] if case["gate"] == "channel" else state["gate"][rows]).double()
            r = r * {"none": lambda v: v, "sigmoid": torch.sigmoid, "tanh": torch.tanh}[case["gate_act"]](g)
        r = case["scale"] * r
        if state["residual"] is not None:
            r = case["residual_scale"] * state["residual"][rows].double() + r
            got["residual"].append(r)
        if case["before"] != "none":
            got["y"].append(_exact_rows(r, case["before"], state["before_w"], state["before_b"]))
    return {name: torch.cat(parts) for name, parts in got.items() if parts}


def _exact_route(case, state):
    logits, k, experts = state["logits"].double(), case["top_k"], case["experts"]
    index = torch.arange(experts, device=logits.device)
    if case["score"] == "sigmoid":
        score = torch.sigmoid(logits)
    else:
        score = torch.softmax(torch.where(torch.isinf(logits).all(-1, keepdim=True), 0.0, logits), -1)
    key = logits.clone() if state["bias"] is None else score + state["bias"].double() + torch.where(torch.isinf(logits), logits, 0.0)
    choice, weights = [], []
    for _ in range(k):                                  # the largest that is left, the first of several
        top = key.amax(-1, keepdim=True)
        at = torch.where(key == top, index, experts).amin(-1)
        some = top[:, 0] != -math.inf
        choice.append(torch.where(some, at, -1))
        weights.append(torch.where(some, score.gather(1, at[:, None])[:, 0], 0.0))
        key[torch.arange(len(at), device=at.device), at] = -math.inf
    choice, weights = torch.stack(choice, 1), torch.stack(weights, 1)
    if case["renormalise"]:
        total = weights.sum(-1, keepdim=True)
        weights = torch.where(total > 0, weights / total, 0.0)
    # every choice's row: those of earlier experts, and of earlier tokens among its own
    flat = choice.flatten()
    mine = (flat[:, None] == index).to(torch.int32)
    start = torch.cat([torch.zeros(1, dtype=torch.long, device=flat.device), mine.sum(0).cumsum(0)])
    before = (mine.cumsum(0) - mine).gather(1, flat.clamp(min=0)[:, None])[:, 0]
    row = torch.where(flat < 0, -1, start[flat.clamp(min=0)] + before)
    row_token = torch.full_like(flat, -1)
    row_token[row[flat >= 0]] = torch.arange(len(flat), device=flat.device)[flat >= 0] // k
    whole = torch.int32
    return {"choice": choice.to(whole), "weights": weights * case["scale"], "expert_start": start.to(whole),
            "row_token": row_token.to(whole), "token_row": row.view(-1, k).to(whole)}


def _exact_experts(case, state):
    got, n = torch.zeros(state["out"].shape, dtype=torch.float64, device="cuda"), case["n"]
    acts = {"none": lambda v: v, "relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v),
            "gelu": lambda v: v * 0.5 * torch.erfc(-v / math.sqrt(2.0)),
            "gelu_tanh": lambda v: v * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))}
    start = state["expert_start"].tolist()
    for r in range(case["ranks"]):
        for e in range(case["experts"]):
            lo, hi = start[e], start[e + 1]
            if lo == hi:
                continue
            x = state["x"][r, lo:hi] if case["by_row"] else state["x"].index_select(0, state["row_token"][lo:hi])
            y = torch.nn.functional.linear(x.double(), state["w"][r, e].double(),
                                           None if state["bias"] is None else state["bias"][r, e].double())
            got[r, lo:hi] = acts[case["act"]](y[:, :n]) * (y[:, n:] if case["gated"] else 1.0)
    return got


def _exact_combine(case, state):
    got = torch.zeros(case["ranks"], case["tokens"], case["n"], dtype=torch.float64, device="cuda")
    for j in range(case["top_k"]):                      # one choice of every token at a time
        token = (state["token_row"][:, j] >= 0).nonzero()[:, 0]
        rows = state["y"].index_select(1, state["token_row"][token, j])
        got.index_add_(1, token, rows.double() * state["weights"][token, j].double()[:, None])
    if state["residual"] is not None:
        for r in range(case["ranks"]):
            if case["root"] in (-1, r):
                got[r] += state["residual"].double()
    return got
