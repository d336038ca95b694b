"""Cases of the operators around the AllReduces of a tensor-parallel decoder layer.

Three operators, each with a plain form in elementary torch operations and the library's call:

* ``linear``     matrix product with bias, activation and residual in its epilogue, for one matrix or one per rank;
* ``append``     new keys and values rotated, quantised to 4 bits and written to a paged cache, the queries rotated in
                 the same call, and the written entries read back as the values they stand for;
* ``attention``  attention of the new tokens over that cache.

The cache.  A page holds ``page`` tokens of one key/value head:

    K codes [page][D/2] bytes | V codes [page][D/2] bytes | K words [page][D/64] u32 | V words [page][D/64] u32

Channel c of a token is nibble c (low nibble first).  Each group of 64 channels has one 32-bit word: a float32 scale s
whose four lowest bits hold the zero point z; a code n stands for s * (n - z).  Quantising a group x: lo = min(0, x),
hi = max(0, x), s = hi/15 - lo/15 with its four lowest bits cleared (0 where that is below 2^-126), z = rint(-lo / s),
n = clamp(rint(x / s) + z, 0, 15), the divisions taken as products with the float32 reciprocal of s.

Sequence b's new tokens are rows token_start[b] .. token_start[b+1] of q, k and v (row b where token_start is None) and
the last ones of its lengths[b] tokens; token t lies in page page_table[b][t // page].  A query sees the tokens up to its
own, at most ``window`` of them where that is not 0; one that sees none gives zeros.
"""
import math

import torch

own = False

GROUP = 64
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------
def _linear(name, groups, m, n, k, out="bf16", act="none", bias=False, residual=False, root=-1, shared=False):
    return {"name": name, "op": "linear", "groups": groups, "m": m, "n": n, "k": k, "out": out, "act": act,
            "bias": bias, "residual": residual, "root": root, "shared": shared}


def _append(name, seqs, new, ctx, q_heads, kv_heads, dim, page, rot, interleaved=False, dtype="bf16", ragged=False):
    return {"name": name, "op": "append", "seqs": seqs, "new": new, "ctx": ctx, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "page": page, "rot": rot, "interleaved": interleaved, "dtype": dtype,
            "ragged": ragged}


def _attention(name, seqs, new, ctx, q_heads, kv_heads, dim, page, window=0, ragged=False):
    return {"name": name, "op": "attention", "seqs": seqs, "new": new, "ctx": ctx, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "page": page, "window": window, "ragged": ragged}


def listed():
    return [
        # one token through one rank's small projection: latency
        _linear("linear_token", 1, 1, 1024, 1024, act="silu", bias=True),
        # the output projection of eight ranks at batch 4 (hidden size 8192): the product before every AllReduce; the
        # residual joins on one rank
        _linear("linear_ranks", 8, 4, 8192, 1024, residual=True, root=0),
        # odd sizes, float32 partial sums: rows that no 16-byte access fits
        _linear("linear_odd", 2, 333, 1003, 2049, out="f32", act="gelu", bias=True, shared=True),
        # a prompt through the first feed-forward product
        _linear("linear_prompt", 1, 4096, 8192, 8192, act="gelu_tanh", bias=True, residual=True),
        # one sequence's next token on one rank: latency
        _append("append_token", 1, 1, 511, 8, 1, 128, 64, 128),
        # a decode batch, all heads, interleaved rotation
        _append("append_decode", 64, 1, 4000, 64, 8, 128, 16, 128, interleaved=True, ragged=True),
        # ragged prompts, part of the head rotated, float32 activations
        _append("append_ragged", 5, 1501, 77, 16, 4, 64, 32, 32, dtype="f32", ragged=True),
        # long prompts: bandwidth
        _append("append_prompt", 4, 4096, 0, 64, 8, 128, 64, 128),
        # one sequence's next token on one rank: latency
        _attention("attention_token", 1, 1, 511, 8, 1, 128, 64),
        # a decode batch of unequal lengths, an idle slot among them
        _attention("attention_decode", 64, 1, 4095, 64, 8, 128, 16, ragged=True),
        # one long sequence: the work split over the cache
        _attention("attention_long", 1, 1, 131072, 64, 8, 128, 64),
        # pieces of prompts on top of what is cached, windowed
        _attention("attention_prompt", 2, 1024, 4099, 64, 8, 128, 32, window=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    """(query heads, key/value heads): one rank's share up to all of them."""
    kv = rng.choice([1, 2, 4, 8])
    return kv * rng.choice([1, 2, 4, 5, 8, 16]), kv


def draw(rng):
    op = rng.choice(["linear", "append", "attention"])
    if op == "linear":
        while True:
            g = rng.choice([1, 1, 2, 4, 8])
            m, n, k = _log(rng, 1, 4096), _log(rng, 128, 16384), _log(rng, 128, 16384)
            if rng.random() < 0.5:
                n, k = max(64, n // 64 * 64), max(64, k // 64 * 64)
            # no more than the largest listed case: operations, operands and results
            if g * n * k <= 1 << 26 and g * m * (n + k) <= 1 << 26 and g * m * n * k <= 1 << 38:
                break
        c = _linear("", g, m, n, k, out=rng.choice(["bf16", "bf16", "f32"]),
                    act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), bias=rng.random() < 0.5,
                    residual=rng.random() < 0.5, root=rng.choice([-1, 0, g - 1]), shared=rng.random() < 0.5)
    elif op == "append":
        while True:
            hq, hkv = _heads(rng)
            d = rng.choice([64, 128, 128, 256])
            seqs, new = _log(rng, 1, 256), rng.choice([1, _log(rng, 1, 8192)])
            if seqs * new * (hq + 2 * hkv) * d <= 160 << 20 and seqs * new <= 16384:
                break
        ctx = _log(rng, 1, 8192) if seqs * hkv * d <= 1 << 14 else _log(rng, 1, 1024)
        c = _append("", seqs, new, ctx - 1, hq, hkv, d, rng.choice([16, 32, 64, 128]), rng.choice([d, d, d // 2, d // 4]),
                    interleaved=rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "f32"]), ragged=rng.random() < 0.6)
    else:
        while True:
            hq, hkv = _heads(rng)
            d = rng.choice([64, 128, 128, 256])
            seqs, new = _log(rng, 1, 128), rng.choice([1, 1, _log(rng, 1, 1024)])
            ctx = _log(rng, 1, 131072)
            cells = seqs * hkv * (ctx + new) * d
            if cells <= 1 << 27 and seqs * hq * new * (ctx + new) <= 1 << 29 and \
                    4 * seqs * hq * new * (ctx + new) * d <= 3 << 37:
                break
        c = _attention("", seqs, new, ctx - 1, hq, hkv, d, rng.choice([16, 32, 64, 128]),
                       window=rng.choice([0, 0, _log(rng, 1, 8192)]), ragged=rng.random() < 0.6)
    del c["name"]
    return c


def _spread(i, most):
    """A length between 1 and `most`: the longest for the first sequence, spread evenly over the range for the others."""
    return most if i == 0 else 1 + int((i * 0.6180339887498949 % 1.0) * (most - 1))


def _sequences(case):
    """(new tokens, total tokens) of every sequence."""
    got = []
    for i in range(case["seqs"]):
        new = _spread(i, case["new"]) if case["ragged"] else case["new"]
        ctx = (_spread(i + 1 if i else 0, case["ctx"]) if case["ragged"] and case["ctx"] > 0 else case["ctx"])
        got.append((new, ctx + new))
    if case["op"] == "attention" and case["ragged"] and case["new"] == 1 and case["seqs"] > 2:
        got[-1] = (1, 0)            # an idle slot of a decode batch: a row that sees no token
    return got


def work(case):
    if case["op"] == "linear":
        g, m, n, k = case["groups"], case["m"], case["n"], case["k"]
        wide = 4 if case["out"] == "f32" else 2
        added = g if case["root"] < 0 else 1
        return {"bytes": 2 * (g * n * k + (1 if case["shared"] else g) * m * k) + wide * g * m * n
                + (wide * added * m * n if case["residual"] else 0) + (2 * added * n if case["bias"] else 0),
                "flops": 2 * g * m * n * k}
    seqs, d, hq, hkv = _sequences(case), case["dim"], case["q_heads"], case["kv_heads"]
    tokens = sum(n for n, _ in seqs)
    entry = 2 * hkv * (d // 2 + 4 * (d // GROUP))           # a token's codes and words, keys and values
    if case["op"] == "append":
        wide = 4 if case["dtype"] == "f32" else 2
        return {"bytes": tokens * (wide * d * (2 * hq + 2 * hkv) + entry + 4 * case["rot"] + entry + 2 * wide * d * hkv),
                "flops": tokens * d * (3 * hq + 10 * hkv)}
    seen, read = 0, 0
    for new, total in seqs:
        window = case["window"] or total
        first = max(0, total - new - window + 1)
        read += max(0, total - first)
        # query i of the sequence sees min(window, total - new + i + 1) tokens
        a, b = total - new + 1, total
        whole = max(0, min(b, window) - max(a, 1) + 1)
        seen += whole * (max(a, 1) + min(b, window)) // 2 + window * max(0, b - max(window, a - 1)) if total else 0
    return {"bytes": read * entry + 2 * 2 * tokens * hq * d, "flops": 4 * d * hq * seen}


# ---------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------
def _quantise(x):
    """Codes (int32) and words (int32) of x [..., D] float32, by the rule at the top."""
    g = x.unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1).clamp(max=0.0), g.amax(-1).clamp(min=0.0)
    bits = (hi * _FIFTEENTH - lo * _FIFTEENTH).view(torch.int32) & ~15
    s = bits.view(torch.float32)
    some = s >= 2.0 ** -126
    inv = torch.where(some, 1.0 / s, 0.0)
    z = torch.round(-lo * inv)
    n = (torch.round(g * inv.unsqueeze(-1)) + z.unsqueeze(-1)).clamp(0, 15)
    words = torch.where(some, bits | z.to(torch.int32), 0)
    return n.to(torch.int32).flatten(-2), words


_FIFTEENTH = torch.tensor(1.0 / 15.0, dtype=torch.float32).item()


def _page_bytes(d, page):
    return page * d + 8 * page * (d // GROUP)


def _tables(case, gen):
    """Pages for every sequence in a shuffled pool: (pages in the pool, page table, lengths, token starts)."""
    seqs, page = _sequences(case), case["page"]
    width = max(1, max(-(-total // page) for _, total in seqs))
    pool = len(seqs) * width + 3
    table = torch.randperm(pool, generator=gen, device="cuda")[: len(seqs) * width].view(len(seqs), width).to(torch.int32)
    lengths = torch.tensor([t for _, t in seqs], dtype=torch.int32, device="cuda")
    starts = None
    if any(n != 1 for n, _ in seqs):
        starts = torch.tensor([0] + [n for n, _ in seqs], dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    return pool, table, lengths, starts


def _rotations(positions, rot, factor):
    """(cos, sin) of every position and pair, [positions][rot/2][2] float32, positions interpolated by `factor`."""
    inv = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * (inv / factor)
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16, scale=1.0):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)

    state = {"case": dict(case)}
    if case["op"] == "linear":
        g, m, n, k = case["groups"], case["m"], case["n"], case["k"]
        state["w"] = normal(g, n, k, scale=k ** -0.5)
        state["x"] = normal(1 if case["shared"] else g, m, k).expand(g, m, k)
        state["bias"] = normal(g, n) if case["bias"] else None
        state["residual"] = normal(g, m, n, dtype=DTYPES[case["out"]]) if case["residual"] else None
        return state
    d, hq, hkv, page = case["dim"], case["q_heads"], case["kv_heads"], case["page"]
    pool, state["page_table"], state["lengths"], state["token_start"] = _tables(case, gen)
    tokens = sum(n for n, _ in _sequences(case))
    if case["op"] == "append":
        dtype = DTYPES[case["dtype"]]
        state["pages"] = torch.zeros(pool, hkv, _page_bytes(d, page), dtype=torch.uint8, device="cuda")
        # one fused projection's result: queries, keys and values of a token side by side
        qkv = normal(tokens, hq + 2 * hkv, d, dtype=dtype)
        state["q"], state["k"], state["v"] = qkv.split([hq, hkv, hkv], 1)
        most = max(t for _, t in _sequences(case))
        state["rotations"] = _rotations(most, case["rot"], 4.0 if most > 4096 else 1.0)
        return state
    # a cache that earlier steps have filled: normal keys and values, quantised
    state["pages"] = torch.empty(pool, hkv, _page_bytes(d, page), dtype=torch.uint8, device="cuda")
    for p in range(0, pool, 1024):
        _fill(state["pages"][p:p + 1024], normal(min(1024, pool - p), hkv, 2, page, d, dtype=torch.float32), d, page)
    state["q"] = normal(tokens, hq, d)
    return state


def _fill(pages, kv, d, page):
    codes, words = _quantise(kv)
    pages[..., :page * d].copy_((codes[..., 0::2] | codes[..., 1::2] << 4).to(torch.uint8).flatten(2))
    pages[..., page * d:].copy_(words.flatten(2).contiguous().view(torch.uint8))


# ---------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state)


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


def _plain_linear(state):
    case, root = state["case"], state["case"]["root"]
    y = torch.matmul(state["x"].float(), state["w"].float().transpose(1, 2))
    at = slice(None) if root < 0 else slice(root, root + 1)
    if state["bias"] is not None:
        y[at] += state["bias"][at].float()[:, None]
    y = _activate(y, case["act"])
    if state["residual"] is not None:
        y[at] += state["residual"][at].float()
    return y.to(DTYPES[case["out"]])


def _places(state):
    """Sequence and position of every new token."""
    lengths, starts = state["lengths"].long(), state["token_start"]
    token = torch.arange(state["q"].shape[0], device="cuda")
    if starts is None:
        return token, lengths - 1
    seq = torch.searchsorted(starts[1:].long(), token, right=True)
    return seq, lengths[seq] - (starts.long()[seq + 1] - token)


def _rotate(x, cs, interleaved):
    """x [T][H][D] float32 with its first 2 * cs.shape[1] channels rotated."""
    rot = 2 * cs.shape[1]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _values(codes, words):
    """float32 values of packed codes [..., D/2] uint8 and words [..., D/64] int32."""
    n = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).unflatten(-1, (-1, GROUP)).to(torch.int32)
    s, z = (words & ~15).view(torch.float32), words & 15
    return ((n - z.unsqueeze(-1)).float() * s.unsqueeze(-1)).flatten(-2)


def _parts(pages, d, page):
    """The two regions of every page as [pool][heads][2][page][...]: packed codes (uint8) and words (int32)."""
    codes = pages[..., :page * d].unflatten(-1, (2, page, d // 2))
    words = pages[..., page * d:].view(torch.int32).unflatten(-1, (2, page, d // GROUP))
    return codes, words


def _plain_append(state):
    case = state["case"]
    d, page, dtype = case["dim"], case["page"], DTYPES[case["dtype"]]
    seq, position = _places(state)
    cs = state["rotations"][position]
    q = _rotate(state["q"].float(), cs, case["interleaved"])
    k = _rotate(state["k"].float(), cs, case["interleaved"])
    n, words = _quantise(torch.stack([k, state["v"].float()], 2))
    packed = (n[..., 0::2] | n[..., 1::2] << 4).to(torch.uint8)
    at, slot = state["page_table"][seq, position // page].long(), position % page
    codes_in, words_in = _parts(state["pages"], d, page)
    codes_in[at, :, :, slot] = packed
    words_in[at, :, :, slot] = words
    back = _values(codes_in[at, :, :, slot], words_in[at, :, :, slot]).to(dtype)
    return {"q": q.to(dtype), "k": back[:, :, 0], "v": back[:, :, 1]}


def _plain_attention(state):
    case = state["case"]
    d, page, hq, hkv = case["dim"], case["page"], case["q_heads"], case["kv_heads"]
    table, lengths = state["page_table"].long(), state["lengths"].long()
    seqs, most = case["seqs"], case["new"]
    codes, words = _parts(state["pages"], d, page)
    # every sequence's pages side by side: [seqs][heads][K or V][tokens][D]
    kv = _values(codes[table].permute(0, 2, 3, 1, 4, 5).flatten(3, 4), words[table].permute(0, 2, 3, 1, 4, 5).flatten(3, 4))
    seq, position = _places(state)
    row = torch.arange(len(seq), device="cuda") if state["token_start"] is None else state["token_start"].long()[seq]
    row = torch.arange(len(seq), device="cuda") - row
    q = torch.zeros(seqs, most, hq, d, device="cuda")
    at = torch.full((seqs, most), -1, dtype=torch.long, device="cuda")
    q[seq, row], at[seq, row] = state["q"].float(), position
    q = q.view(seqs, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).flatten(2, 3)
    scores = torch.matmul(q, kv[:, :, 0].transpose(2, 3)).unflatten(2, (hq // hkv, most)) * d ** -0.5
    token = torch.arange(kv.shape[3], device="cuda")
    seen = token <= at[:, :, None]
    if case["window"]:
        seen &= token > at[:, :, None] - case["window"]
    scores = scores.masked_fill(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0.0, 1.0, total)
    out = torch.matmul(p.flatten(2, 3), kv[:, :, 1]).unflatten(2, (hq // hkv, most))
    return out.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, row].to(torch.bfloat16)


_plain = {"linear": _plain_linear, "append": _plain_append, "attention": _plain_attention}

_context = None


def _kv():
    """The context of the cache operators that a program keeps for its stream."""
    global _context
    from paper_2607_16100_b200 import symar
    if _context is None:
        _context = symar.KVContext()
    return symar, _context


def _own_linear(state):
    from paper_2607_16100_b200 import symar
    case = state["case"]
    return symar.linear(state["x"], state["w"], bias=state["bias"], residual=state["residual"], act=case["act"],
                        root=case["root"], out_dtype=DTYPES[case["out"]])


def _own_append(state):
    symar, kv = _kv()
    case = state["case"]
    cache = symar.PagedKV(state["pages"], case["dim"], case["page"])
    batch = symar.KVBatch(state["lengths"], state["page_table"], state["token_start"])
    q = kv.append(cache, batch, state["k"], state["v"], q=state["q"], rotations=state["rotations"],
                  interleaved=case["interleaved"])
    k, v = kv.read(cache, batch, state["q"].shape[0], dtype=DTYPES[case["dtype"]])
    return {"q": q, "k": k, "v": v}


def _own_attention(state):
    symar, kv = _kv()
    case = state["case"]
    cache = symar.PagedKV(state["pages"], case["dim"], case["page"])
    batch = symar.KVBatch(state["lengths"], state["page_table"], state["token_start"])
    return kv.attention(cache, batch, state["q"], window=case["window"])


_own = {"linear": _own_linear, "append": _own_append, "attention": _own_attention}


# ---------------------------------------------------------------------------------
# the definitions in 64 bits, one sequence or matrix at a time
# ---------------------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "linear":
        got = []
        for g in range(case["groups"]):
            mine = case["root"] in (-1, g)
            y = state["x"][g].double() @ state["w"][g].double().T
            if state["bias"] is not None and mine:
                y = y + state["bias"][g].double()
            t = {"none": lambda v: v, "relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v),
                 "gelu": lambda v: v * 0.5 * torch.erfc(-v / math.sqrt(2.0)),
                 "gelu_tanh": lambda v: v * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))}
            y = t[case["act"]](y)
            got.append(y + state["residual"][g].double() if state["residual"] is not None and mine else y)
        return torch.stack(got)
    seqs, first = _sequences(case), 0
    if case["op"] == "append":
        q, k, v = [], [], []
        for new, total in seqs:
            rows = slice(first, first + new)
            turn = torch.view_as_complex(state["rotations"][total - new:total].double())[:, None]
            q.append(_exact_turn(state["q"][rows].double(), turn, case["interleaved"]))
            k.append(_exact_cached(_exact_turn(state["k"][rows].double(), turn, case["interleaved"])))
            v.append(_exact_cached(state["v"][rows].double()))
            first += new
        return {"q": torch.cat(q), "k": torch.cat(k), "v": torch.cat(v)}
    got, hkv, page, d = [], case["kv_heads"], case["page"], case["dim"]
    share = case["q_heads"] // hkv
    for b, (new, total) in enumerate(seqs):
        q = state["q"][first:first + new].double()
        first += new
        o = torch.zeros_like(q)
        if total:
            mine = state["pages"][state["page_table"][b, :-(-total // page)].long()]
            for h in range(hkv):
                kv = _exact_entries(mine[:, h], d, page)[:, :total]
                at = torch.arange(total - new, total, device="cuda")[:, None]
                token = torch.arange(total, device="cuda")
                hidden = (token > at) | (token <= at - (case["window"] or total))
                for j in range(h * share, (h + 1) * share):
                    logits = (q[:, j] @ kv[0].T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                    o[:, j] = torch.softmax(logits, -1) @ kv[1]
        got.append(o)
    return torch.cat(got)


def _exact_turn(x, turn, interleaved):
    half = turn.shape[-1]
    part, rest = x[..., :2 * half], x[..., 2 * half:]
    pairs = part.unflatten(-1, (half, 2)) if interleaved else part.unflatten(-1, (2, half)).transpose(-1, -2)
    pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    return torch.cat([(pairs if interleaved else pairs.transpose(-1, -2)).flatten(-2), rest], -1)


def _exact_cached(x):
    g = x.unflatten(-1, (-1, GROUP))
    lo = torch.minimum(g.min(-1, keepdim=True).values, torch.zeros((), dtype=g.dtype, device=g.device))
    hi = torch.maximum(g.max(-1, keepdim=True).values, torch.zeros((), dtype=g.dtype, device=g.device))
    s = (((hi - lo) / 15.0).float().view(torch.int32) & ~15).view(torch.float32).double()   # what a word can hold
    z = torch.round(-lo / s)
    return ((torch.clamp(torch.round(g / s) + z, 0, 15) - z) * s).flatten(-2)


def _exact_entries(pages, d, page):
    """[2][tokens][D] of one head's pages in order, from the bytes."""
    count = pages.shape[0]
    nibbles = torch.stack([pages[:, :page * d] % 16, pages[:, :page * d] // 16], -1).double()
    n = nibbles.view(count, 2, page, d // GROUP, GROUP)
    words = pages[:, page * d:].contiguous().view(torch.int32).view(count, 2, page, d // GROUP, 1)
    z = words % 16
    s = (words - z).view(torch.float32).double()
    return ((n - z) * s).transpose(0, 1).reshape(2, count * page, d)
