"""symar_route against the definition in 64 bits.

Choices and lists are whole numbers and have to be equal.  Weights: a score takes the function's two units (2^-22), the rounding of logit - top
(at most 2^-24 times 90, where the score is not below 2^-130), at most 37 additions of a softmax's sum, a quotient, the sum over the chosen (5 additions), a
quotient and the scale: 180 x 2^-24 of the weight."""
import math

import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def normal(*shape, seed, scale=1.0, dtype=F32):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def reference(logits, top_k, bias, score, renormalise, scale):
    x = logits.double().cpu()
    x = torch.where(torch.isnan(x), -math.inf, x)
    tokens, experts = x.shape
    there = x > -math.inf
    s = torch.sigmoid(x) if score == "sigmoid" else torch.nan_to_num(torch.softmax(x, -1), nan=0.0)
    key = x if bias is None else torch.where(there, s + bias.double().cpu(), -math.inf)
    key = torch.where(torch.isnan(key), -math.inf, key)
    best = torch.sort(key, dim=1, descending=True, stable=True)
    some = best.values[:, :top_k] > -math.inf
    choice = torch.where(some, best.indices[:, :top_k], -1)
    w = torch.where(some, s.gather(1, best.indices[:, :top_k]), 0.0)
    if renormalise:
        w = torch.where(w.sum(-1, keepdim=True) > 0, w / w.sum(-1, keepdim=True), 0.0)
    lists = [[] for _ in range(experts)]
    for t, row in enumerate(choice.tolist()):
        for j, e in enumerate(row):
            if e >= 0:
                lists[e].append((t, j))
    flat = [tj for rows in lists for tj in rows]
    start = [0]
    for rows in lists:
        start.append(start[-1] + len(rows))
    row_token = torch.tensor([t for t, _ in flat] + [-1] * (tokens * top_k - len(flat)))
    token_row = torch.full((tokens, top_k), -1)
    for r, (t, j) in enumerate(flat):
        token_row[t, j] = r
    return choice, w * scale, torch.tensor(start), row_token, token_row


def check(logits, top_k, bias=None, score="softmax", renormalise=True, scale=1.0, **kw):
    choice, w, start, row_token, token_row = reference(logits, top_k, bias, score, renormalise, scale)
    r = symar.route(logits, top_k, bias=bias, score=score, renormalise=renormalise, scale=scale, **kw)
    for got, want in ((r.choice, choice), (r.expert_start, start), (r.row_token, row_token), (r.token_row, token_row)):
        assert got.dtype == torch.int32 and got.shape == want.shape and torch.equal(got.cpu().long(), want.long())
    assert ((r.weights.double().cpu() - w).abs() <= 180 * 2.0 ** -24 * w.abs() + 1e-37).all()
    return r


@pytest.mark.parametrize("experts", [1, 2, 7, 31, 32, 33, 60, 64, 65, 128, 200, 256, 257, 512, 513, 1000, 1024])
@pytest.mark.parametrize("tokens", [1, 5, 33, 128, 129, 700])
def test_sizes(tokens, experts):
    for i, top_k in enumerate({1, min(8, experts), min(32, experts)}):
        x = normal(tokens, experts, seed=experts + i, dtype=(F32, BF16)[i % 2])
        check(x, top_k)
        check(x, top_k, score="sigmoid", bias=normal(experts, seed=3, scale=0.1), renormalise=False, scale=2.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("renormalise", [False, True])
def test_kinds(score, biased, dtype, renormalise):
    x = normal(5000, 160, seed=1, scale=2.0, dtype=dtype)
    check(x, 6, normal(160, seed=2, scale=0.02) if biased else None, score, renormalise, 0.5)


@pytest.mark.parametrize("tokens", [40, 3000])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_equal_keys_and_keys_next_to_each_other(tokens, score):
    """Few different logits, and biases that undo the scores' differences up to the last bits."""
    x = (normal(tokens, 96, seed=1) * 2).round() / 2
    check(x, 8, score=score)
    check(x, 8, torch.zeros(96, device="cuda"), score)
    check(x, 8, (normal(96, seed=2) * 4).round() / 8, score)
    check(torch.zeros_like(x), 8, score=score)
    check(torch.where(x > 0, 0.0, -0.0), 8, score=score)
    y = normal(1, 96, seed=3).expand(tokens, 96) + normal(tokens, 96, seed=4, scale=1e-6)
    s = torch.sigmoid(y[0].double()) if score == "sigmoid" else torch.softmax(y[0].double(), -1)
    check(y, 8, (0.25 - s).float(), score)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,top_k", [(40, 32), (700, 32), (300, 8), (1024, 20)])
def test_many_choices_next_to_each_other(experts, top_k, score):
    """More equal and nearly equal keys than are looked at together, also all of a lane's."""
    x = (normal(60, experts, seed=1)).round()
    y = normal(1, experts, seed=3).expand(60, experts) + normal(60, experts, seed=4, scale=1e-6)
    s = torch.sigmoid(y[0].double()) if score == "sigmoid" else torch.softmax(y[0].double(), -1)
    z = torch.full((60, experts), -3.0, device="cuda")
    z[:, ::32] = normal(60, len(range(0, experts, 32)), seed=5)
    for logits, bias in ((x, None), (x, torch.zeros(experts, device="cuda")), (x, x[0] / 64), (y, (0.25 - s).float()), (y * 1e-3, None), (z, None), (z, x[0] / 64)):
        check(logits, top_k, bias, score)


def test_masked_experts_and_tokens():
    for tokens in (20, 1000):
        x = normal(tokens, 64, seed=1)
        x[3] = -math.inf
        x[7, 5:] = -math.inf
        x[8, 1::2] = math.nan
        x[9] = math.nan
        x[10, 2] = -1e38
        b = normal(64, seed=2, scale=0.1)
        b[11], b[12] = -math.inf, math.nan
        for score in ("softmax", "sigmoid"):
            r = check(x, 8, None, score)
            assert (r.choice[3] == -1).all() and (r.choice[7, 5:] == -1).all() and (r.weights[9] == 0).all()
            r = check(x, 8, b, score)
            assert not ((r.choice == 11) | (r.choice == 12)).any()
        r = check(torch.full_like(x, -math.inf), 4)
        assert (r.expert_start == 0).all() and (r.row_token == -1).all()


def test_sizes_of_values():
    x = normal(300, 64, seed=1, scale=30.0)
    check(x, 4), check(x, 4, score="sigmoid"), check(x * 1e36, 4, renormalise=False)
    x[:, 5] = math.inf
    r = symar.route(x, 4)
    assert (r.choice[:, 0] == 5).all() and torch.isnan(r.weights[:, 0]).all()


def test_strides_streams_and_graphs():
    wide = normal(900, 80, seed=1)
    for x in (wide[:, 3:67], wide[::2, 16:], wide[:1, :64].expand(400, 64)):
        check(x, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want = check(wide, 6)
    got = symar.route(wide, 6, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got.row_token, want.row_token)
    x = wide.clone()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            a = symar.route(x, 6)
            b = symar.route(x[:50], 2, score="sigmoid")
    for seed in (5, 6):
        x.copy_(normal(900, 80, seed=seed))
        graph.replay()
        torch.cuda.synchronize()
        for got, want in ((a, check(x, 6)), (b, check(x[:50], 2, score="sigmoid"))):
            assert all(torch.equal(getattr(got, f), getattr(want, f)) for f in ("choice", "weights", "expert_start", "row_token", "token_row"))


def test_no_tokens_and_refusals():
    r = symar.route(torch.empty(0, 16, device="cuda"), 4)
    assert (r.expert_start == 0).all() and r.choice.shape == (0, 4) and r.rows == 0
    x = normal(4, 16, seed=1)
    for bad in (lambda: symar.route(x, 0), lambda: symar.route(x, 17), lambda: symar.route(x.half(), 2), lambda: symar.route(x.cpu(), 2),
                lambda: symar.route(x.T, 2), lambda: symar.route(x[0], 2), lambda: symar.route(x, 2, score="relu"),
                lambda: symar.route(x, 2, bias=x[0, :8]), lambda: symar.route(x, 2, bias=x[0].bfloat16()), lambda: symar.route(x, 2, scale=math.nan),
                lambda: symar.Routes(r.choice, r.weights.double(), r.expert_start, r.row_token, r.token_row),
                lambda: symar.Routes(r.choice.long(), r.weights, r.expert_start, r.row_token, r.token_row),
                lambda: symar.Routes(r.choice, r.weights, r.expert_start[:0], r.row_token, r.token_row),
                lambda: symar.Routes(r.choice, r.weights.cpu(), r.expert_start, r.row_token, r.token_row)):
        with pytest.raises(symar.SymarError):
            bad()
    for x in (torch.zeros(2, 1025, device="cuda"), torch.zeros(2, 64, device="cuda")):
        with pytest.raises(symar.SymarError) as e:
            symar.route(x, 33)
        assert e.value.code == symar.ERR_UNSUPPORTED
