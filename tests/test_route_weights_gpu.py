"""Weights of symar_route whose scores pass binary32's range, against logarithms in 64 bits: the scores' quotients are ordinary numbers.

Bound: that of test_route_gpu.py (180 x 2^-24 of the weight), and what binary32 has no smaller numbers for: 2^-149."""
import math

import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def check(x, top_k, bias=None, score="sigmoid", renormalise=True, scale=1.0):
    r = symar.route(x, top_k, bias=bias, score=score, renormalise=renormalise, scale=scale)
    l = x.double()
    log = torch.nn.functional.logsigmoid(l) if score == "sigmoid" else torch.log_softmax(l, -1)
    some = r.choice >= 0
    log = torch.where(some, log.gather(1, r.choice.clamp(min=0).long()), -math.inf)
    want = torch.nan_to_num(torch.softmax(log, -1), nan=0.0) if renormalise else log.exp()
    want = want * scale
    err = (r.weights.double() - want).abs()
    assert torch.isfinite(r.weights).all()
    assert (err <= 180 * 2.0 ** -24 * want.abs() + 2.0 ** -149).all(), (r.weights[err.argmax() // top_k], want[err.argmax() // top_k])
    return r


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens", [7, 300])
@pytest.mark.parametrize("low", [-60.0, -80.0, -86.5, -88.0, -90.0, -100.0, -104.0, -150.0, -700.0, -800.0, -1e4, -1e30])
def test_far_logits(low, tokens, dtype):
    """All of a token's logits far below zero, next to each other, with one that is not, and with idle experts."""
    g = torch.Generator("cuda").manual_seed(1)
    x = low + torch.randn(tokens, 96, generator=g, device="cuda") * 3
    x[::3, 5::2] = -math.inf
    x[1::5] = -math.inf
    x = x.to(dtype)
    for top_k in (1, 4, 8):
        r = check(x, top_k)
        assert ((r.weights.sum(-1) - 1).abs()[(r.choice >= 0).any(-1)] < 1e-6).all()
        check(x, top_k, scale=-2.5), check(x, top_k, score="softmax"), check(x, top_k, renormalise=False)
    y = x.clone()
    y[:, 7], y[:, 40] = 2.0, -1.0
    check(y, 8), check(y, 8, score="softmax"), check(y, 8, renormalise=False), check(y, 8, score="softmax", renormalise=False)
    if low >= -104:
        check(x, 4, renormalise=False, scale=1e30)


@pytest.mark.parametrize("low", [-30.0, -80.0, -120.0, -900.0])
def test_choices_by_bias_far_below_the_largest(low):
    """A softmax's chosen experts need not be near its largest one where a bias decides."""
    g = torch.Generator("cuda").manual_seed(2)
    x = low + torch.randn(200, 64, generator=g, device="cuda")
    x[:, 3] = 0.0
    bias = torch.rand(64, generator=g, device="cuda")
    bias[3] = -5.0
    for score in ("softmax", "sigmoid"):
        r = check(x, 4, bias, score)
        assert not (r.choice == 3).any() and (r.choice >= 0).all() and ((r.weights.sum(-1) - 1).abs() < 1e-6).all()


def test_ordinary_weights():
    """Scores well inside binary32's range; the only choice of a token weighs exactly 1."""
    x = torch.randn(500, 64, generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    r = check(x, 1)
    assert (r.weights == 1).all()
    check(x * 4, 6), check(x * 4, 6, score="softmax")
