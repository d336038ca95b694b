"""symar_route where the last choice has an equal behind it and a larger one behind that: keys that binary32, or the bits that an expert's place takes,
cannot tell apart, at the border of a token's choices."""
import math

import pytest
import torch

from test_route_gpu import BF16, F32, check

pytestmark = pytest.mark.gpu


def drawn(*shape, seed, below):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, below, shape, generator=g).float().cuda()


@pytest.mark.parametrize("experts", [33, 64, 100, 128, 256, 500, 512, 1000, 1024])
@pytest.mark.parametrize("top_k", [1, 2, 8])
def test_a_unit_above_two_equal_logits(experts, top_k):
    """Two equal logits in the lowest place, a third one unit in the last place above them wherever a lane can have it."""
    one, above = 1.0, 1.0 + 2.0 ** -23
    places = list(range(32, experts))
    x = torch.full((len(places), experts), -10.0, device="cuda")
    x[:, 2:2 + top_k - 1] = 10.0 + torch.arange(top_k - 1, device="cuda")
    free = [e for e in (0, 1, 20, 21)][:2]
    x[:, free] = one
    for t, e in enumerate(places):
        x[t, e] = above
    r = check(x, top_k)
    assert r.choice[:, top_k - 1].tolist() == places
    r = check(-x.flip(1).contiguous(), top_k)
    # more equal ones than a token has choices, some in every place
    x[:, ::3] = torch.where(x[:, ::3] < 0, one, x[:, ::3])
    check(x, top_k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("experts", [3, 31, 64, 100, 256, 512, 1000])
@pytest.mark.parametrize("top_k", [1, 2, 8])
def test_scores_that_binary32_rounds_to_one(experts, dtype, top_k):
    """Sigmoid and a bias of zeros, as a router starts: scores of logits from 16 on are 1 in binary32, and not in exact arithmetic."""
    if top_k > experts:
        pytest.skip("as many choices as experts at most")
    zeros = torch.zeros(experts, device="cuda")
    x = torch.full((1, experts), -3.0, device="cuda")
    x[0, :3] = torch.tensor([20.0, 20.0, 20.125])
    check(x.to(dtype), top_k, zeros, "sigmoid")
    high = 16 + drawn(700, experts, seed=experts, below=40) / 8
    for share in (2, 5, 30, 2 * experts):                            # saturated ones among others
        some = drawn(700, experts, seed=share, below=experts) < share
        check(torch.where(some, high, -high / 8).to(dtype), top_k, zeros, "sigmoid")
        check(torch.where(some, high, -high / 8).to(dtype), top_k, zeros + 0.375, "sigmoid", False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("experts", [31, 64, 100, 256, 1000])
@pytest.mark.parametrize("top_k", [1, 2, 8])
def test_scores_that_a_bias_swallows(experts, dtype, top_k):
    """Softmax and one bias for all: small scores differ by less than a unit of the sum."""
    x = (-drawn(700, experts, seed=experts, below=80) / 8).to(dtype)
    check(x, top_k, torch.full((experts,), 8.0, device="cuda"))
    check(x, top_k, torch.full((experts,), -0.25, device="cuda"), "softmax", False, 1.5)
    x[:, ::2] = -math.inf
    check(x, min(top_k, experts // 2), torch.full((experts,), 8.0, device="cuda"))


@pytest.mark.parametrize("experts", [20, 64, 200, 256, 300, 1024])
def test_all_equal(experts):
    for value in (0.0, -2.5):
        x = torch.full((90, experts), value, device="cuda")
        for top_k in (1, 8):
            for bias in (None, torch.zeros(experts, device="cuda")):
                for score in ("softmax", "sigmoid"):
                    r = check(x, top_k, bias, score)
                    assert (r.choice == torch.arange(top_k, device="cuda")).all()
