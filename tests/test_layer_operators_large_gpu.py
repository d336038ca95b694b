"""Norm, router, experts and combine where offsets pass 32 bits: the last rows of tensors of more than 2^31 elements, against the same rows alone."""
import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def normal(*shape, seed, dtype=BF16):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("n", [8192, 8193, 1000])
def test_norm(n):
    m = 2 ** 31 // n + 700
    x = torch.zeros(m, n, dtype=BF16, device="cuda")
    x[-5:], x[:3] = normal(5, n, seed=1), normal(3, n, seed=2)
    before = symar.Norm("rms", normal(n, seed=3))
    y, _ = symar.norm(x, before=before)
    assert torch.equal(y[-5:], symar.norm(x[-5:].clone(), before=before)[0]) and (y[1000:1010] == 0).all()
    # (a row's sums go by as many threads as the call has rows for; another order of them moves a rounding by a step at most)
    few = symar.norm(x[-700:].clone(), before=before)[0]
    assert torch.equal(y[-700:], few) or (y[-700:].double() - few.double()).abs().max() <= 2.0 ** -7 * few.double().abs().max()


def test_route():
    m = 2 ** 31 // 1000 + 90
    x = torch.zeros(m, 1000, dtype=BF16, device="cuda")
    x[-80:] = normal(80, 1000, seed=1)
    r, alone = symar.route(x, 2), symar.route(x[-80:].clone(), 2)
    assert torch.equal(r.choice[-80:], alone.choice) and torch.equal(r.weights[-80:], alone.weights)
    assert (r.choice[:-80] == torch.tensor([0, 1], dtype=torch.int32, device="cuda")).all() and int(r.expert_start[-1]) == 2 * m
    assert torch.equal(r.row_token[r.token_row[-80:].long()], torch.arange(m - 80, m, device="cuda", dtype=torch.int32)[:, None].expand(80, 2))


@pytest.mark.parametrize("out", [BF16, F32])
def test_experts_and_combine(out):
    tokens, n = 2 ** 31 // 4096 // 2 + 100, 4096
    logits = torch.zeros(tokens, 3, device="cuda")
    logits[:, 2] = -1
    r = symar.route(logits, 2)
    x, w = torch.zeros(tokens, 64, dtype=BF16, device="cuda"), torch.randint(-3, 4, (3, n, 64), device="cuda").to(BF16)
    x[-40:] = torch.randint(-3, 4, (40, 64), device="cuda").to(BF16)
    y = symar.experts(x, w, r, out_dtype=out)
    assert y.shape[0] == 2 * tokens and y.numel() > 2 ** 31
    want = torch.stack([x[-40:].double() @ w[e].double().T for e in (0, 1)], 1)          # [token][choice]
    assert torch.equal(y[r.token_row[-40:].long()].double(), want.float().to(out).double())
    z = symar.combine(y, r, out_dtype=F32)
    # (two logits of 0: weights of exactly a half, and halves of whole numbers are exact)
    assert torch.equal(z[-40:].double(), y[r.token_row[-40:].long()].double().mean(1)) and (z[:100] == 0).all()
