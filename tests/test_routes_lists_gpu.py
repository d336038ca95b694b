"""symar.Routes of lists that a program made go by them as they are when a call takes them: they may have other memory by then."""
import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu


def normal(*shape, seed, dtype=torch.bfloat16):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def test_lists_with_other_memory():
    x, y, w = normal(2, 64, seed=4), normal(4, 64, seed=1), normal(2, 16, 64, seed=2)
    start, row = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda")
    choice, weights = torch.tensor([[0, 1], [0, 1]], dtype=torch.int32, device="cuda"), torch.ones(2, 2, device="cuda")
    token_row, row_token = torch.tensor([[0, 2], [1, 3]], dtype=torch.int32, device="cuda"), row % 2
    kept = token_row.data, weights.data, row_token.data, start.data
    r = symar.Routes(choice, weights, start, row_token, token_row)
    want = symar.experts(x, w, r)
    assert torch.equal(symar.combine(y, r, out_dtype=torch.float32), y[:2].float() + y[2:].float())
    token_row.data, weights.data = token_row.flip(0).contiguous(), weights * 2
    assert torch.equal(symar.combine(y, r, out_dtype=torch.float32), 2 * (y[:2].float() + y[2:].float()).flip(0))
    row_token.data = 1 - row_token
    assert torch.equal(symar.experts(x, w, r), want[[1, 0, 3, 2]])
    start.data = torch.tensor([0, 0, 4], dtype=torch.int32, device="cuda")
    assert torch.equal(symar.experts(x, w, r)[2:], want[[3, 2]])
    assert torch.equal(symar.experts(y, w, r, by_row=True), symar.linear(y, w[1]))
    r.weights.data = torch.ones(1, 2, device="cuda")
    with pytest.raises(symar.SymarError):
        symar.combine(y, r)
    del kept


def test_lists_of_the_router_with_other_memory():
    r = symar.route(normal(6, 8, seed=1, dtype=torch.float32), 2)
    y = normal(r.rows, 32, seed=2)
    first = symar.combine(y, r, out_dtype=torch.float32)             # (before any list was asked for)
    kept = r.weights.data
    r.weights.data = r.weights * 4
    assert torch.equal(symar.combine(y, r, out_dtype=torch.float32), 4 * first)
    r.weights.mul_(0.25)
    assert torch.equal(symar.combine(y, r, out_dtype=torch.float32), first)
    del kept
