"""symar_linear where a multiprocessor has several tiles, one after the other: the accumulators in turn, results of a tile beside the next
tile's products, and more than sixteen tiles of tokens, which are gone through in bands.  Bound and checks are those of test_linear_gpu.py."""
import pytest
import torch

from paper_2607_16100_b200 import symar
from test_linear_gpu import check, normal, whole

pytestmark = pytest.mark.gpu

# m, n, k: tiles are 128 channels by 256 tokens (128 for float32 results and for rows on no 16-byte boundary)
SHAPES = [(1000, 12793, 72),              # 4 x 100 tiles, two slices of k each
          (4357, 1500, 64),               # 18 x 12, a second band of two; one slice
          (4357, 1500, 328), (2179, 1499, 201),               # the second on no boundary
          (1, 40000, 128), (20, 50001, 136), (100, 70000, 64),          # 313, 391 and 547 tiles of few tokens
          (8200, 300, 520)]               # 33 x 3 tiles in three bands


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_whole_numbers_are_exact(m, n, k, out):
    x, w = whole(m, k, seed=m + n), whole(n, k, seed=k)
    got = symar.linear(x, w, out_dtype=out)
    want = (x.double() @ w.double().T).to(torch.float32).to(out)
    assert torch.equal(got, want)
    assert torch.equal(got, symar.linear(x, w, out_dtype=out))


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(1000, 12793, 72), (2179, 1499, 201), (4357, 1500, 328)])
def test_bias_activation_and_residual(m, n, k, out):
    x, w = normal(m, k, seed=m), normal(n, k, seed=n + 1, scale=k ** -0.5)
    bias, residual = normal(n, seed=5), normal(m, n, seed=6, dtype=out)
    for act in ("none", "gelu_tanh"):
        check(symar.linear(x, w, bias=bias, residual=residual, act=act, out_dtype=out), x, w, bias, residual, act)


@pytest.mark.parametrize("groups,m,n,k", [(5, 4, 8192, 64), (3, 300, 5000, 136), (2, 2179, 1000, 77)])
@pytest.mark.parametrize("root", [-1, 1])
def test_ranks(groups, m, n, k, root):
    x, w = normal(groups, m, k, seed=1), normal(groups, n, k, seed=2, scale=k ** -0.5)
    bias, residual = normal(groups, n, seed=3), normal(groups, m, n, seed=4)
    check(symar.linear(x, w, bias=bias, residual=residual, act="silu", root=root), x, w, bias, residual, "silu", root)
