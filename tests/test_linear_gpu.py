"""symar_linear against the formula in 64 bits.

Two kinds of checks.  Small whole numbers: every product and sum is exact in binary32 in whatever order, so the result
has to be the exact value rounded once.  Real numbers: the bound below, from the roundings that the call is allowed.

Bound.  S = sum |x w|.  bf16 products are exact in binary32; an addition of the tensor cores truncates, at most 2^-23 of
the running sum each.  A float32 result adds chains of at most 128 products with IEEE additions (2^-24 each):
(min(k, 128) 2^-23 + ceil(k / 128) 2^-24) S; a bf16 result may be one chain: k 2^-23 S.  Bias, activation and residual add
a few roundings of 2^-24; |act'| < 1.13 for every activation.  The result is rounded once: 2^-8 (bf16) or 2^-24.
"""
import math

import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu

ACTS = {
    "none": lambda y: y,
    "relu": lambda y: y.clamp(min=0),
    "gelu": lambda y: 0.5 * y * torch.erfc(-y / math.sqrt(2)),
    "gelu_tanh": lambda y: 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))),
    "silu": lambda y: y * torch.sigmoid(y),
}


def reference(x, w, bias, residual, act, root, groups):
    got = []
    for g in range(groups):
        xg, wg = (t[g] if t.dim() == 3 else t for t in (x, w))
        y, s = xg.double() @ wg.double().T, xg.double().abs() @ wg.double().abs().T
        mine = root in (-1, g)
        if bias is not None and mine:
            b = (bias[g] if bias.dim() == 2 else bias).double()
            y, s = y + b, s + b.abs()
        r = 0.0
        if residual is not None and mine:
            r = (residual[g] if residual.dim() == 3 else residual).double()
        got.append((ACTS[act](y) + r, s))
    return torch.stack([a for a, _ in got]), torch.stack([b for _, b in got])


def check(got, x, w, bias=None, residual=None, act="none", root=-1):
    groups = got.shape[0] if got.dim() == 3 else 1
    k = x.shape[-1]
    want, s = reference(x, w, bias, residual, act, root, groups)
    chain = (min(k, 128) * 2.0 ** -23 + math.ceil(k / 128) * 2.0 ** -24) if got.dtype == torch.float32 else k * 2.0 ** -23
    tol = 1.13 * (chain + 8 * 2.0 ** -24) * s + (2.0 ** -24 if got.dtype == torch.float32 else 2.0 ** -8) * want.abs() + \
        8 * 2.0 ** -24 * want.abs() + 1e-37
    err = (got.double().view_as(want) - want).abs()
    assert torch.isfinite(got).all()
    assert (err <= tol).all(), (err / tol).max().item()


def normal(*shape, seed, scale=1.0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def whole(*shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-4, 5, shape, generator=g, device="cuda").to(torch.bfloat16)


SHAPES = [(1, 1, 1), (1, 128, 64), (1, 1024, 1024), (2, 7, 3), (3, 130, 72), (16, 256, 512), (17, 129, 1000), (33, 64, 4096),
          (64, 1000, 128), (65, 136, 200), (127, 128, 192), (129, 257, 65), (200, 384, 640), (256, 512, 256), (300, 520, 2056),
          (513, 1024, 1024), (1, 8192, 328), (31, 2049, 1031)]


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_whole_numbers_are_exact(m, n, k, out):
    x, w = whole(m, k, seed=m + n), whole(n, k, seed=k)
    got = symar.linear(x, w, out_dtype=out)
    want = x.double() @ w.double().T
    assert torch.equal(got, want.to(torch.float32).to(out))


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_real_numbers(m, n, k, out, act):
    x, w = normal(m, k, seed=m), normal(n, k, seed=n + 1, scale=k ** -0.5)
    bias, residual = normal(n, seed=5), normal(m, n, seed=6, dtype=out)
    got = symar.linear(x, w, bias=bias, residual=residual, act=act, out_dtype=out)
    check(got, x, w, bias, residual, act)


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_activations_over_their_range(act, out):
    # k = 1: the product is the argument itself, from the smallest to the largest that matters
    x = torch.cat([torch.linspace(-30, 30, 2001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e4, -1e4])]).cuda().bfloat16()[:, None]
    w = torch.ones(24, 1, device="cuda", dtype=torch.bfloat16)
    got = symar.linear(x, w, act=act, out_dtype=out)
    want = ACTS[act](x.double()).expand(-1, 24)
    # absolute: where the activation's value is far below its argument, 1 + erf or 1 + tanh keep 2^-24 of 1
    tol = (2.0 ** -8 if out == torch.bfloat16 else 8 * 2.0 ** -24) * want.abs() + 4 * 2.0 ** -24 * x.double().abs() + 1e-37
    assert ((got.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("groups,m,n,k,root", [(8, 4, 512, 128, 0), (8, 4, 512, 128, 7), (4, 33, 136, 320, -1), (2, 333, 123, 77, 1),
                                               (8, 1, 64, 1024, 3), (3, 200, 260, 520, 2)])
@pytest.mark.parametrize("shared", ["none", "x", "w"])
def test_ranks(groups, m, n, k, root, shared):
    x = normal(*(() if shared == "x" else (groups,)), m, k, seed=1)
    w = normal(*(() if shared == "w" else (groups,)), n, k, seed=2, scale=k ** -0.5)
    bias, residual = normal(groups, n, seed=3), normal(groups, m, n, seed=4)
    got = symar.linear(x, w, bias=bias, residual=residual, root=root)
    assert got.shape == (groups, m, n)
    check(got, x, w, bias, residual, root=root)


@pytest.mark.parametrize("m,n,k", [(5, 136, 200), (70, 264, 136), (150, 300, 520)])
@pytest.mark.parametrize("offset", [0, 1, 4, 8])
def test_strides_and_offsets(m, n, k, offset):
    """Operands and results inside larger tensors, at any alignment; nothing beside the result is written."""
    pad = 8 + offset
    xb, wb = normal(2, m, k + pad, seed=1), normal(2, n, k + pad, seed=2, scale=k ** -0.5)
    x, w = xb[:, :, offset:offset + k], wb[:, :, offset:offset + k]
    for dtype in (torch.bfloat16, torch.float32):
        room = torch.full((2, m, n + pad), 7.0, device="cuda", dtype=dtype)
        out = room[:, :, offset:offset + n]
        symar.linear(x, w, out=out)
        check(out, x, w)
        assert (room[:, :, :offset] == 7.0).all() and (room[:, :, offset + n:] == 7.0).all()
    # groups side by side in a token's row, as attention leaves its heads: [m][group][k]
    x = normal(m, 2, k, seed=3).transpose(0, 1)
    check(symar.linear(x, w), x, w)


def test_result_may_be_the_residual():
    x, w, r = normal(37, 520, seed=1), normal(260, 520, seed=2, scale=0.05), normal(37, 260, seed=3)
    want = symar.linear(x, w, residual=r)
    got = symar.linear(x, w, residual=r, out=r)
    assert got is r and torch.equal(got, want)


@pytest.mark.parametrize("m,n", [(3, 40), (200, 300)])
def test_nothing_to_sum(m, n):
    x, w = torch.empty(m, 0, device="cuda", dtype=torch.bfloat16), torch.empty(n, 0, device="cuda", dtype=torch.bfloat16)
    b, r = normal(n, seed=1), normal(m, n, seed=2)
    got = symar.linear(x, w, bias=b, residual=r, act="relu")
    want = (b.float().clamp(min=0)[None] + r.float()).bfloat16()
    assert torch.equal(got, want)


@pytest.mark.parametrize("m,n,k", [(4, 200, 256), (140, 300, 512)])
def test_values_that_are_not_finite_stay_in_their_row_and_column(m, n, k):
    x, w = whole(m, k, seed=1), whole(n, k, seed=2)
    w = torch.where(w == 0, torch.ones_like(w), w)
    x[1, 3], w[7, 5] = math.inf, math.nan
    got, want = symar.linear(x, w, out_dtype=torch.float32), x.double() @ w.double().T
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    fine = torch.isfinite(want)
    assert torch.equal(got[fine].double(), want[fine])


def test_two_calls_give_the_same_bits_and_a_graph_replays():
    x, w, b = normal(48, 4096, seed=1), normal(1024, 4096, seed=2, scale=1 / 64), normal(1024, seed=3)
    first = symar.linear(x, w, bias=b, act="silu")
    out = torch.empty_like(first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            symar.linear(x, w, bias=b, act="silu", out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)


def test_python_refusals():
    x, w = normal(4, 64, seed=1), normal(32, 64, seed=2)
    for bad in (dict(bias=x), dict(residual=x), dict(act="tanh"), dict(out=torch.empty(4, 31, device="cuda", dtype=torch.bfloat16)),
                dict(out=torch.empty(32, 4, device="cuda", dtype=torch.bfloat16).T), dict(out_dtype=torch.float16), dict(root=1)):
        with pytest.raises(symar.SymarError):
            symar.linear(x, w, **bad)
    for a, b in ((x.float(), w), (x, w[:, :32]), (x.cpu(), w), (x, w.T.contiguous().T)):
        with pytest.raises(symar.SymarError):
            symar.linear(a, b)
