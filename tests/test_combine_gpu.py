"""symar_combine against the formula in 64 bits.  Bound: top_k products and additions in binary32 and one for the residual, a rounding of 2^-24 of the
terms' sizes each, and half a step of the result."""
import math

import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def normal(*shape, seed, scale=1.0, dtype=BF16):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def routes_of(tokens, experts, top_k, seed=0, idle=()):
    x = normal(tokens, experts, seed=seed, dtype=F32)
    for t in idle:
        x[t] = -math.inf
    return symar.route(x, top_k)


def check(y, routes, residual=None, root=-1, **kw):
    ranks, n = (y.shape[0] if y.dim() == 3 else 1), y.shape[-1]
    at, w = routes.token_row.long(), routes.weights.double()
    on = (at >= 0) & (at < routes.rows)
    want = torch.zeros(ranks, routes.tokens, n, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    for g in range(ranks):
        rows = (y[g] if y.dim() == 3 else y).double()
        if routes.rows:
            terms = torch.where(on[..., None], rows[at.clamp(0, routes.rows - 1)] * w[..., None], 0.0)
            want[g], size[g] = terms.sum(1), terms.abs().sum(1)
        if residual is not None and root in (-1, g):
            r = (residual[g] if residual.dim() == 3 else residual).double()
            want[g], size[g] = want[g] + r, size[g] + r.abs()
    got = symar.combine(y, routes, residual=residual, root=root, **kw)
    assert got.shape == (want.shape if y.dim() == 3 else want.shape[1:])
    half = 2.0 ** -8 if got.dtype == BF16 else 2.0 ** -24
    tol = half * want.abs() + (2 * routes.top_k + 2) * 2.0 ** -24 * (1 + half) * size + 1e-37
    assert ((got.double().view_as(want) - want).abs() <= tol).all()
    return got


@pytest.mark.parametrize("n", [1, 8, 63, 64, 100, 136, 1000, 2049, 2056, 5000])
@pytest.mark.parametrize("tokens,top_k", [(1, 1), (1, 8), (7, 3), (40, 9), (300, 2)])
def test_sizes(n, tokens, top_k):
    r = routes_of(tokens, 16, top_k, idle=(0,) if tokens > 5 else ())
    for y_type, out_type in ((BF16, BF16), (BF16, F32), (F32, BF16)):
        check(normal(r.rows, n, seed=1, dtype=y_type), r, out_dtype=out_type)
        check(normal(3, r.rows, n, seed=1, dtype=y_type), r, normal(tokens, n, seed=2, dtype=out_type), root=1, out_dtype=out_type)


@pytest.mark.parametrize("offset", [0, 1, 4, 8])
def test_strides(offset):
    r = routes_of(21, 8, 2)
    y = normal(2, r.rows, 150, seed=1)[..., offset:offset + 128]
    room = torch.full((21, 2, 150), 7.0, dtype=BF16, device="cuda")
    out = room[..., offset:offset + 128].transpose(0, 1)
    res = normal(2, 21, 150, seed=3)[..., offset:offset + 128]
    want = check(y, r, res, out=out)
    assert want is out and (room[..., :offset] == 7).all() and (room[..., offset + 128:] == 7).all()
    plain = symar.combine(y, r, residual=res)
    assert torch.equal(plain, out)
    assert torch.equal(symar.combine(y, r, residual=res, out=res), plain)          # the result in the residual's place
    shared = normal(r.rows, 64, seed=5).expand(4, r.rows, 64)
    check(shared, r, normal(21, 64, seed=6), root=3)


def test_rows_that_are_none():
    """What stands in rows of nobody, and weights of rows that are none, do not reach a result."""
    r = routes_of(6, 4, 2, idle=(1, 4))
    y = normal(r.rows, 72, seed=1)
    y[int(r.expert_start[-1]):] = math.nan
    r.weights[1], r.weights[4] = math.nan, math.inf
    got = check(y, r)
    assert (got[1] == 0).all() and (got[4] == 0).all()
    r.token_row[0, 0], r.token_row[2, 1] = r.rows, 2 ** 31 - 1
    check(y, r)
    empty = symar.route(torch.empty(0, 4, device="cuda"), 2)
    assert symar.combine(torch.empty(0, 72, device="cuda"), empty).shape == (0, 72)


def test_no_weights(lib=None):
    """At the library's boundary weights may be left out: they count as 1."""
    import ctypes
    r = routes_of(5, 4, 2)
    y, out = normal(r.rows, 40, seed=1), torch.empty(5, 40, device="cuda", dtype=F32)
    a = symar.CombineArgs(y=y.data_ptr(), y_ld=40, y_group=0, token_row=r.token_row.data_ptr(), out=out.data_ptr(), out_ld=40, out_group=0, groups=1,
                          tokens=5, top_k=2, rows=r.rows, n=40, dtype=symar.BF16, out_dtype=symar.F32, root=-1)
    assert symar.load().symar_combine(ctypes.byref(a), None) == symar.OK
    torch.cuda.synchronize()
    assert torch.equal(out, y[r.token_row.long()].float().sum(1))


def test_refusals():
    r = routes_of(6, 4, 2)
    y = normal(r.rows, 64, seed=1)
    for bad in (lambda: symar.combine(y[:-1], r), lambda: symar.combine(y.cpu(), r), lambda: symar.combine(y.half(), r), lambda: symar.combine(y[0], r),
                lambda: symar.combine(y.T.contiguous().T, r), lambda: symar.combine(y, r, out=y[:5]), lambda: symar.combine(y, r, residual=y[:6].float()),
                lambda: symar.combine(y, r, root=1), lambda: symar.combine(y, r, root=-2), lambda: symar.combine(y, r, out_dtype=torch.float16),
                lambda: symar.combine(y, r, out=torch.empty(1, 64, device="cuda", dtype=BF16).expand(6, 64))):
        with pytest.raises(symar.SymarError):
            bad()
