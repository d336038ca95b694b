"""symar_norm against the formula in 64 bits.

Bound.  e = 2^-24.  A thread adds up at most 32 elements, then 10 additions join a row's threads: a sum is off by at most 42 e of the sum of its
terms' sizes.  So a mean is off by 42 e mean|v|, what is left after it by 43 e max|v|; the root of a mean of squares by (42 + 4) / 2 + 2 e of
itself, twice 43 e max|v| / rms more where a mean was taken; weight, bias, gate, scale and residual add a rounding each, the gate's function four.  Per norm
that is below 160 e of the row's largest element before weights (max|v| is at least rms), and what enters the second norm carries the first one's.
Together: 400 e times the row's largest size on the way (the sum of the sizes of what was added, so that a small difference of large terms
counts as large), plus half a step of the result."""
import math

import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
E = 400 * 2.0 ** -24


def normal(*shape, seed, scale=1.0, dtype=BF16):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def side(v, size, s):
    """(value, size that the bound counts) of a norm, by the formula."""
    if s is None:
        return v, size
    kind, w, b, eps, plus = s
    w = torch.ones(v.shape[-1], device="cuda").double() if w is None else w.double() + plus
    b = 0.0 if b is None else b.double()
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
        size = size + size.mean(-1, keepdim=True)
    by = 1 / (v.square().mean(-1, keepdim=True) + eps).sqrt()
    # the size of the row's largest element, as an error there reaches every element through the factor
    size = (size.amax(-1, keepdim=True) * by) * (1 + v.abs() * by) * w.abs()
    return v * by * w + b, size + abs(b)


def reference(x, residual, after, before, gate, gate_act, scale, residual_scale):
    a, size = side(x.double(), x.double().abs(), after)
    if gate is not None:
        g = {"none": lambda t: t, "sigmoid": torch.sigmoid, "tanh": torch.tanh}[gate_act](gate.double())
        a, size = a * g, size * g.abs()
    r, size = scale * a, abs(scale) * size
    if residual is not None:
        r, size = r + residual_scale * residual.double(), size + abs(residual_scale) * residual.double().abs()
    y, ysize = side(r, size, before) if before else (None, None)
    return y, ysize, r, size


def close(got, want, size):
    half = 2.0 ** -8 if got.dtype == BF16 else 2.0 ** -24
    tol = half * want.abs() + E * (1 + half) * size + 1e-37
    assert got.shape == want.shape and torch.isfinite(got).all()
    assert ((got.double() - want).abs() <= tol).all(), ((got.double() - want).abs() / tol).max().item()


def check(x, residual=None, after=None, before=None, gate=None, gate_act="none", scale=1.0, residual_scale=1.0, **kw):
    make = lambda s: None if s is None else symar.Norm(s[0], s[1], s[2], eps=s[3], plus_one=bool(s[4]))      # noqa: E731
    y, ysize, r, size = reference(x, residual, after, before, gate, gate_act, scale, residual_scale)       # (before it is overwritten)
    got, got_r = symar.norm(x, residual, after=make(after), before=make(before), gate=gate, gate_act=gate_act, scale=scale,
                            residual_scale=residual_scale, **kw)
    assert (got is None) == (before is None)
    if got is not None:
        assert got.dtype == x.dtype
        close(got, y, ysize)
    assert (got_r is None) == (residual is None and before is not None and kw.get("residual_out") is None)
    if got_r is not None:
        close(got_r, r, size)
    return got, got_r


SIZES = [1, 2, 7, 8, 9, 64, 128, 250, 256, 257, 264, 1000, 1024, 1025, 1032, 1535, 1999, 2049, 2700, 3333, 3583, 4095, 4096, 4100, 4104, 8192, 8200, 11111, 16384, 16392, 32767, 32768]


@pytest.mark.parametrize("n", SIZES)
@pytest.mark.parametrize("rows", [1, 3, 300, 700])
def test_sizes(n, rows):
    x, res, w, w2 = normal(rows, n, seed=n), normal(rows, n, seed=1, scale=3), normal(n, seed=2), normal(n, seed=3, dtype=F32)
    check(x, res, before=("rms", w, None, 1e-6, 0))
    check(x, res, after=("rms", w2, None, 1e-5, 1), before=("layer", w, normal(n, seed=4), 1e-5, 0), scale=0.5, residual_scale=1.25)


@pytest.mark.parametrize("xt", [BF16, F32])
@pytest.mark.parametrize("st", [BF16, F32])
@pytest.mark.parametrize("gate", [None, "channel", "row", "all", "one"])
@pytest.mark.parametrize("m,n", [(5, 136), (5, 517), (5, 3080), (700, 64), (613, 120), (1200, 256), (777, 136), (601, 300), (999, 1000), (599, 1032),
                                 (1500, 2056), (650, 6400), (600, 9000), (594, 16384)])
def test_types_gates_and_kinds(xt, st, gate, m, n):
    x, res = normal(m, n, seed=1, dtype=xt), normal(m, n, seed=2, dtype=st)
    g = {None: None, "channel": (n,), "row": (m, 1), "all": (m, n), "one": ()}[gate]
    g = normal(*g, seed=3, dtype=xt) if g is not None else None
    w, b = normal(n, seed=4, dtype=st), normal(n, seed=5, dtype=st)
    for act in ("none", "sigmoid", "tanh"):
        for after, before in ((None, "rms"), ("rms", None), ("layer", "rms"), ("rms", "layer"), (None, None)):
            check(x, res, after and (after, w, b, 1e-5, 0), before and (before, w, None, 1e-5, 1), g, act, 0.7, -1.5)
            check(x, None, after and (after, None, b, 1e-5, 0), before and (before, None, None, 1e-5, 0), g, act)


def test_a_large_mean_costs_no_digits():
    x = normal(40, 4096, seed=1, dtype=F32) + 1000.0
    check(x, before=("layer", None, None, 1e-5, 0))
    got, _ = symar.norm(x, before=symar.Norm("layer", eps=0.0))
    v = x.double() - x.double().mean(-1, keepdim=True)
    assert (got.double() - v / v.square().mean(-1, keepdim=True).sqrt()).abs().max() < 43 * 2.0 ** -24 * 1004 * 2


@pytest.mark.parametrize("offset", [0, 1, 4, 8])
@pytest.mark.parametrize("n", [128, 1000, 2049])
def test_strides_groups_and_offsets(offset, n):
    """Rows inside wider ones; nothing beside the results is written."""
    for dtype in (BF16, F32):
        room = [normal(3, 6, n + 16, seed=s, dtype=dtype)[..., offset:offset + n] for s in range(2)]
        outs = [torch.full((3, 6, n + 16), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
        views = [o[..., offset:offset + n] for o in outs]
        w = normal(n + 16, seed=5)[offset:offset + n]
        check(room[0], room[1], before=("rms", w, None, 1e-6, 0), out=views[0], residual_out=views[1])
        check(room[0].transpose(0, 1), room[1].transpose(0, 1), after=("layer", w, None, 1e-6, 0), before=("rms", None, None, 1e-6, 0),
              gate=normal(1, 3, 1, seed=6, dtype=dtype), out=views[0].transpose(0, 1), residual_out=views[1].transpose(0, 1))
        for o in outs:
            assert (o[..., :offset] == 7).all() and (o[..., offset + n:] == 7).all()
    # heads of a fused projection's result, and one row for all
    qkv = normal(7, 5 * n, seed=9).view(7, 5, n)
    check(qkv[:, 1:4], before=("rms", None, None, 1e-6, 0))
    check(qkv[:1, :1].expand(7, 3, n), qkv[:, 1:4], before=("rms", None, None, 1e-6, 0))


def test_results_may_be_the_operands():
    for m, n in ((9, 256), (9, 1000), (9, 2049), (9, 8192), (1801, 128), (703, 1024), (1203, 2048), (601, 2050), (599, 8192)):
        x, res, w = normal(m, n, seed=1), normal(m, n, seed=2, dtype=F32), normal(n, seed=3)
        y, r = symar.norm(x, res, before=symar.Norm("rms", w))
        a, b = x.clone(), res.clone()
        got = symar.norm(a, b, before=symar.Norm("rms", w), out=a, residual_out=b)
        assert got[0] is a and got[1] is b and torch.equal(a, y) and torch.equal(b, r)


def test_zeros_and_values_that_are_not_finite():
    x = normal(4, 640, seed=1, dtype=F32)
    x[0] = 0
    x[1, 7], x[2, 9] = math.nan, math.inf
    y, _ = symar.norm(x, before=symar.Norm("rms", eps=1e-6))
    assert (y[0] == 0).all() and torch.isnan(y[1]).all() and torch.isnan(y[2, 9]) and (y[2, :9] == 0).all()
    close(y[3], x[3].double() / (x[3].double().square().mean() + 1e-6).sqrt(), 10 * x[3].abs().max().double())
    y, _ = symar.norm(x, before=symar.Norm("layer", eps=0.0))
    assert torch.isnan(y[:3]).all() and torch.isfinite(y[3]).all()


def test_nothing_to_do_and_refusals():
    for shape in ((0, 64), (3, 0), (0, 3, 64), (2, 0, 64)):
        x = torch.empty(shape, device="cuda", dtype=BF16)
        y, r = symar.norm(x, x, before=symar.Norm())
        assert y.shape == shape and r.shape == shape
    x, w = normal(4, 64, seed=1), normal(64, seed=2)
    n = symar.Norm("rms", w)
    for kw in (dict(residual=x[:, :32]), dict(gate=w.float()), dict(gate=w[:32]), dict(out=x[:2]), dict(gate_act="relu"), dict(residual_out=x.float(), residual=x),
               dict(before=None, out=x), dict(out=x.float()), dict(residual=x.cpu()), dict(gate=x[:, ::2].repeat(1, 2).T), dict(scale=math.nan), dict(scale=1e39), dict(residual_scale=None),
               dict(out=torch.empty(1, 64, device="cuda", dtype=BF16).expand(4, 64))):
        with pytest.raises(symar.SymarError):
            symar.norm(x, **{"before": n, **kw})
    for bad in (x.cpu(), x.half(), x[0], x.T, x[:, :32], x[None, None]):
        with pytest.raises(symar.SymarError):
            symar.norm(bad, before=n)
    with pytest.raises(symar.SymarError) as e:
        symar.norm(torch.empty(1, 32769, device="cuda"), before=symar.Norm())
    assert e.value.code == symar.ERR_UNSUPPORTED
    for bad in (lambda: symar.Norm("batch"), lambda: symar.Norm("rms", w.cpu()), lambda: symar.Norm("rms", w, w[:3]), lambda: symar.Norm("rms", w, w.float()),
                lambda: symar.Norm("rms", w[::2]), lambda: symar.Norm("rms", x)):
        with pytest.raises(symar.SymarError):
            bad()


def test_a_graph_replays_the_same_bits():
    x, res, w = normal(64, 4096, seed=1), normal(64, 4096, seed=2), normal(4096, seed=3)
    n = symar.Norm("rms", w)
    y, r = symar.norm(x, res, after=n, before=n)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            y2, r2 = symar.norm(x, res, after=n, before=n)
            y3, r3 = symar.norm(y2, r2, before=n)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y2, y) and torch.equal(r2, r)
        want = symar.norm(y, r, before=n)
        assert torch.equal(y3, want[0]) and torch.equal(r3, want[1])
    assert torch.equal(symar.norm(x, res, after=n, before=n, stream=s.cuda_stream)[0], y)
