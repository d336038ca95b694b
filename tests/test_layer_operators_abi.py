"""Norm, router, experts and combine: what the library refuses on the host, so none of this needs a GPU."""
import ctypes
import math

import pytest

from paper_2607_16100_b200 import build, symar

SOME = 1 << 20          # an aligned address that is never touched


@pytest.fixture(scope="module")
def lib():
    build.build_lib()
    return symar.load()


def ids(c):
    return ",".join(f"{k}={v}" for k, v in c.items())


def norm_rc(lib, after=None, before=None, **change):
    f = {n + s: v for n in ("x", "residual", "residual_out", "out") for s, v in (("", SOME), ("_ld", 64), ("_group", 256))}
    f.update(gate=SOME, gate_ld=0, gate_group=0, gate_step=1, gate_act=0, groups=2, m=4, n=64, dtype=symar.BF16, stream_dtype=symar.F32, scale=1.0,
             residual_scale=1.0)
    s = dict(weight=SOME, bias=SOME, eps=1e-6, kind=1, dtype=symar.BF16, plus_one=0)
    f.update(after=symar.NormSide(**{**s, **(after or {})}), before=symar.NormSide(**{**s, **(before or {})}))
    f.update(change)
    return lib.symar_norm(ctypes.byref(symar.NormArgs(**f)), None)


@pytest.mark.parametrize("change", [
    dict(x=None), dict(out=None), dict(m=-1), dict(n=-1), dict(groups=-1), dict(dtype=2), dict(stream_dtype=-1), dict(x=SOME + 1), dict(gate=SOME + 1),
    dict(residual=SOME + 2), dict(residual_out=SOME + 2), dict(out=SOME + 1), dict(gate_act=3), dict(gate_act=-1), dict(gate_step=2), dict(x_ld=-1),
    dict(x_group=-1), dict(residual_ld=-1), dict(gate_ld=-1), dict(gate_group=-1), dict(out_ld=63), dict(out_group=0), dict(out_group=255),
    dict(residual_out_ld=0), dict(residual_out_group=32), dict(scale=math.nan), dict(scale=math.inf), dict(residual_scale=-math.inf),
    dict(after=dict(kind=3)), dict(before=dict(kind=-1)), dict(before=dict(kind=0)), dict(after=dict(eps=-1.0)), dict(after=dict(eps=math.nan)),
    dict(before=dict(eps=math.inf)), dict(after=dict(dtype=2)), dict(after=dict(plus_one=2)), dict(before=dict(weight=SOME + 1)),
    dict(before=dict(bias=SOME + 2, dtype=symar.F32)), dict(out=None, before=dict(kind=0), residual_out=None),
], ids=ids)
def test_norm_refuses(lib, change):
    assert norm_rc(lib, **change) == symar.ERR_INVAL


def test_norm_sizes(lib):
    assert lib.symar_norm(None, None) == symar.ERR_INVAL
    assert norm_rc(lib, n=32769, out_ld=40000, out_group=1 << 20, residual_out_ld=40000, residual_out_group=1 << 20) == symar.ERR_UNSUPPORTED
    assert norm_rc(lib, groups=1 << 16, m=1 << 15) == symar.ERR_UNSUPPORTED
    for empty in ("m", "n", "groups"):
        assert norm_rc(lib, **{empty: 0, "x": None, "residual": None}) == symar.OK


def route_rc(lib, **change):
    f = dict(logits=SOME, ld=64, bias=SOME, choice=SOME, weights=SOME, expert_start=SOME, row_token=SOME, token_row=SOME, workspace=SOME,
             workspace_bytes=1 << 20, scale=1.0, tokens=400, experts=64, top_k=4, dtype=symar.F32, score=0, renormalise=1)
    f.update(change)
    return lib.symar_route(ctypes.byref(symar.RouteArgs(**f)), None)


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(choice=None), dict(weights=None), dict(expert_start=None), dict(row_token=None), dict(token_row=None), dict(workspace=None),
    dict(tokens=-1), dict(experts=0), dict(top_k=0), dict(top_k=65), dict(dtype=2), dict(score=2), dict(score=-1), dict(renormalise=2), dict(ld=-1),
    dict(scale=math.nan), dict(scale=math.inf), dict(logits=SOME + 2), dict(logits=SOME + 1, dtype=symar.BF16), dict(bias=SOME + 2), dict(choice=SOME + 1),
    dict(weights=SOME + 2), dict(expert_start=SOME + 3), dict(row_token=SOME + 2), dict(token_row=SOME + 2), dict(workspace=SOME + 2),
    dict(tokens=0, expert_start=None),
], ids=ids)
def test_route_refuses(lib, change):
    assert route_rc(lib, **change) == symar.ERR_INVAL


def test_route_limits(lib):
    assert lib.symar_route(None, None) == symar.ERR_INVAL
    assert route_rc(lib, experts=1025) == symar.ERR_UNSUPPORTED
    assert route_rc(lib, top_k=33) == symar.ERR_UNSUPPORTED
    assert route_rc(lib, tokens=1 << 29) == symar.ERR_UNSUPPORTED
    need = lib.symar_route_workspace(400, 64)
    assert need > 0 and lib.symar_route_workspace(1, 64) == 0
    assert route_rc(lib, workspace_bytes=need - 1) == symar.ERR_NOMEM
    assert max(lib.symar_route_workspace(t, 1024) for t in (129, 5000, 1 << 30)) <= 148 * 4096


def combine_rc(lib, **change):
    f = {n + s: v for n in ("y", "residual", "out") for s, v in (("", SOME), ("_ld", 64), ("_group", 1024))}
    f.update(token_row=SOME, weights=SOME, groups=2, tokens=8, top_k=2, rows=16, n=64, dtype=symar.BF16, out_dtype=symar.F32, root=0)
    f.update(change)
    return lib.symar_combine(ctypes.byref(symar.CombineArgs(**f)), None)


@pytest.mark.parametrize("change", [
    dict(y=None), dict(out=None), dict(token_row=None), dict(groups=-1), dict(tokens=-1), dict(top_k=-1), dict(rows=-1), dict(n=-1), dict(dtype=2),
    dict(out_dtype=-1), dict(root=2), dict(root=-2), dict(y=SOME + 1), dict(out=SOME + 2), dict(residual=SOME + 2), dict(token_row=SOME + 2),
    dict(weights=SOME + 2), dict(y_ld=-1), dict(y_group=-1), dict(residual_ld=-1), dict(residual_group=-1), dict(out_ld=63), dict(out_ld=0),
    dict(out_group=0), dict(out_group=100), dict(out_group=-1),
], ids=ids)
def test_combine_refuses(lib, change):
    assert combine_rc(lib, **change) == symar.ERR_INVAL


def test_combine_sizes(lib):
    assert lib.symar_combine(None, None) == symar.ERR_INVAL
    assert combine_rc(lib, n=(1 << 30) + 1, out_ld=1 << 31, out_group=1 << 40) == symar.ERR_UNSUPPORTED
    assert combine_rc(lib, n=1 << 30, tokens=1 << 20, out_ld=1 << 31, out_group=1 << 52) == symar.ERR_UNSUPPORTED
    assert combine_rc(lib, groups=65536) == symar.ERR_UNSUPPORTED
    for empty in ("groups", "tokens", "n"):
        assert combine_rc(lib, **{empty: 0, "y": None, "out": None, "token_row": None}) == symar.OK


def experts_rc(lib, **change):
    f = dict(x=SOME, x_ld=64, x_group=512, w=SOME, w_ld=64, w_expert=4096, w_group=1 << 15, bias=SOME, bias_expert=64, bias_group=512, out=SOME, out_ld=32,
             out_group=1024, expert_start=SOME, row_token=SOME, groups=2, experts=8, rows=16, x_rows=8, n=32, k=64, out_dtype=symar.BF16, act=4, gated=1,
             status=SOME)
    f.update(change)
    return lib.symar_experts(ctypes.byref(symar.ExpertsArgs(**f)), None)


@pytest.mark.parametrize("change", [
    dict(x=None), dict(w=None), dict(out=None), dict(expert_start=None), dict(groups=-1), dict(experts=-1), dict(rows=-1), dict(x_rows=-1), dict(n=-1),
    dict(k=-1), dict(act=5), dict(act=-1), dict(gated=2), dict(gated=-1), dict(out_dtype=2), dict(x=SOME + 1), dict(w=SOME + 1), dict(bias=SOME + 1),
    dict(out=SOME + 1), dict(out=SOME + 2, out_dtype=symar.F32), dict(expert_start=SOME + 2), dict(row_token=SOME + 2), dict(status=SOME + 2),
    dict(row_token=None), dict(x_rows=0), dict(x_ld=-8), dict(x_group=-8), dict(w_ld=-8), dict(w_expert=-8), dict(w_group=-8), dict(bias_expert=-1),
    dict(bias_group=-1), dict(out_ld=31), dict(out_ld=-32), dict(out_group=0), dict(out_group=500),
], ids=ids)
def test_experts_refuses(lib, change):
    assert experts_rc(lib, **change) == symar.ERR_INVAL


@pytest.mark.parametrize("change", [
    dict(experts=1025), dict(rows=(1 << 30) + 1), dict(n=(1 << 30) + 1), dict(k=(1 << 30) + 1), dict(x_rows=(1 << 30) + 1), dict(x=SOME + 8), dict(w=SOME + 2),
    dict(x_ld=68), dict(x_ld=0), dict(x_group=100), dict(w_ld=12), dict(w_ld=0), dict(w_expert=4), dict(w_expert=0), dict(w_group=9),
    dict(x_ld=1 << 39, x_group=1 << 39), dict(w_expert=1 << 40),
], ids=ids)
def test_experts_is_not_for(lib, change):
    assert experts_rc(lib, **change) == symar.ERR_UNSUPPORTED


def test_experts_without_work(lib):
    assert lib.symar_experts(None, None) == symar.ERR_INVAL
    for empty in ("groups", "experts", "rows", "n"):
        assert experts_rc(lib, **{empty: 0, "x": None, "w": None, "out": None, "expert_start": None, "status": None}) == symar.OK
