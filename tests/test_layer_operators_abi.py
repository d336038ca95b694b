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
