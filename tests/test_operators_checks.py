"""Operators around the AllReduces: more of what the library refuses on the host (no GPU needed), beside test_operators_abi.py."""
import ctypes
import math
import subprocess

import pytest

from paper_2607_16100_b200 import build, symar
from test_operators_abi import SOME, call, lib, linear_args      # noqa: F401  (lib is a fixture)


@pytest.mark.parametrize("which", ["append", "read", "attention"])
def test_a_page_table_beyond_all_addresses(lib, which):          # noqa: F811
    for bad in (1 << 48, 1 << 60, (1 << 63) - 1):
        assert call(lib, which, batch=dict(table_ld=bad)) == symar.ERR_INVAL, bad



MEET = r"""
#include <stdio.h>
#include <stdlib.h>
#include "symar_rows.h"
int main(int n, char **v)
{
    for (int i = 1; i + 4 < n; i += 5) {
        long long x[5];
        for (int j = 0; j < 5; ++j) x[j] = atoll(v[i + j]);
        printf("%d", (int)symar::rows_meet(x[0], x[1], x[2], x[3], x[4]));
    }
    return 0;
}
"""
LAYOUTS = [(na, a, nb, b) for na in (1, 2, 3, 6) for a in (0, 100, 128, 129, 256, 300, 384, 640, 1000)
           for nb in (1, 2, 5) for b in (0, 127, 128, 200, 256, 257, 384, 512, 768, 5000)]


def meet(na, a, nb, b, n=128):
    rows = sorted(i * a + j * b for i in range(na) for j in range(nb))
    return any(y - x < n for x, y in zip(rows, rows[1:]))


def test_rows_meet_as_counted(tmp_path):
    """The rule against all rows of a layout in order; and strides near 2^63."""
    (tmp_path / "meet.cpp").write_text(MEET)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", str(build.CSRC), str(tmp_path / "meet.cpp"), "-o", str(tmp_path / "meet")],
                   check=True)
    far = [(4, 1 << 62, 4, 128), (4, 128, 4, (1 << 62) + 1), (1 << 20, 1 << 62, 4096, 128), (4096, 1 << 62, 4096, (1 << 62) + 127)]
    cases = LAYOUTS + far
    got = subprocess.run([str(tmp_path / "meet"), *(str(x) for c in cases for x in (*c, 128))], check=True, capture_output=True, text=True).stdout
    want = [meet(*c) for c in LAYOUTS] + [False, False, False, True]
    assert any(want) and not all(want)
    assert [c == "1" for c in got] == want


@pytest.mark.parametrize("na,a,nb,b", [x for x in LAYOUTS if meet(*x)])
def test_rows_that_share_an_element_are_refused(lib, na, a, nb, b):          # noqa: F811
    """As many tokens as na, and heads or ranks as nb."""
    batch = dict(seqs=na, tokens=na)
    assert call(lib, "append", batch=batch, args=dict(q_out_ld=a, q_out_head=b, q_heads=nb)) == symar.ERR_INVAL
    assert call(lib, "attention", cache=dict(kv_heads=1), batch=batch, args=dict(out_ld=a, out_head=b, q_heads=nb)) == symar.ERR_INVAL
    for n in "kv":
        assert call(lib, "read", cache=dict(kv_heads=nb), batch=batch, args={n + "_ld": a, n + "_head": b}) == symar.ERR_INVAL
    assert lib.symar_linear(linear_args(m=na, out_ld=a, groups=nb, out_group=b, n=128), None) == symar.ERR_INVAL


@pytest.mark.parametrize("bad", [
    dict(base=math.inf), dict(base=math.nan), dict(magnitude=math.nan), dict(magnitude=math.inf), dict(magnitude=-math.inf),
    dict(kind=1, factor=math.nan), dict(kind=1, factor=math.inf), dict(kind=1, factor=5e-324), dict(kind=2, factor=math.inf), dict(kind=2, factor=1e300, base=1e300),
    dict(kind=2, factor=1e-300, base=1e-300), dict(kind=3, original=math.inf), dict(kind=3, high=math.inf), dict(kind=3, low=-math.inf),
    dict(kind=3, low=math.nan),
], ids=lambda c: ",".join(f"{k}={v}" for k, v in c.items()))
def test_rope_table_refuses_what_is_not_finite(lib, bad):        # noqa: F811
    f = dict(base=1e4, factor=2.0, original=64.0, low=1.0, high=4.0, magnitude=1.0, kind=0, rot_dim=64)
    f.update(bad)
    assert lib.symar_rope_table(SOME, 16, ctypes.byref(symar.RopeScaling(**f)), None) == symar.ERR_INVAL
    assert lib.symar_rope_table(None, 0, ctypes.byref(symar.RopeScaling(**f)), None) == symar.ERR_INVAL


def test_sizes_whose_last_tile_would_pass_2_31(lib):             # noqa: F811
    big = 2 ** 31 - 1
    for bad in (dict(m=big), dict(n=big, out_ld=big), dict(k=big, x_ld=big, w_ld=big), dict(k=2 ** 31 - 511, x_ld=big, w_ld=big),
                dict(m=big, n=0), dict(k=big, m=0)):
        assert lib.symar_linear(linear_args(**bad), None) == symar.ERR_UNSUPPORTED, bad
    for which in ("append", "read", "attention"):
        assert call(lib, which, batch=dict(tokens=big, token_start=SOME)) == symar.ERR_UNSUPPORTED
    f = dict(base=1e4, factor=2.0, original=64.0, low=1.0, high=4.0, magnitude=1.0, kind=0, rot_dim=64)
    for rows in (1 << 48, (1 << 63) - 1):
        assert lib.symar_rope_table(SOME, rows, ctypes.byref(symar.RopeScaling(**f)), None) == symar.ERR_INVAL
