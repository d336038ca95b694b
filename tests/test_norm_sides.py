"""What of a norm's description reaches the kernels, which read weights and biases wherever there is a pointer: the library's own code (csrc/symar_norm_side.h), replayed
on the host.  A norm that is none leads to no memory, whatever stands in its fields."""
import subprocess

from paper_2607_16100_b200 import build

REPLAY = r"""
#include <stdio.h>
#include "symar_norm_side.h"
using namespace symar;
int main()
{
    char some[64];
    for (int kind = SYMAR_NORM_NONE; kind <= SYMAR_NORM_LAYER; ++kind)
        for (int dtype = -1; dtype <= SYMAR_BF16; ++dtype)
            for (int w = 0; w < 3; ++w)
                for (int b = 0; b < 3; ++b) {
                    const symar_norm_side_t s{w ? some + w : nullptr, b ? some + b : nullptr, 0.5f, kind, dtype, 1};
                    const Side got = side_of(s);
                    if (got.kind != kind) return 1;
                    if (kind == SYMAR_NORM_NONE ? got.weight || got.bias : got.weight != s.weight || got.bias != s.bias) return 2;
                    if (kind != SYMAR_NORM_NONE && (got.wide != (dtype == SYMAR_F32) || got.plus_one != 1 || got.eps != 0.5f)) return 3;
                }
    return 0;
}
"""


def test_a_norm_that_is_none_has_no_weights(tmp_path):
    (tmp_path / "replay.cpp").write_text(REPLAY)
    exe = tmp_path / "replay"
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", str(build.CSRC), "-I", str(build.ROOT / "include"), str(tmp_path / "replay.cpp"),
                    "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def test_the_kernels_get_their_norms_by_that_rule_alone():
    text = (build.CSRC / "symar_norm.cu").read_text()
    assert "a.after = side_of(p.after);  a.before = side_of(p.before);" in text
    assert "Side{" not in text
