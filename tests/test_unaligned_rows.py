"""Which bytes the product reads of rows on no 16-byte boundary: the library's own arithmetic (csrc/symar_rows.h), replayed on the host over
small and odd lengths, row strides and alignments.  No piece that is loaded whole may leave the operand, and no element may be missed."""
import subprocess

from paper_2607_16100_b200 import build

REPLAY = r"""
#include <stdio.h>
#include <vector>
#include "symar_rows.h"
using namespace symar;
int main()
{
    long outside = 0, missed = 0, whole = 0, parts = 0;
    const int rows_of[] = {1, 2, 5, 130}, pads[] = {0, 1, 2, 3, 4, 5, 6, 7, 8, 63, 64, 200};
    for (int k = 1; k <= 333; k = k < 140 ? k + 1 : k + 17)
        for (int rows : rows_of)
            for (int pad : pads)
                for (int base = 0; base < 16; base += 2) {
                    const int64_t ld = k + pad;
                    const uintptr_t at0 = 1 << 20 | base;
                    const Span s{at0, at0 + ((rows - 1) * ld + k) * 2};
                    for (int i = 0; i < rows; ++i) {
                        const uintptr_t row = at0 + i * ld * 2, first = row & ~(uintptr_t)15;
                        const int kind = row_kind(row, true, k, s), slices = (k + kSlice - 1) / kSlice;
                        if (row_kind(row, false, k, s) & 16 || !(kind & 16) || (kind & 15) != (int)(row & 15)) ++missed;
                        std::vector<char> have(2 * k, 0);
                        for (int slice = 0; slice <= slices; ++slice)       // one more than the row has: what its shift leaves over
                            for (int c = 0; c < 8; ++c) {
                                if (!piece_wanted(k, slice, c)) continue;
                                const uintptr_t at = first + slice * 128 + c * 16;
                                const bool all = piece_whole(at, kind, s);
                                all ? ++whole : ++parts;
                                if (all && (at < s.lo || at + 16 > s.hi)) ++outside;
                                for (int b = 0; b < 16; ++b)
                                    if (at + b >= row && at + b < row + 2 * k) have[at + b - row] = 1;
                            }
                        for (char h : have) missed += !h;
                    }
                }
    // lengths near 2^31: the last slice is there, what lies behind it is not
    const int k = 0x7fffffff, slices = (int)(((int64_t)k + kSlice - 1) / kSlice);
    if (!piece_wanted(k, slices - 1, 7) || !piece_wanted(k, slices, 0) || piece_wanted(k, slices, 1) || piece_wanted(k, slices + 1, 0)) ++missed;
    printf("%ld %ld %ld %ld\n", outside, missed, whole, parts);
    return 0;
}
"""


def test_no_piece_leaves_the_operand_and_none_is_missed(tmp_path):
    (tmp_path / "replay.cpp").write_text(REPLAY)
    exe = tmp_path / "replay"
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", str(build.CSRC), str(tmp_path / "replay.cpp"), "-o", str(exe)], check=True)
    outside, missed, whole, parts = map(int, subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split())
    assert whole > 0 and parts > 0
    assert outside == 0 and missed == 0


def test_the_kernel_asks_for_pieces_by_that_rule_alone():
    """No load of a row's piece but the one that the rule stands before."""
    text = (build.CSRC / "symar_linear.cu").read_text()
    assert text.count("load_if(") == 2 and text.count("edge_piece(") == 2          # each defined once, used once
    assert "const bool on = piece_wanted(k, slice, c);" in text
