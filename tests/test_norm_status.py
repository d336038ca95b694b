"""The status word of symar_norm at the library's boundary: on the CPU, so what is refused."""
import pytest

from paper_2607_16100_b200 import build, symar
from test_layer_operators_abi import SOME, norm_rc


@pytest.fixture(scope="module")
def lib():
    build.build_lib()
    return symar.load()


def test_a_word_on_no_boundary_is_refused(lib):
    for offset in (1, 2, 3):
        assert norm_rc(lib, status=SOME + offset) == symar.ERR_INVAL
    assert norm_rc(lib, status=SOME, x=None) == symar.ERR_INVAL
    for empty in ("m", "n", "groups"):
        assert norm_rc(lib, status=None, **{empty: 0}) == symar.OK


def test_a_wait_that_gives_up_is_reported_and_asks_for_nothing_more():
    """(A wait for the kernel's own copies cannot be made to run out: by the source.)"""
    text = (build.CSRC / "symar_norm.cu").read_text()
    ring = text[text.index("ring_kernel(const"):text.index("Ring ring_of")]
    assert ring.count("warp_wait(") == 1 and ring.count("bar_expect(") == 1
    assert "whole &= warp_wait(" in ring and ring.count("ask(row") == 2 and "if (i == 0 && whole) ask(row" in ring
    assert "atomicCAS(a.status, 0u, (unsigned)SYMAR_ERR_TIMEOUT)" in ring[ring.index("by = next;"):]
