"""Router, combine and norm near the limits of their sizes: what the library refuses or says on the host, so none of this needs a GPU."""
import pytest

from paper_2607_16100_b200 import build, symar
from test_layer_operators_abi import SOME, norm_rc, route_rc

MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    build.build_lib()
    return symar.load()


@pytest.mark.parametrize("tokens", [65, 4736, 4737, 10 ** 6 + 7, 2 ** 30, MOST - 4736, MOST - 4735, MOST - 1024, MOST])
def test_a_routers_blocks_are_counted_beyond_31_bits(lib, tokens):
    """Blocks of as many tokens for each of 32 warps, 148 of them at most."""
    of_block = 32 * -(-tokens // (148 * 32))
    for experts in (1, 2, 64, 1024):
        need = lib.symar_route_workspace(tokens, experts)
        assert need == -(-tokens // of_block) * experts * 4
        if experts > 1 and tokens <= MOST - 1024:
            assert route_rc(lib, tokens=tokens, experts=experts, top_k=1, workspace_bytes=need - 1) == symar.ERR_NOMEM
    assert route_rc(lib, tokens=MOST - 1023, experts=2, top_k=1) == symar.ERR_UNSUPPORTED


def test_a_norms_two_results_are_two(lib):
    """Both in x's or the residual's place: one of them would be lost."""
    for change in ({}, dict(stream_dtype=symar.BF16), dict(out_ld=128, out_group=512)):
        assert norm_rc(lib, **change) == symar.ERR_INVAL            # (everything at one address)
    apart = dict(out=SOME + (1 << 16))
    for change in (dict(out_ld=63), dict(out_group=0), dict(out_group=255), dict(residual_out_ld=0), dict(residual_out_group=32)):
        assert norm_rc(lib, **{**apart, **change}) == symar.ERR_INVAL
