"""Operators around the AllReduces: more of what the library refuses on the host (no GPU needed), beside test_operators_abi.py."""
import ctypes

import pytest

from paper_2607_16100_b200 import symar
from test_operators_abi import SOME, call, lib, linear_args      # noqa: F401  (lib is a fixture)


@pytest.mark.parametrize("which", ["append", "read", "attention"])
def test_a_page_table_beyond_all_addresses(lib, which):          # noqa: F811
    for bad in (1 << 48, 1 << 60, (1 << 63) - 1):
        assert call(lib, which, batch=dict(table_ld=bad)) == symar.ERR_INVAL, bad
