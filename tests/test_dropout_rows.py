"""Rows of dropout that pass 2^32, or whose sum passes 64 bits, are refused on the host."""
import pytest

import paper_2607_21653_gb300 as molt
from test_block_args import drop, dropout


@pytest.fixture(scope="module")
def lib():
    molt.build()
    return molt.load()


@pytest.mark.parametrize("T,first_row", [(4, 2**63 - 1), (4, 2**63 - 4), (4, 2**63 - 5), (1, 2**63 - 1), (4, 2**32), (2**32, 1),
                                         (2**32, 2**63 - 2**32), (4, -(2**63)), (0, 2**63 - 1), (0, 2**32 + 1)])
def test_rows_that_there_are_not(lib, T, first_row):
    n0 = lib.molt_kernel_launches()
    assert dropout(lib, drop(T=T, first_row=first_row), out=None) == "MOLT_ERR_UNSUPPORTED_SHAPE"
    assert lib.molt_kernel_launches() == n0


@pytest.mark.parametrize("T,first_row", [(4, 2**32 - 4), (2**32, 0), (0, 2**32)])
def test_the_last_rows(lib, T, first_row):
    """(refused for the missing output only)"""
    assert dropout(lib, drop(T=T, first_row=first_row), out=None) == ("MOLT_OK" if T == 0 else "MOLT_ERR_INVALID_ARG")
