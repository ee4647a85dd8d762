"""Limits of the residual norm's descriptor, refused on the host.

The persistent kernels count rows in 32 bits and step by a grid's rows, at most 8 blocks an
SM of 4 rows each: a row count within one step of 2^31 would wrap past it.  2^17 covers the step
of 4096 SMs."""
import ctypes

import pytest

import paper_2607_21653_gb300 as molt
from paper_2607_21653_gb300 import stream as S

FAKE = 0x1000   # never dereferenced
MOST = (1 << 31) - (1 << 17)


@pytest.fixture(scope="module")
def lib():
    molt.build()
    return molt.load()


def desc(T, H, gate=S.GATE_NONE):
    return S.NormDesc(T, H, 0, 0, 0, 0, 0, 0, gate, 1.0, 1e-6, 0.0)


@pytest.mark.parametrize("T", [MOST + 1, (1 << 31) - 4864, (1 << 31) - 1])
def test_rows_past_the_limit(lib, T):
    d = ctypes.byref(desc(T, 1))
    # (a pointer is missing, so that an accepted row count ends here too)
    st = lib.molt_residual_norm_fwd(d, None, FAKE, None, None, FAKE, FAKE, FAKE, None, None, None)
    assert molt.STATUS[st] == "MOLT_ERR_UNSUPPORTED_SHAPE"
    st = lib.molt_residual_norm_bwd(d, *[None] * 14, 0, None, 0, None)
    assert molt.STATUS[st] == "MOLT_ERR_UNSUPPORTED_SHAPE"
    assert lib.molt_residual_norm_bwd_workspace_bytes(d) == 0


def test_rows_at_the_limit(lib):
    d = ctypes.byref(desc(MOST, 1))
    st = lib.molt_residual_norm_fwd(d, None, FAKE, None, None, FAKE, FAKE, FAKE, None, None, None)
    assert molt.STATUS[st] == "MOLT_ERR_INVALID_ARG"
    assert lib.molt_residual_norm_bwd_workspace_bytes(d) > 0


def test_in_place_residual_needs_rows_side_by_side(lib):
    """r' is written with its rows side by side: over a residual whose rows are not, it would
    overwrite rows that are still to be read."""
    def call(T, stride, r, r_out):
        d = S.NormDesc(T, 64, 0, stride, 0, 0, 0, 0, S.GATE_NONE, 1.0, 1e-6, 0.0)
        return molt.STATUS[lib.molt_residual_norm_fwd(ctypes.byref(d), FAKE, r, None, None, None, None, r_out, None, None, None)]

    n0 = lib.molt_kernel_launches()
    assert call(4, 72, FAKE, FAKE) == "MOLT_ERR_INVALID_ARG"
    assert b"in place" in lib.molt_last_error()
    assert lib.molt_kernel_launches() == n0
    # no rows: nothing to overwrite
    assert call(0, 72, FAKE, FAKE) == "MOLT_OK"
