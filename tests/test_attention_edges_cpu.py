"""Calls at the edges of what the attention library takes, without a GPU."""
import ctypes as C

import pytest

from paper_2301_04285_amd import attention as A, build_attention, taps


@pytest.fixture(scope="module", autouse=True)
def built():
    import os
    if not os.path.exists(A.LIB_PATH):
        build_attention.build()


def _heads(ptr=0x1000, strides=(512, 512, 64)):
    return A.Heads(ptr, *strides)


NONE = A.Heads(None, 0, 0, 0)


@pytest.mark.parametrize("size", [4, 8])
def test_positions_without_a_table_row_are_refused(size):
    """No position is a row of an empty table: there is no row to read in its place."""
    a = A.NormRotateArgs(1, 4, 8, 0, 64, 64, A.BF16, A.BF16, 0, 1e-6, None, None, 0x1000, 0, size,
                         0x1000, 0)
    L, need = A.load(), C.c_uint64()
    assert L.taps_norm_rotate(C.byref(a), _heads(), NONE, _heads(), NONE, None) == taps.ERR_ARG
    assert "no rows" in A.last_error()
    assert L.taps_norm_rotate_backward(C.byref(a), _heads(), NONE, _heads(), NONE, _heads(), NONE,
                                       None, None, 0x1000, C.byref(need), None) == taps.ERR_ARG
    assert "no rows" in A.last_error()
    a.tokens = 0   # nothing to look up
    assert L.taps_norm_rotate(C.byref(a), _heads(), NONE, _heads(), NONE, None) == taps.OK
