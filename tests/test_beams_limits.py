"""Sizes beyond what a launch's indices hold are refused on the host."""
import ctypes as C

import pytest

from paper_2407_20272_amd import binding as B
from test_beams_abi import OK, P, UNSUPPORTED, desc


@pytest.mark.parametrize("n", [(1 << 30) + 1, (1 << 31) - 1])
def test_more_moves_than_their_list_is_indexed_for(n):
    """A move's two entries stand at 2 m and 2 m + 1, in 32 bits."""
    cache, quant, d = B.ee_kv_cache(P, P, 10, 16), B.ee_quant_cache(P, P, P, 2, 8, 16, 4, 64, B.EE_QUANT_INT8), desc()
    assert B.lib().ee_kv_copy(C.byref(d), C.byref(cache), P, n, None, None) == UNSUPPORTED and "moves" in B.ee_last_error()
    assert B.lib().ee_kv_quant_copy(C.byref(quant), P, n, P, None) == UNSUPPORTED and "moves" in B.ee_last_error()
    assert B.lib().ee_kv_copy(C.byref(d), C.byref(cache), P, 0, None, None) == OK
