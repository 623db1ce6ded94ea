"""Rows and outputs near the end of 32 bits: tiles and groups of outputs round their counts up, so that what
would leave 32 bits there is refused, by the queries too.  Host-side, no kernel is launched."""
import ctypes

import pytest

from paper_1512_06473_gb300 import _lib
from test_int8_abi import P, _dense

lib = _lib.load()
INT_MAX = 2 ** 31 - 1
TOO_LARGE = [(INT_MAX, 8, 1), (INT_MAX - 255, 8, 1), (INT_MAX - 100, 131071, 4), (1, 8, INT_MAX), (1, 8, INT_MAX - 2),
             (9, 5000, INT_MAX - 255), (INT_MAX, 1, INT_MAX)]


@pytest.mark.parametrize("N,Cs,Ct", TOO_LARGE)
def test_too_many_rows_or_outputs(N, Cs, Ct):
    nb, info = ctypes.c_size_t(), (ctypes.c_int * 4)()
    assert lib.qcnn_int8_dense_workspace_size(N, Cs, Ct, 1, 1, ctypes.byref(nb)) == _lib.ERR_UNSUPPORTED
    assert lib.qcnn_int8_route_info(N, Cs, Ct, info) == _lib.ERR_UNSUPPORTED
    for xs in (None, P):
        assert _dense(N=N, Cs=Cs, Ct=Ct, ldx=Cs, ldw=Cs, ldy=Ct, xs=xs, wsb=1 << 60) == _lib.ERR_UNSUPPORTED


@pytest.mark.parametrize("N,Cs,Ct", [(INT_MAX - 256, 8, 1), (1, 8, INT_MAX - 256), (9, 5000, INT_MAX - 256)])
def test_the_largest_there_are(N, Cs, Ct):
    nb, info = ctypes.c_size_t(), (ctypes.c_int * 4)()
    assert lib.qcnn_int8_dense_workspace_size(N, Cs, Ct, 1, 1, ctypes.byref(nb)) == _lib.OK
    assert lib.qcnn_int8_route_info(N, Cs, Ct, info) == _lib.OK
    assert info[0] == 1 or nb.value >= N * 16 * ((Cs + 7) // 8)
