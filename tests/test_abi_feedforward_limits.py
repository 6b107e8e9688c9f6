"""Sizes past a launch's threads are refused before any launch. No kernel is launched here."""
import ctypes

import pytest

i64, vp, i32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
INVAL = -1


@pytest.mark.parametrize("chunks, n", [(5347, 50203),    # 2^28 - 15: blocks of 2^32 threads in all
                                       (6235, 43053),    # 2^28 - 1
                                       (16, 1 << 24)])   # 2^28
def test_pack_of_too_many_chunks(chunks, n):
    import paper_2512_13886_amd as L
    f = ctypes.CDLL(L.library_path()).optima_w4_pack
    f.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp]
    # Addresses that do not overlap at these sizes.
    assert f(1 << 40, 0, n, 128 * chunks, 128, 1 << 42, 1 << 44, None) == INVAL
