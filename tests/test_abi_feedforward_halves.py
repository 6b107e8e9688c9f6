"""Token matrices as columns of one buffer: no element is shared, so that no call refuses them.
No kernel is launched here: the calls end at the workspace that they are not given."""
import ctypes

import pytest

i64, vp, i32, sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
BF16, INVAL, WORKSPACE = 1, -1, -4
MB = 1 << 20


def _gated(G, ldg, U, ldu, H=8 * MB, ldh=32, n=100):
    import paper_2512_13886_amd as L
    f = ctypes.CDLL(L.library_path()).optima_gated_forward
    f.argtypes = [vp, i64, i64, i64, vp, vp, i64, i32, vp, i64, i32, vp, i64, vp, i64, vp, sz, vp]
    return f(1 * MB, 128, n, 128, 2 * MB, 3 * MB, 32, 1, H, ldh, BF16, G, ldg, U, ldu, None, 0, None)


A = 4 * MB  # rows of 64 values, 128 bytes; 32 of them, 64 bytes, are a matrix's


@pytest.mark.parametrize("G, U, status", [
    (A, A + 64, WORKSPACE), (A + 64, A, WORKSPACE),           # halves
    (A, A + 62, INVAL), (A + 62, A, INVAL),                   # one value in both
    (A, A + 66, INVAL), (A + 66, A, INVAL),                   # the last one and the next row's first
    (A, A + 128 * 7 + 64, WORKSPACE), (A, A + 128 * 7 + 62, INVAL),
    (A, A + 128 * 99 + 62, INVAL),                            # the last row alone
    (A + 128 * 99 + 62, A, INVAL),
    (A, A + 128 * 99 + 66, WORKSPACE), (A + 128 * 99 + 66, A, WORKSPACE),  # past the last row
    (A, A + 128 * 100, WORKSPACE), (A, A, INVAL),
])
def test_columns_of_one_buffer(G, U, status):
    assert _gated(G, 64, U, 64) == status


def test_three_columns_and_other_pitches():
    assert _gated(A, 96, A + 64, 96, A + 128, 96) == WORKSPACE
    assert _gated(A, 96, A + 64, 96, A + 126, 96) == INVAL
    assert _gated(A, 64, A + 64, 96) == INVAL     # different pitches: the extents


def test_overlap_of_spans_is_that_of_their_elements():
    # Every pair of small matrices in one buffer, against the elements themselves.
    import itertools
    for pitch, a, b, n in itertools.product((32, 40, 64, 71), range(0, 130, 13), range(0, 130, 17),
                                            (66,)):
        def elements(at):
            return {at + r * pitch + c for r in range(n) for c in range(32)}
        shared = bool(elements(a) & elements(b))
        got = _gated(A + 2 * a, pitch, A + 2 * b, pitch, n=n)
        assert got == (INVAL if shared else WORKSPACE), (pitch, a, b)
