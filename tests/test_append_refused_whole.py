"""An append in codes that is refused for its size has not rotated its queries before.  (On the CPU: a launch would be an error of
another kind.)"""
import ctypes

import paper_2311_08252_b200 as rest

UNSUPPORTED = 2


def strides(*s):
    return (ctypes.c_int64 * len(s))(*s)


def test_refused_before_the_queries_are_rotated():
    """One block of rows a context more than those of the queries: 2^31 thread blocks."""
    N, B = (1 << 30) - 20, 16
    assert B * 2 * ((N + 30) // 16) == 1 << 31 and B * 2 * ((N + 15) // 16) < 1 << 31     # (two to a block of rows)
    rows = strides(1 << 40, 2048, 128)
    got = rest.lib().rest_paged_kv_append_scaled(
        256, 256, strides(8 * 16 * 128, 16 * 128, 128), 256, 256, 4, 16, 256, 3, 3, 256, 256, 256, rows, None, 0, 256, 256, 64, 0,
        1.0, 256, rows, 256, rows, 16, B, 8, N, 128, None)
    assert got == UNSUPPORTED
