"""Descriptors of page pools as C callers fill them: decided on the host, before any device is touched."""
import ctypes

import pytest

SHAPE, ALIGN, WORKSPACE = 2, 4, 5
P = 1 << 20                                       # a pointer that is never followed


@pytest.fixture(scope="module")
def ac():
    from paper_2606_07665_b200 import binding, build
    build.build()
    return binding


def fork(ac, base, page_bytes, segments, last):
    """A pool of pages of 32 slots in a fork.  (One that is accepted meets the workspace, which is too small.)"""
    pools = (ac.AcPagePool * 1)()
    assert ctypes.sizeof(pools) == 24
    for at, value in ((0, ctypes.c_uint64(base)), (8, ctypes.c_int64(page_bytes)), (16, ctypes.c_int32(segments)), (20, ctypes.c_int32(last))):
        ctypes.memmove(ctypes.addressof(pools) + at, ctypes.byref(value), ctypes.sizeof(value))
    return ac.lib().ac_cache_fork(pools, 1, P, 4, P, P, P, 1, 4, 32, 64, P, 0, None, None)


@pytest.mark.parametrize("last", [0, 1, -1, 77, 2**31 - 1])
def test_the_int_behind_segments_means_nothing(ac, last):
    assert fork(ac, P, 16 * 17, 1, last) == SHAPE and fork(ac, P, 16 * 32, 1, last) == WORKSPACE
    assert fork(ac, P, 16 * 17, ac.AC_PAGE_WHOLE, last) == WORKSPACE
    assert fork(ac, P, 16 * 17 + 8, ac.AC_PAGE_WHOLE, last) == ALIGN and fork(ac, P + 8, 16, ac.AC_PAGE_WHOLE, last) == ALIGN
    for segments in (0, -2, -2**31):
        assert fork(ac, P, 16 * 32, segments, last) == SHAPE
