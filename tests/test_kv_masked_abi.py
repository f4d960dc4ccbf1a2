"""Masked attention's entry points without a device: what is refused before any device work."""
import ctypes as C
import os

import pytest


@pytest.fixture(scope="module")
def lpq():
    from paper_2110_08919_amd import build, lpq as m
    if not os.path.exists(m.LIB_PATH):
        build.build()
    m.lib()
    return m


def test_null_arguments_are_refused(lpq):
    L = lpq.lib()
    one = C.c_int(1)
    p = C.addressof(one)
    for window, sinks, tree in ((4, 0, None), (0, 0, p), (0, 0, None), (-1, 0, None), (4, -1, None), (0, 3, None), (4, 0, p)):
        assert L.lpq_kv_attend_masked(None, p, 1, 1, 1, 0, 1, 1, 1, 1.0, p, p, 1, 1, None, 0, window, sinks, tree, 1, 1, p, 1, 1, 1, None, p, 256,
                                      None) == lpq.EINVAL
        assert L.lpq_kv_attend_masked_workspace_bytes(None, 1, 1, 1, 1, 0, window, sinks, tree is not None) == 0


def test_rotated_writes_of_no_cache_are_refused(lpq):
    one = C.c_int(1)
    p = C.addressof(one)
    assert lpq.lib().lpq_kv_write_rotated(None, p, 1, 1, p, 1, 1, 0, 1, 1, p, None, p, 1, 1, p, p, 1, 1, 2, 0, None, p, 1, 1, 1, p, 1, 1,
                                          None) == lpq.EINVAL
