"""The key-value cache's entry points without a device: argument checks that precede any device work, storage sizes."""
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
    h = C.c_void_p()
    one = C.c_int(1)
    p = C.addressof(one)
    assert L.lpq_kv_create(None, p, p, 1, 16, 1, 0, p, p, p) == lpq.EINVAL
    assert L.lpq_kv_create(C.byref(h), None, None, 1, 16, 1, 0, p, p, p) == lpq.EINVAL
    assert h.value is None
    assert L.lpq_kv_write(None, p, 1, 1, p, 1, 1, 0, 1, 1, p, None, p, 1, 1, None) == lpq.EINVAL
    assert L.lpq_kv_read(None, p, 1, 1, p, 1, 1, 0, 1, 1, p, None, p, 1, 1, None) == lpq.EINVAL
    assert L.lpq_kv_select(None, p, 1, 1, 1, 0, 1, 1, 1, p, p, 1, 1, 1, 0, 0, p, p, 256, None) == lpq.EINVAL
    assert L.lpq_kv_attend(None, p, 1, 1, 1, 0, 1, 1, 1, 1.0, p, p, 1, 1, None, 0, p, 1, 1, 1, None, p, 256, None) == lpq.EINVAL
    assert b"null" in L.lpq_last_error()
    assert L.lpq_kv_select_workspace_bytes(None, 1, 1) == 0
    assert L.lpq_kv_attend_workspace_bytes(None, 1, 1, 1, 1, 0) == 0
    L.lpq_kv_destroy(None)


@pytest.mark.parametrize("dim,row", [(1, 64), (64, 64), (65, 128), (128, 128), (129, 192), (192, 192), (200, 256), (256, 256)])
@pytest.mark.parametrize("packed", [0, 1])
def test_storage_bytes(lpq, dim, row, packed):
    codes, bounds, got = C.c_size_t(), C.c_size_t(), C.c_int()
    assert lpq.lib().lpq_kv_storage_bytes(8, dim, 64, 100_000, packed, C.byref(codes), C.byref(bounds), C.byref(got)) == lpq.OK
    assert got.value == row
    assert codes.value == 100_000 * 8 * 64 * row // (2 if packed else 1)
    assert bounds.value == 100_000 * 8 * 2 * row


def test_storage_shapes_that_are_refused(lpq):
    f = lpq.lib().lpq_kv_storage_bytes
    for heads, dim, page, pages, code in ((0, 64, 16, 1, lpq.EINVAL), (1, 0, 16, 1, lpq.EINVAL), (1, 64, 8, 1, lpq.EINVAL),
                                          (1, 64, 48, 1, lpq.EINVAL), (1, 64, 512, 1, lpq.EINVAL), (1, 64, 16, 0, lpq.EINVAL),
                                          (1, 257, 16, 1, lpq.ERANGE), (1, 64, 16, 1 << 31, lpq.ERANGE), (40000, 64, 16, 1, lpq.ERANGE)):
        assert f(heads, dim, page, pages, 0, None, None, None) == code
