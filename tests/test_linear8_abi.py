"""Linear layers on codes: refusals that need no device."""
import ctypes as C
import os

import pytest
import torch


@pytest.fixture(scope="module")
def L():
    from paper_2110_08919_amd import build, lpq
    if not os.path.exists(lpq.LIB_PATH):
        build.build()
    return lpq.lib()


def test_sizes_of_codes_and_workspaces(L):
    assert [L.lpq_row_codes_bytes(1, d) for d in (-1, 0, 1, 128, 129, 131072, 131073)] == [0, 0, 2048, 2048, 4096, 16 * 131072, 0]
    assert [L.lpq_row_codes_bytes(n, 1) for n in (-1, 0, 16, 17, 1 << 25, (1 << 25) + 1)] == [0, 0, 2048, 4096, 1 << 32, 0]
    for m, n, d in ((0, 5, 5), (5, 0, 5), (5, 5, 0), (5, 5, 1 << 20), ((1 << 25) + 1, 5, 5), (5, (1 << 25) + 1, 5), (-1, 5, 5)):
        assert L.lpq_linear8_workspace_bytes(m, n, d) == 0 and L.lpq_matmul_i8_workspace_bytes(m, n, d) == 0
    for m, n, d in ((1, 1, 1), (300, 700, 1000), (48, 11_111, 4100)):
        both, product = L.lpq_linear8_workspace_bytes(m, n, d), L.lpq_matmul_i8_workspace_bytes(m, n, d)
        assert both >= product


def test_refusals(L):
    from paper_2110_08919_amd import lpq
    a = C.create_string_buffer(4096)
    p = (C.addressof(a) + 255) // 256 * 256

    def encode(x=p, ldx=64, kind=0, n=2, d=64, codes=p, scales=p):
        return L.lpq_encode_rows(x, ldx, kind, n, d, codes, scales, None)

    def product(pa=p, sa=p, m=2, pb=p, sb=p, n=2, d=64, out=p, ldo=2, kind=0, ws=None, size=0):
        return L.lpq_matmul_i8(pa, sa, m, pb, sb, n, d, None, out, ldo, kind, ws, size, None)

    def linear(x=p, ldx=64, kind=0, m=2, codes=p, scales=p, n=2, d=64, out=p, ldo=2, ws=p, size=1 << 30):
        return L.lpq_linear8(x, ldx, kind, m, codes, scales, n, d, None, out, ldo, ws, size, None)

    for call in (encode, linear):
        assert call(d=0) == lpq.EINVAL and call(d=131_073, ldx=1 << 20) == lpq.ERANGE
        assert call(kind=3) == lpq.EINVAL and call(x=None) == lpq.EINVAL and call(codes=None) == lpq.EINVAL and call(scales=None) == lpq.EINVAL
        assert call(ldx=-1) == lpq.EINVAL and call(ldx=(1 << 40) + 1) == lpq.EINVAL
        assert call(codes=p + 128) == lpq.EINVAL
        assert call(n=-1) == lpq.EINVAL
    assert encode(n=(1 << 25) + 1) == lpq.ERANGE and linear(n=(1 << 25) + 1, ldo=1 << 26) == lpq.ERANGE
    assert encode(n=0, x=None, codes=None, scales=None) == lpq.OK
    for call in (product, linear):
        assert call(out=None) == lpq.EINVAL and call(ldo=1) == lpq.EINVAL and call(kind=-1) == lpq.EINVAL
        assert call(m=(1 << 25) + 1) == lpq.ERANGE and call(m=-1) == lpq.EINVAL
        assert call(m=1 << 25, n=1 << 20, ldo=1 << 20) == lpq.ERANGE       # more tiles than a launch has
        assert call(m=0, out=None) == lpq.OK and call(n=0) == lpq.OK
    assert product(pa=p + 16) == lpq.EINVAL and product(pb=p + 64) == lpq.EINVAL and product(pa=None) == lpq.EINVAL and product(sa=None) == lpq.EINVAL and product(sb=None) == lpq.EINVAL
    assert linear(m=9, ws=None) == lpq.EINVAL and linear(m=9, ws=p + 128) == lpq.EINVAL and linear(m=9, size=16) == lpq.ERANGE
    assert b"workspace" in L.lpq_last_error()


def test_which_way_products_go(L):
    """Few rows past LDS, up to 4 tiles of channels where there are many; tiles that grow with the product; parts only where workgroups are few."""
    from paper_2110_08919_amd import lpq
    info = lpq.linear8_plan_info
    assert info(1, 4096, 4096) == [16, 16, 0, 1] and info(8, 4096, 4096)[3] == 0 and info(8, 4096, 2048)[3] == 1 and info(1, 8, 16_385)[3] == 0
    assert info(48, 11_111, 4100) == [48, 48, 0, 0] and info(33, 4096, 4096)[:3] == [48, 16, 0]
    assert info(8192, 8192, 8192) == [256, 256, 1, 0] and info(1024, 4096, 4096) == [128, 128, 1, 0]
    assert info(300, 100, 100)[2] == 1 and info(128, 1024, 16_384)[2] > 1
    for m in (1, 16, 17, 33, 64, 65, 128, 129, 1000, 30_000):
        for n in (1, 16, 500, 5000, 70_000):
            for d in (1, 64, 65, 1000, 16_384, 131_072):
                rows, channels, parts, fused = info(m, n, d)
                stages = -(-d // 64)
                if parts == 0:
                    assert rows >= m and rows in (16, 32, 48, 64, 96, 128) and channels in (16, 32, 48, 64) and rows // 16 * channels // 16 <= 18
                else:
                    assert m > 32 and rows == channels and rows in (64, 128, 256) and (parts == 1 or rows < 256)
                    assert (parts - 1) * -(-stages // parts) < stages          # no part is empty
                    need = L.lpq_matmul_i8_workspace_bytes(m, n, d)
                    assert need == (0 if parts == 1 else parts * m * -(-n // 4) * 16)
    out = (C.c_int64 * 4)()
    assert L.lpq_linear8_plan_info(1, 1, 1, out, 3) == lpq.EINVAL and L.lpq_linear8_plan_info(0, 1, 1, out, 4) == lpq.EINVAL
    assert L.lpq_linear8_plan_info(1, 1, 1 << 18, out, 4) == lpq.ERANGE


def test_binding_takes_device_rows_only():
    from paper_2110_08919_amd import lpq
    lpq.lib()
    with pytest.raises(AssertionError):
        lpq.encode_rows(torch.zeros(2, 4))
    with pytest.raises(AssertionError):
        lpq.Linear8(torch.zeros(2, 4))
    with pytest.raises(AssertionError):
        lpq.RowCodes(torch.zeros(1, 2, 4, 16, 16, dtype=torch.int8), torch.zeros(2), 4)
