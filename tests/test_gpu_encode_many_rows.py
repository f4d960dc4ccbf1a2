"""Codes of many rows (2048 and more, and 1024 to 2047 long ones, which go ways of their own) against their definition, and products of such
rows from the definition's codes: a wrong code cannot cancel out.  Equal throughout."""
import pytest
import torch

from test_gpu_linear8 import TYPES, WAYS, codes_of, make, product_of, rows_of, same

pytestmark = pytest.mark.gpu


def special(x):
    """Rows of zeros, of small and large values, and some that are not finite, at their beginnings and ends."""
    n, d = x.shape
    x[3] = 0.0
    x[n // 2] *= 2.0 ** -12
    if x.dtype is not torch.float16:
        x[7] = (x[7].float() * 2.0 ** -124).to(x.dtype)             # below 2^-100, some of it subnormal
        x[n - 2] = (x[n - 2].float() * 2.0 ** 110).to(x.dtype)
    x[11, d - 1], x[n - 1, 0], x[n - 3, d // 2] = float("inf"), float("nan"), -float("inf")
    return x


# (from 2048 rows on: 1024 features to a turn through LDS, rows of more than 8192 values, float32 4096, read twice; below: 4 rows to a workgroup,
# rows of more than 4096 values read twice)
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,d", [(2048, 1), (2050, 127), (2049, 1025), (2055, 3000), (2064, 4097), (2051, 8200), (2049, 16_500), (4099, 2048), (1024, 4096),
                                 (1025, 4100), (1030, 16_500), (2047, 5000), (9000, 64)])
def test_many_rows_to_codes(kind, n, d):
    from paper_2110_08919_amd import lpq
    x = special(make(n, d, kind, 3 * d + n))
    got = lpq.encode_rows(x.cuda())
    codes, scales = codes_of(x)
    assert got.n == n and got.d == d and got.blocks.shape == ((n + 15) // 16, (d + 127) // 128 * 2, 4, 16, 16)
    assert torch.equal(rows_of(got).cpu()[:, :d].long(), codes)
    assert not rows_of(got)[:, d:].any()
    same(got.scales, scales)
    assert torch.isnan(scales[[11, n - 1, n - 3]]).all() and int(torch.isnan(scales).sum()) == 3 and scales[3] == 0


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_many_strided_rows_and_the_rows_behind_the_last(kind):
    from paper_2110_08919_amd import lpq
    n, d = 2053, 1300
    whole = make(n + 2, d + 9, kind, 5).cuda()
    x = whole[1:n + 1, 3:d + 3]
    codes, scales = codes_of(x.cpu())
    got = lpq.encode_rows(x)
    assert torch.equal(rows_of(got).cpu()[:, :d].long(), codes) and torch.equal(got.scales.cpu(), scales)
    one = lpq.encode_rows(whole[5:6, 3:d + 3].expand(n, -1))
    assert (one.blocks.permute(0, 3, 1, 2, 4).flatten(0, 1)[:n] == one.blocks[0, :, :, 0]).all()
    assert torch.equal(one.codes[0].cpu().long(), codes[4])
    blocks = torch.full_like(got.blocks, 55)
    room = torch.full((n + 3,), 5.0, device="cuda")
    assert lpq.lib().lpq_encode_rows(x.data_ptr(), x.stride(0), lpq._TYPE[x.dtype], n, d, blocks.data_ptr(), room.data_ptr(),
                                     torch.cuda.current_stream().cuda_stream) == lpq.OK
    rows = blocks.permute(0, 3, 1, 2, 4).flatten(0, 1).flatten(1)
    assert torch.equal(rows[:n], rows_of(got)) and (rows[n:] == 55).all() and (room[n:] == 5).all()


@pytest.mark.parametrize("rows,channels,parts,m,n,d", [w for w in WAYS if max(w[3:5]) >= 1024])
def test_products_of_the_definitions_codes(rows, channels, parts, m, n, d):
    from paper_2110_08919_amd import lpq
    x, w = make(m, d, "bf16", m + 1), make(n, d, "bf16", n + 2, 0.1)
    (a, sa), (b, sb) = codes_of(x), codes_of(w)
    want = product_of(a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), None, torch.bfloat16)
    assert torch.equal(lpq.Linear8(w.cuda())(x.cuda()), want)
