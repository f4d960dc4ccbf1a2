"""Linear layers on codes: sums beyond 2^24, which binary32 does not hold all of, in every way of a product."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n", [(1, 5), (9, 40), (40, 5000), (130, 61), (500, 900), (2000, 2100), (3900, 4001)])
def test_a_sum_is_rounded_before_it_is_scaled(m, n):
    """The sum 2^24 + 1, times scales of 3 and 1: 3 (2^24 + 1) would round to 3 x 2^24 + 4, the definition gives 3 x 2^24."""
    from paper_2110_08919_amd import lpq
    a, b = torch.full((1065,), 127.0), torch.ones(1065)
    a[1064], b[:1040] = 9.0, 127.0
    assert int((a * b).sum(dtype=torch.float64)) == 2 ** 24 + 1
    x, w = (3 * a).expand(m, -1).cuda(), b.expand(n, -1).cuda()
    codes = lpq.encode_rows(x[:1])
    assert torch.equal(codes.codes[0].cpu().float(), a) and float(codes.scales[0]) == 3.0
    assert (lpq.Linear8(w)(x) == 3.0 * 2 ** 24).all()
    assert (lpq.matmul_i8(lpq.encode_rows(x), lpq.encode_rows(w), dtype=torch.float32) == 3.0 * 2 ** 24).all()
