"""Linear layers on codes: rows and outputs whose offsets pass 2^31 elements."""
import pytest
import torch

from test_gpu_linear8 import codes_of, make, product_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,d", [(3, 70, 300), (20, 600, 1400), (100, 8000, 3100), (130, 61, 1500), (500, 900, 64), (2000, 2100, 300), (3900, 4001, 2600)])
def test_rows_far_apart(m, n, d):
    """Rows of inputs and of outputs whose last is more than 2^31 elements behind the first, in every way of a product."""
    from paper_2110_08919_amd import lpq
    apart = (2 ** 31 + 2 ** 20) // (m - 1)
    room = torch.full((m, apart), 3.0, dtype=torch.bfloat16, device="cuda")
    assert (m - 1) * apart > 2 ** 31
    x, w = make(m, d, "bf16", m), make(n, d, "bf16", n + 1, 0.1)
    layer, far = lpq.Linear8(w.cuda()), room[:, 1:d + 1]
    far.copy_(x.cuda())
    out = room[:, d + 4:d + 4 + n]
    (a, sa), (b, sb) = codes_of(x), codes_of(w)
    want = product_of(a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), None, torch.bfloat16)
    assert torch.equal(layer(far, out=out), want)
    assert torch.equal(lpq.encode_rows(far).codes.cpu().long(), a)
    assert torch.equal(far.cpu(), x) and (room[:, d + 1:d + 4] == 3).all() and (room[:, d + 4 + n:d + 40 + n] == 3).all()


def test_an_output_of_more_values_than_32_bits_count():
    from paper_2110_08919_amd import lpq
    m, n, d = 70_000, 32_000, 70
    x, w = make(m, d, "bf16", 1), make(n, d, "bf16", 2, 0.1)
    layer = lpq.Linear8(w.cuda())
    y = layer(x.cuda())
    assert y.numel() > 2 ** 31
    (b, sb) = codes_of(w)
    for part in (slice(0, 300), slice(67_000, 67_300), slice(69_700, 70_000)):
        a, sa = codes_of(x[part])
        assert torch.equal(y[part], product_of(a.cuda(), sa.cuda(), b.cuda(), sb.cuda(), None, torch.bfloat16))
