"""Attention holds small weights to the same part of the largest whatever a token sees: without a mask, with a window, over a tree, and
on the way of windows on many rows."""
import numpy as np
import pytest
import torch

from test_gpu_kv_cache import TYPES, ints, lpq  # noqa: F401  (lpq is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("way", ["none", "window", "tree", "rows"])
def test_weights_35_powers_of_two_below_the_largest(lpq, way, kind):
    """1000 tokens, every 32nd of the first 256 with nearly all the weight and values of 0, the others at 2^-35 of it with values of 127.  Weights are held
    to 2^-38 of the largest (half of fp16's last step, 2^-25, beside 2^13), an eighth of a small one; its score, 35 in powers of two, is off by 8
    roundings to 2^-24 at most, a factor of 1 +- 2^-16.  A result x is (x + 1/2) s + k with k = -s / 2 in binary32: two roundings of 2^-25; and one to
    the type, of 2^-9 of it or (float16) 2^-25.  lse: 16 roundings to 2^-24 of numbers up to 32.  Steps and constants are powers of two, keys differ in one feature, so that nothing else is rounded."""
    n, dim, page = 1000, 64, 16
    base, width = torch.full((dim,), -0.5), 128.0
    quant = [lpq.Quantizer(dim, 8).set_params(base, base - width, base + width) for _ in range(2)]      # codes read back as whole numbers
    cache = lpq.KVCache(*quant, heads=1, page=page, pages=63)
    k, v = torch.zeros(n, 1, dim), torch.full((n, 1, dim), 127.0)
    large = torch.arange(5, 256, 32)
    k[:, 0, 3] = -60.0
    k[large, 0, 3], v[large] = 40.0, 0.0
    table = torch.full((1, 64), -1, dtype=torch.int32, device="cuda")
    table[0, :63] = torch.arange(63)
    cache.write(k.to(TYPES[kind]).cuda(), v.to(TYPES[kind]).cuda(), ints([0]), table, ints([0, n]))
    seqs, group = (512, 33) if way == "rows" else (1, 2)
    q = torch.zeros(seqs, 1, group, dim, dtype=TYPES[kind], device="cuda")
    q[..., 3] = 1.0
    kw = {"none": {}, "tree": dict(tree=torch.ones(1, 1, dtype=torch.bool, device="cuda"))}.get(way, dict(window=1010))
    out, lse = cache.attend(q, ints([n] * seqs), table.expand(seqs, -1).contiguous(), scale=35 * np.log(2.0) / 100, return_lse=True, **kw)
    few, many = len(large), n - len(large)
    want = many * 127 * 2.0 ** -35 / (few + many * 2.0 ** -35)
    bound = many * 127 * 2.0 ** -38 / few + want * (2.0 ** -16 + 2.0 ** -9) + 3 * 2.0 ** -25
    assert bound < want / 2                                   # without them the result would be 0
    assert float((out.double() - want).abs().max()) <= bound
    assert float((lse.double() - (40 * 0.35 * np.log(2.0) + np.log(few))).abs().max()) <= 2.0 ** -15
