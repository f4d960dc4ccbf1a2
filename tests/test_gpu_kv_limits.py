"""How much a call of attention over a key-value cache takes, and prompts that are longer."""
import pytest
import torch

from test_gpu_kv_cache import Case, ints, lpq  # noqa: F401  (lpq is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mask", [{}, dict(window=40, sinks=3)])
def test_too_many_rows_are_refused(lpq, mask):
    c = Case(lpq, 1, 64, 16, [300, 20], "bf16")
    q = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16, device="cuda")
    for seqs, new, heads in ((1, 4097, 16), (1, 1, 65_537), (2, 32_769, 2), (65, 4096, 16)):
        with pytest.raises(lpq.LpqError) as e:
            c.cache.attend(q.expand(seqs, new, heads, 64), ints([300] * seqs), c.table[:1].expand(seqs, -1).contiguous(), **mask)
        assert e.value.code == lpq.ERANGE
    assert c.cache.attend(q.expand(1, 4096, 16, 64), ints([300]), c.table[:1], **mask).shape == (1, 4096, 16, 64)


@pytest.mark.parametrize("mask", [{}, dict(window=40, sinks=3), dict(window=2000)])
def test_a_prompt_in_parts(lpq, mask):
    """Parts, each with the length up to its end, see what the tokens see in one call.  A row's roundings depend on the rows and tokens beside it (where
    their common maximum stood): weights to 2^-11, twice the values' spread; the result to 2^-8."""
    c = Case(lpq, 2, 64, 16, [700], "bf16", seed=3)
    q = c.queries(3, 700).cuda()
    whole = c.cache.attend(q, ints([700]), c.table, **mask).float()
    spread = float((c.vx[0].max(0) - c.vx[0].min(0)).max())
    at = 0
    for part in (1, 16, 300, 383):
        got = c.cache.attend(q[:, at:at + part], ints([at + part]), c.table, **mask).float()
        want = whole[:, at:at + part]
        assert bool(((got - want).abs() <= 2 * 2.0 ** -11 * 2 * spread + 2 * 2.0 ** -8 * want.abs()).all())
        at += part
    assert at == 700
