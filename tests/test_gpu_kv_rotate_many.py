"""Rotated writes of so many rows that a workgroup of queries takes more of them: equal to the definition, as in test_gpu_kv_rotate.py."""
import numpy as np
import pytest
import torch

import kv_plain as plain
from test_gpu_kv_cache import Case, lpq  # noqa: F401  (a fixture)
from test_gpu_kv_rotate import Rotated, equal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,packed,heads,dim,group,rotated,interleaved", [
    ("bf16", False, 1, 128, 32, 128, False), ("f16", True, 2, 100, 9, 52, True), ("f32", False, 1, 33, 30, 22, False), ("bf16", True, 3, 80, 8, 64, True)])
def test_prompts_of_many_rows(lpq, kind, packed, heads, dim, group, rotated, interleaved):
    before, added = [0, 300, 7, 0], [7000, 2, 4100, 5903]
    c = Case(lpq, heads, dim, 64, [b + a for b, a in zip(before, added)], kind, packed, seed=dim)
    r = Rotated(c, group, before, added, rotated, interleaved)
    q = r.q.cuda()
    out = r.call(c.cache, c.table, queries=q)
    assert equal(out.cpu(), r.want_queries()) and torch.equal(q.cpu(), r.q)
    kcodes, vcodes = plain.codes(r.turned(r.k), c.kc, packed), plain.codes(r.v.float().numpy(), c.vc, packed)
    for b, n in enumerate(before):
        rows = slice(int(r.starts[b]), int(r.starts[b + 1]))
        want = np.concatenate([c.kcodes[b][:n], kcodes[rows]])
        assert np.array_equal(c.stored(b, "k"), want)
        assert np.array_equal(c.stored(b, "v"), np.concatenate([c.vcodes[b][:n], vcodes[rows]]))
        pages = c.table_np[b, :-(-len(want) // 64)]
        assert np.array_equal(c.cache.bounds.cpu().numpy()[pages], plain.bounds(want, 64))
    assert r.call(c.cache, c.table, queries=q, out=q) is q
    assert equal(q.cpu(), r.want_queries())
