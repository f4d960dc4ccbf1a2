"""Attention with a window for query rows that fill the chip (parts of prompts, many conversations), which goes a way of its own: a wave to 16 rows,
codes shared through LDS.  Against the plain definition in 64 bits, within the bound that kv_plain.py derives for attention."""
import numpy as np
import pytest
import torch

import kv_plain as plain
from test_gpu_kv_cache import TYPES, Case, ints, lpq  # noqa: F401  (lpq is a fixture)
from test_gpu_kv_masked import roomy, window_mask

pytestmark = pytest.mark.gpu


def goes_by_rows(c, group, new):
    rows = group * new
    return rows > 32 and len(c.lengths) * c.heads * -(-rows // 128) >= (512 if c.dim <= 128 else 256)


def check(c, q, out, lse, group, sees, some=None):
    """Of all sequences, or of `some`."""
    kind = {v: k for k, v in TYPES.items()}[q.dtype]
    scale = c.dim ** -0.5
    q, out, lse = q.float().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b in range(len(c.lengths)) if some is None else some:
        n, mask = c.lengths[b], sees[b]
        err, lerr = plain.attend_bound(q[b], c.kcodes[b], c.vx[b], c.kc, group, scale, kind)
        for j in range(q.shape[2]):
            empty = ~mask.any(1)
            assert (out[b, empty, j] == 0).all() and np.isneginf(lse[b, empty, j]).all()
            if n == 0 or empty.all():
                continue
            t = np.where(mask, scale * (q[b, :, j].astype(np.float64) @ c.kx[b][:, j // group].T), -np.inf)[~empty]
            most = t.max(1, keepdims=True)
            p = np.exp(t - most)
            o, want = p @ c.vx[b][:, j // group] / p.sum(1, keepdims=True), (most + np.log(p.sum(1, keepdims=True)))[:, 0]
            assert (np.abs(out[b, ~empty, j] - o) <= err[~empty, j]).all(), (b, j)
            assert (np.abs(lse[b, ~empty, j] - want) <= lerr[~empty, j]).all(), (b, j)


# heads, dim, page, sequences, longest, type, packed, group, new, window, sinks
CASES = [
    (8, 128, 32, 64, 200, "bf16", False, 4, 9, 70, 3),
    (8, 128, 16, 64, 150, "bf16", True, 3, 43, 33, 0),       # 129 rows: a tile and one row
    (8, 96, 64, 64, 300, "f16", True, 11, 3, 100, 20),
    (4, 128, 32, 128, 130, "f16", False, 33, 1, 50, 1),      # one new token, many query heads
    (8, 100, 16, 64, 90, "f32", False, 4, 10, 17, 5),
    (8, 33, 16, 64, 140, "f32", True, 2, 20, 64, 130),       # sinks beyond some sequences
    (16, 64, 128, 32, 260, "bf16", False, 1, 40, 1, 0),
    (8, 50, 16, 64, 120, "f16", False, 5, 8, 1000, 0),       # a window beyond most of the sequences
    (4, 192, 32, 64, 160, "bf16", True, 6, 7, 48, 2),
    (8, 180, 16, 32, 200, "f32", False, 3, 13, 90, 33),
    (4, 256, 64, 64, 170, "f16", False, 2, 30, 75, 4),
    (8, 256, 32, 32, 100, "f32", True, 4, 9, 40, 1),
    (8, 200, 16, 32, 130, "bf16", False, 8, 33, 60, 7),      # 264 rows: three tiles, the last with 8
]


@pytest.mark.parametrize("heads,dim,page,seqs,longest,kind,packed,group,new,window,sinks", CASES)
def test_many_rows(lpq, heads, dim, page, seqs, longest, kind, packed, group, new, window, sinks):
    lengths = [0, 1, new - 1, new, new + 1, longest] + [int(x) for x in np.random.default_rng(dim).integers(0, longest, seqs - 6)]
    c = Case(lpq, heads, dim, page, lengths, kind, packed, seed=window)
    assert goes_by_rows(c, group, new)
    q = c.queries(group, new)
    sees = [window_mask(n, new, window, sinks) for n in lengths]
    for columns in (None, 4000):
        out, lse = c.cache.attend(q.cuda(), ints(lengths), roomy(c, columns), window=window, sinks=sinks, return_lse=True)
        # (few of the sequences without room, all with it)
        check(c, q, out, lse, group, sees, list(range(6)) + [seqs - 1] if columns is None else None)
        assert torch.equal(out, c.cache.attend(q.cuda(), ints(lengths), roomy(c, columns), window=window, sinks=sinks))


@pytest.mark.parametrize("kind,packed,dim,window,sinks", [("bf16", False, 128, 1100, 4), ("f16", True, 96, 1500, 0), ("f32", False, 64, 1300, 100)])
def test_parts_of_prompts(lpq, kind, packed, dim, window, sinks):
    """Thousands of rows on a few heads, windows of more than 64 tiles of tokens: nothing is split, no workspace asked for."""
    lengths, new, group, heads = [5200, 1400], 1030, 4, 8
    c = Case(lpq, heads, dim, 64, lengths, kind, packed, seed=4)
    assert goes_by_rows(c, group, new)
    assert lpq.lib().lpq_kv_attend_masked_workspace_bytes(c.cache._h, 2, new, heads * group, 4000, 0, 1100, 4, 0) == 0
    q = c.queries(group, new)
    out, lse = c.cache.attend(q.cuda(), ints(lengths), roomy(c, 4000), window=window, sinks=sinks, return_lse=True)
    pick = np.r_[0:40, 500:520, new - 20:new]                # of the new tokens
    part = torch.from_numpy(pick)
    for b, n in enumerate(lengths):
        one = type("Part", (), dict(dim=dim, lengths=[n], kcodes=[c.kcodes[b]], vx=[c.vx[b]], kx=[c.kx[b]], kc=c.kc))
        check(one, q[b:b + 1, part], out[b:b + 1, part.cuda()], lse[b:b + 1, part.cuda()], group, [window_mask(n, new, window, sinks)[pick]])


def test_a_window_over_listed_pages(lpq):
    lengths = [int(x) for x in np.random.default_rng(1).integers(0, 150, 256)]
    c = Case(lpq, 2, 72, 16, lengths, "bf16", seed=21)
    group, new, window, sinks = 5, 9, 40, 3
    assert goes_by_rows(c, group, new)
    q = c.queries(group, new)
    pages = torch.from_numpy(np.stack([[np.r_[c.rng.permutation(12)[:5], -1] for _ in range(2)] for _ in lengths]).astype(np.int32))
    out, lse = c.cache.attend(q.cuda(), ints(lengths), c.table, pages=pages.cuda(), window=window, sinks=sinks, return_lse=True)
    for b in range(0, 256, 7):
        n = lengths[b]
        for h in range(2):
            sees = window_mask(n, new, window, sinks) & np.isin(np.arange(n) // 16, pages[b, h].numpy())[None]
            one = type("Part", (), dict(dim=72, lengths=[n], kcodes=[c.kcodes[b][:, h:h + 1]], vx=[c.vx[b][:, h:h + 1]], kx=[c.kx[b][:, h:h + 1]],
                                        kc=type("Constants", (), dict(s=c.kc.s[h:h + 1], k=c.kc.k[h:h + 1]))))
            part = slice(5 * h, 5 * h + 5)
            check(one, q[b:b + 1, :, part], out[b:b + 1, :, part], lse[b:b + 1, :, part], group, [sees])


def test_what_is_not_seen_missing_pages_and_rows_that_are_not_finite(lpq):
    lengths = [int(x) for x in np.random.default_rng(2).integers(30, 260, 64)]
    c = Case(lpq, 8, 128, 16, lengths, "f16", True, seed=22)
    group, new, window, sinks = 4, 10, 50, 18
    assert goes_by_rows(c, group, new)
    q = c.queries(group, new).cuda()
    want, want_lse = c.cache.attend(q, ints(lengths), c.table, window=window, sinks=sinks, return_lse=True)
    hidden = c.table.clone()
    for b, n in enumerate(lengths):
        seen = window_mask(n, new, window, sinks).any(0)
        for p in range(-(-n // 16)):
            rows = np.flatnonzero(~seen[p * 16:(p + 1) * 16])
            for pool in (c.cache.k, c.cache.v):
                pool[int(c.table_np[b, p]), :, rows.tolist()] = 119
            if len(rows) == len(seen[p * 16:(p + 1) * 16]):
                hidden[b, p] = (-1, c.cache.pages + 5)[p & 1]
    assert (hidden != c.table).sum() > 60
    for table in (c.table, hidden):
        out, lse = c.cache.attend(q, ints(lengths), table, window=window, sinks=sinks, return_lse=True)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    q[:, 3, 7, 5], q[:, 9, 0, 0] = float("nan"), float("inf")
    out, lse = c.cache.attend(q, ints(lengths), hidden, window=window, sinks=sinks, return_lse=True)
    bad = torch.zeros(64, new, 32, dtype=torch.bool, device="cuda")
    bad[:, 3, 7] = bad[:, 9, 0] = True
    assert torch.equal(torch.isnan(lse), bad) and torch.equal(torch.isnan(out), bad[..., None].expand_as(out))
    # the other rows: equal but for where their maximum stood meanwhile, a rounding of weights (2^-11) and of the result (2^-11)
    good = (~bad[..., None]).expand_as(out)
    spread = float(max((v.max(0) - v.min(0)).max() for v in c.vx))
    assert ((out.float() - want.float())[good].abs() <= 2 * 2.0 ** -10 * spread + 2.0 ** -10 * want.float()[good].abs()).all()
    # nothing to see: lengths of 0, below 0, windows behind the table
    for n in (0, -5, -(2 ** 31)):
        out, lse = c.cache.attend(q, ints([n] * 64), c.table, window=window, sinks=sinks, return_lse=True)
        assert not out.any() and torch.isneginf(lse).all()
    room = c.table.shape[1] * 16
    a = c.cache.attend(q, ints([room] * 64), c.table, window=window, sinks=sinks)
    b = c.cache.attend(q, ints([2 ** 31 - 1, room + 1] * 32), c.table, window=window, sinks=sinks)
    assert torch.equal(a.nan_to_num(), b.nan_to_num())


def test_strides_streams_and_graphs(lpq):
    lengths = [int(x) for x in np.random.default_rng(3).integers(0, 200, 64)]
    c = Case(lpq, 8, 72, 32, lengths, "f32", seed=23)
    group, new = 3, 12
    assert goes_by_rows(c, group, new)
    q, n, kw = c.queries(group, new).cuda(), ints(lengths), dict(window=60, sinks=2)
    want = c.cache.attend(q, n, c.table, **kw)
    wide = torch.full((64, 24, new, 80), 5.0, device="cuda")
    out = wide[..., 3:75].permute(0, 2, 1, 3)
    spread = torch.zeros(64, new, 24, 75, device="cuda")
    spread[..., 1:73] = q
    assert c.cache.attend(spread[..., 1:73], n, c.table, out=out, **kw) is out
    assert torch.equal(out, want)
    out.fill_(5.0)
    assert (wide == 5.0).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.cache.attend(q, n, c.table, **kw)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    fed = q.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = c.cache.attend(fed, n, c.table, **kw)
    for i in range(4):
        fed.copy_(q * (i + 1))
        graph.replay()
        assert torch.equal(got, c.cache.attend(q * (i + 1), n, c.table, **kw))
