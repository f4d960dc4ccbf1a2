"""Key-value cache on a real MI355X: codes and bounds as written, what reads back, page selection and attention over all
or listed pages, against the plain definitions in 64 bits (kv_plain.py).  Codes, bounds and selections are integers and
must be equal; attention stays within a bound that is derived from the roundings the kernel makes."""
import numpy as np
import pytest
import torch

import kv_plain as plain

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def lpq():
    from paper_2110_08919_amd import lpq as m
    assert torch.cuda.is_available(), "no GPU visible"
    m.lib()
    return m


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Case:
    """A cache, and what its sequences hold (numpy)."""

    def __init__(self, lpq, heads, dim, page, lengths, kind="bf16", packed=False, bits=None, seed=0, spare=3, write=True):
        self.rng = rng = np.random.default_rng(seed)
        self.heads, self.dim, self.page, self.lengths, self.kind, self.packed = heads, dim, page, list(lengths), kind, packed
        bits = bits or (4 if packed else 8)
        f = heads * dim
        self.mean = 0.5 * rng.standard_normal(f)
        self.std = np.exp(0.4 * rng.standard_normal(f))
        self.std[rng.random(f) < 0.05] *= 6
        width = 4.0 if bits == 8 else 2.5
        ranges = [(m.astype(np.float32), (m - width * self.std).astype(np.float32), (m + width * self.std).astype(np.float32))
                  for m in (self.mean, 0.1 * self.mean)]
        self.kc, self.vc = (plain.Constants(*r, bits, heads) for r in ranges)
        quant = [lpq.Quantizer(f, bits).set_params(*r) for r in ranges]
        counts = [-(-n // page) for n in self.lengths]
        pages = sum(counts) + spare
        order = rng.permutation(pages)
        self.table_np = np.full((len(self.lengths), max(counts + [1])), -1, np.int32)
        at = 0
        for b, c in enumerate(counts):
            self.table_np[b, :c] = order[at:at + c]
            at += c
        self.table = torch.from_numpy(self.table_np).cuda()
        self.cache = lpq.KVCache(*quant, heads=heads, page=page, pages=pages, packed=packed)
        self.k, self.v = [], []
        for n in self.lengths:
            for rows in (self.k, self.v):
                x = torch.from_numpy((rng.standard_normal((n, f)) * self.std + self.mean).astype(np.float32)).to(TYPES[kind])
                rows.append(x.view(n, heads, dim))
        self.kcodes = [plain.codes(x.float().numpy(), self.kc, packed) for x in self.k]
        self.vcodes = [plain.codes(x.float().numpy(), self.vc, packed) for x in self.v]
        self.kx = [plain.values(q, self.kc).astype(np.float64) for q in self.kcodes]
        self.vx = [plain.values(q, self.vc).astype(np.float64) for q in self.vcodes]
        self.starts = np.concatenate([[0], np.cumsum(self.lengths)])
        if write and sum(self.lengths):
            self.cache.write(torch.cat(self.k).cuda(), torch.cat(self.v).cuda(), ints([0] * len(self.lengths)), self.table,
                             ints(self.starts.tolist()))

    def stored(self, b, which):
        """Codes of sequence b as they lie in the pool."""
        pool = (self.cache.k if which == "k" else self.cache.v).cpu().numpy()
        n = self.lengths[b]
        pages = self.table_np[b, :-(-n // self.page)]
        rows = pool[pages].transpose(0, 2, 1, 3).reshape(-1, self.heads, pool.shape[-1])[:n]
        if self.packed:
            rows = np.stack([rows & 15, rows >> 4], -1).reshape(n, self.heads, -1).astype(np.int64) - 8
        assert (rows[..., self.dim:] == 0).all(), "padding must hold code 0"
        return rows[..., :self.dim].astype(np.int64)

    def queries(self, group, new=1, kind=None, strength=2.0):
        kind = kind or self.kind
        q = self.rng.standard_normal((len(self.lengths), new, self.heads, group, self.dim))
        q = strength * q / self.std.reshape(self.heads, 1, self.dim)
        q = torch.from_numpy(q.reshape(len(self.lengths), new, -1, self.dim).astype(np.float32)).to(TYPES[kind])
        return q

    def check_attention(self, q, out, lse, group, scale=None, seen=None, dead=None):
        kind = {v: k for k, v in TYPES.items()}[q.dtype]
        scale = self.dim ** -0.5 if scale is None else scale
        q, out = q.float().numpy(), out.double().cpu().numpy()
        worst = 0.0
        for b, n in enumerate(self.lengths):
            o, want_lse = plain.attend(q[b], self.kx[b], self.vx[b], group, scale, None if seen is None else seen[b],
                                       None if dead is None else dead[b])
            err, lerr = plain.attend_bound(q[b], self.kcodes[b], self.vx[b], self.kc, group, scale, kind)
            empty = np.isinf(want_lse)
            assert (out[b][empty] == 0).all(), "a row that sees nothing is zeros"
            diff = np.abs(out[b] - o)
            assert (diff <= err).all(), (b, n, float((diff - err).max()), float((diff / np.maximum(err, 1e-30)).max()))
            if err.size and err.max() > 0:
                worst = max(worst, float((diff / np.maximum(err, 1e-30)).max()))
            if lse is not None:
                got = lse[b].double().cpu().numpy()
                assert (np.isinf(got) == empty).all() and (got[empty] < 0).all()
                assert (np.abs(got[~empty] - want_lse[~empty]) <= lerr[~empty]).all()
        return worst


SHAPES = [  # heads, dim, page, lengths, type, packed, bits
    (2, 64, 16, [1, 17, 0, 40], "bf16", False, 8),
    (3, 100, 32, [5, 33, 64], "f16", False, 8),
    (1, 128, 64, [130, 1, 64], "f32", False, 8),
    (2, 33, 16, [31, 16], "f32", True, 4),
    (2, 192, 64, [70, 3], "bf16", True, 4),
    (1, 256, 128, [129, 300], "f16", False, 5),
    (4, 80, 256, [257, 10], "bf16", True, 3),
    (1, 1, 16, [20], "f32", False, 8),
]


@pytest.mark.parametrize("heads,dim,page,lengths,kind,packed,bits", SHAPES)
def test_codes_bounds_and_values(lpq, heads, dim, page, lengths, kind, packed, bits):
    c = Case(lpq, heads, dim, page, lengths, kind, packed, bits)
    for b, n in enumerate(lengths):
        assert np.array_equal(c.stored(b, "k"), c.kcodes[b]) and np.array_equal(c.stored(b, "v"), c.vcodes[b])
        if n:
            got = c.cache.bounds.cpu().numpy()[c.table_np[b, :-(-n // page)]]
            assert np.array_equal(got, plain.bounds(c.kcodes[b], page))
    starts = ints(c.starts.tolist())
    for out in ("f32", kind):
        k, v = c.cache.read(ints([0] * len(lengths)), c.table, starts, int(c.starts[-1]), TYPES[out])
        for got, codes, consts in ((k, c.kcodes, c.kc), (v, c.vcodes, c.vc)):
            want = torch.from_numpy(np.concatenate([plain.values(q, consts) for q in codes])).to(TYPES[out])
            assert torch.equal(got.cpu(), want)


def test_special_values_and_features_without_a_range(lpq):
    heads, dim = 2, 40
    k = np.zeros(heads * dim, np.float32)
    sb, se = np.full_like(k, -1), np.full_like(k, 1)
    k[7], sb[7], se[7] = 3.25, 2.0, 2.0                  # no range: code 0, reads back as k
    q = lpq.Quantizer(heads * dim, 8).set_params(k, sb, se)
    cache = lpq.KVCache(q, q, heads=heads, page=16, pages=2)
    x = torch.zeros(1, heads, dim)
    x[0, 0, :6] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.0, -1.0, 2.0])
    cache.write(x.cuda(), x.cuda(), ints([3]), ints([1]).view(1, 1))
    row = cache.k[1, 0, 3].cpu().numpy()
    assert row[:6].tolist() == [0, 127, -128, 127, -128, 127] and row[7] == 0
    got, _ = cache.read(ints([3]), ints([1]).view(1, 1))
    assert got[0, 0, 7].item() == 3.25 and got[0, 1, 0].item() == 0.5 / 128


@pytest.mark.parametrize("packed", [False, True])
def test_token_by_token_and_cut_back(lpq, packed):
    """However tokens are grouped into calls the cache holds the same; a sequence cut back and written on has the bounds
    of what it then holds."""
    c = Case(lpq, 2, 64, 16, [37, 5, 16], packed=packed, write=False)
    other = Case(lpq, 2, 64, 16, [37, 5, 16], packed=packed)
    assert np.array_equal(c.kcodes[0], other.kcodes[0])
    for step in range(37):
        live = [b for b, n in enumerate(c.lengths) if step < n]
        c.cache.write(torch.stack([c.k[b][step] for b in live]).cuda(), torch.stack([c.v[b][step] for b in live]).cuda(),
                      ints([step] * len(live)), c.table[live])
    assert torch.equal(c.cache.k, other.cache.k) and torch.equal(c.cache.v, other.cache.v)
    assert torch.equal(c.cache.bounds, other.cache.bounds)
    # back to 20 tokens, then 2 others: the page of positions 16 .. 21 holds 6
    fresh = (c.k[1][:2] * 3).contiguous()
    c.cache.write(fresh.cuda(), fresh.cuda(), ints([20]), c.table[:1], ints([0, 2]))
    want = np.concatenate([c.kcodes[0][16:20], plain.codes(fresh.float().numpy(), c.kc, packed)])
    got = c.cache.bounds.cpu().numpy()[c.table_np[0, 1]]
    assert np.array_equal(got, plain.bounds(want, 16)[0])


def test_rows_with_strides_and_no_place(lpq):
    """Rows inside a wider tensor, heads before tokens, one row for all; pages and positions that do not exist."""
    c = Case(lpq, 3, 40, 16, [20, 33], "f16")
    wide = torch.zeros(53, 3, 3, 43, dtype=torch.float16)
    wide[:, :, 0, 1:41] = torch.cat(c.k)
    v = torch.cat(c.v).permute(1, 0, 2).contiguous().cuda().permute(1, 0, 2)          # [n, heads, dim], heads outermost
    other = Case(lpq, 3, 40, 16, [20, 33], "f16", write=False)
    other.cache.write(wide.cuda()[:, :, 0, 1:41], v, ints([0, 0]), other.table, ints([0, 20, 53]))
    assert torch.equal(c.cache.k, other.cache.k) and torch.equal(c.cache.v, other.cache.v)
    base = torch.full((53, 3, 100), 7.0, dtype=torch.float16, device="cuda")
    out = torch.zeros(3, 53, 40, dtype=torch.float16, device="cuda").permute(1, 0, 2)
    k, v = c.cache.read(ints([0, 0]), c.table, ints([0, 20, 53]), 53, out=(base[:, :, 5:45], out))
    assert torch.equal(k.cpu().float(), torch.from_numpy(np.concatenate(c.kx)).to(torch.float16).float())
    assert torch.equal(v.cpu().float(), torch.from_numpy(np.concatenate(c.vx)).to(torch.float16).float())
    assert (base[:, :, :5] == 7).all() and (base[:, :, 45:] == 7).all()
    # a row shared by all sequences (stride 0)
    one = c.k[0][:1].cuda().expand(2, -1, -1)
    c.cache.write(one, one, ints([3, 8]), c.table)
    k, _ = c.cache.read(ints([3, 8]), c.table)
    assert torch.equal(k[0], k[1])
    # a page outside the pool, a missing one, positions before 0 and past the table: dropped, and zeros back
    before = c.cache.k.clone(), c.cache.bounds.clone()
    table = torch.tensor([[10 ** 6, -1, -7], [c.cache.pages, -1, -1]], dtype=torch.int32, device="cuda")
    rows = torch.cat(c.k).cuda()
    for first in ([0, 0], [-100, 40], [2 ** 31 - 60, 47]):
        c.cache.write(rows, rows, ints(first), table, ints([0, 20, 53]))
        k, v = c.cache.read(ints(first), table, ints([0, 20, 53]), 53)
        assert not k.any() and not v.any()
    assert torch.equal(before[0], c.cache.k) and torch.equal(before[1], c.cache.bounds)
    # positions -2, -1 are dropped, 0 and 1 written
    c.cache.write(rows[10:14], rows[10:14], ints([-2]), c.table[:1], ints([0, 4]))
    k, _ = c.cache.read(ints([-2]), c.table[:1], ints([0, 4]), 4)
    assert not k[:2].any() and torch.equal(k[2:].cpu(), torch.from_numpy(plain.values(c.kcodes[0][12:14], c.kc)))
    # nothing to do
    c.cache.write(rows[:0], rows[:0], ints([0, 0]), c.table, ints([0, 0, 0]))
    none = torch.zeros(0, 3, dtype=torch.int32, device="cuda")
    c.cache.write(rows[:0], rows[:0], ints([]), none)
    assert c.cache.read(ints([]), none)[0].shape == (0, 3, 40)
    assert c.cache.attend(c.queries(2)[:0].cuda(), ints([]), none).shape == (0, 1, 6, 40)
    assert c.cache.select(c.queries(2)[:0].cuda(), ints([]), none, 2).shape == (0, 3, 2)


SELECT = [  # heads, dim, page, lengths, group, new, n_select, keep_first, keep_last, packed
    (2, 64, 16, [1, 0, 300, 17], 1, 1, 4, 1, 1, False),
    (1, 100, 32, [2000, 31], 4, 1, 7, 0, 1, False),
    (3, 128, 16, [900], 2, 4, 60, 2, 3, True),
    (1, 192, 16, [5000, 4000], 8, 2, 33, 0, 0, True),
    (2, 256, 64, [700], 16, 1, 1, 0, 1, False),
    (1, 40, 16, [20000], 1, 1, 100, 1, 1, False),          # 1250 pages
    (2, 128, 16, [8100, 5000], 3, 1, 40, 1, 1, False),     # 507 pages
    (1, 256, 16, [9000, 16000], 2, 1, 600, 1, 1, True),    # 1000 pages, and fewer than asked for
    (1, 64, 16, [40000, 100], 1, 1, 64, 0, 1, False),      # 2500 pages
    (1, 64, 16, [80000], 2, 1, 700, 3, 3, False),          # 5000 pages
    (1, 64, 16, [400], 16, 8, 9, 0, 0, False),             # 128 query rows
]


@pytest.mark.parametrize("heads,dim,page,lengths,group,new,n_select,first,last,packed", SELECT)
def test_selection_equals_the_definition(lpq, heads, dim, page, lengths, group, new, n_select, first, last, packed):
    c = Case(lpq, heads, dim, page, lengths, packed=packed)
    q = c.queries(group, new)
    got = c.cache.select(q.cuda(), ints(lengths), c.table, n_select, first, last).cpu().numpy()
    for b, n in enumerate(lengths):
        want = plain.select(q[b].float().numpy(), c.kcodes[b], c.kc, page, n_select, first, last, group)
        for h in range(heads):
            w = (want[h] if n else [])
            assert got[b, h].tolist() == w + [-1] * (n_select - len(w)), (b, h)


def test_selection_ties_missing_pages_and_queries_that_are_not_finite(lpq):
    c = Case(lpq, 1, 64, 16, [640])
    same = c.k[0][:16].repeat(40, 1, 1).cuda()
    c.cache.write(same, same, ints([0]), c.table, ints([0, 640]))
    q = c.queries(2)
    got = c.cache.select(q.cuda(), ints([640]), c.table, 7, 0, 2).cpu()[0, 0].tolist()
    assert got == [0, 1, 2, 3, 4, 38, 39]                  # equal scores: the lowest pages, and the two kept ones
    table = c.table.clone()
    table[0, 1] = -1
    table[0, 3] = c.cache.pages
    table[0, 39] = -5
    got = c.cache.select(q.cuda(), ints([640]), table, 7, 0, 2).cpu()[0, 0].tolist()
    assert got == [0, 2, 4, 5, 6, 7, 38]
    got = c.cache.select(q.cuda(), ints([640]), table, 64, 0, 2).cpu()[0, 0].tolist()
    assert got == [p for p in range(40) if p not in (1, 3, 39)] + [-1] * 27
    c = Case(lpq, 1, 64, 16, [640], seed=5)
    q = c.queries(4)
    q[0, 0, 1, 3], q[0, 0, 2, 9], q[0, 0, 3, 1] = float("nan"), float("inf"), -float("inf")
    got = c.cache.select(q.cuda(), ints([640]), c.table, 5, 0, 1).cpu()[0, 0].tolist()
    assert got == plain.select(q[0].float().numpy(), c.kcodes[0], c.kc, 16, 5, 0, 1, 4)[0]
    got = c.cache.select(torch.zeros_like(q).cuda(), ints([640]), c.table, 5, 0, 1).cpu()[0, 0].tolist()
    assert got == [0, 1, 2, 3, 39]
    # lengths beyond the table and below 0
    got = c.cache.select(q.cuda(), ints([10 ** 6]), c.table, 40, 0, 1).cpu()[0, 0].tolist()
    assert got == list(range(40))
    assert c.cache.select(q.cuda(), ints([-3]), c.table, 2, 0, 1).cpu()[0, 0].tolist() == [-1, -1]


def test_selection_of_more_pages_than_a_workgroup_holds(lpq):
    """18 000 columns; the table names few pages of the pool, many times over, so that most scores tie."""
    c = Case(lpq, 1, 64, 16, [16 * 300])
    rng = np.random.default_rng(3)
    columns = rng.integers(0, 300, 18000).astype(np.int32)
    columns[[5, 17000]] = -1
    table = torch.from_numpy(np.where(columns < 0, -1, c.table_np[0][columns])).int().view(1, -1).cuda()
    q = c.queries(2)
    codes = c.kcodes[0].reshape(300, 16, 1, 64)[columns].reshape(-1, 1, 64)
    for n_select in (50, 700, 17000):
        got = c.cache.select(q.cuda(), ints([18000 * 16]), table, n_select, 1, 1).cpu()[0, 0].tolist()
        assert got == plain.select(q[0].float().numpy(), codes, c.kc, 16, n_select, 1, 1, 2, columns >= 0)[0]


ATTEND = [  # heads, dim, page, lengths, group, new, type, packed
    (2, 64, 16, [1, 0, 63, 64, 65], 1, 1, "bf16", False),
    (1, 128, 64, [700, 255, 256, 257, 3], 4, 1, "bf16", False),
    (2, 100, 32, [333, 31], 3, 1, "f16", False),
    (1, 192, 16, [130, 33, 1], 12, 4, "f32", True),
    (3, 80, 64, [200, 7], 5, 3, "bf16", True),
    (1, 256, 128, [500, 128], 16, 2, "f16", False),
    (1, 256, 16, [90, 300], 2, 1, "f32", False),
    (2, 33, 16, [45, 2], 1, 4, "f32", False),             # more new tokens than tokens
    (1, 64, 256, [2000], 40, 1, "f32", True),
    (1, 192, 32, [400], 8, 9, "bf16", False),             # 72 query rows
    (1, 128, 64, [9000, 300], 8, 1, "f16", True),         # parts of a long sequence
    (4, 128, 32, [6000], 1, 1, "f32", False),
    (1, 1, 16, [50], 2, 1, "f32", False),
]


@pytest.mark.parametrize("heads,dim,page,lengths,group,new,kind,packed", ATTEND)
def test_attention(lpq, heads, dim, page, lengths, group, new, kind, packed):
    c = Case(lpq, heads, dim, page, lengths, kind, packed)
    q = c.queries(group, new)
    out, lse = c.cache.attend(q.cuda(), ints(lengths), c.table, return_lse=True)
    worst = c.check_attention(q, out, lse, group)
    print(f"worst error / bound {worst:.3f}")
    again = c.cache.attend(q.cuda(), ints(lengths), c.table)
    assert torch.equal(out, again)                         # fixed order of sums


@pytest.mark.parametrize("heads,dim,page,lengths,group,new,kind,packed", ATTEND[:-1])
def test_attention_over_listed_pages(lpq, heads, dim, page, lengths, group, new, kind, packed):
    c = Case(lpq, heads, dim, page, lengths, kind, packed, seed=1)
    q = c.queries(group, new)
    columns = c.table.shape[1]
    take = min(columns, 5) + 2
    pages = np.full((len(lengths), heads, take), -1, np.int32)
    seen = []
    for b, n in enumerate(lengths):
        have = -(-n // page)
        seen.append([])
        for h in range(heads):
            some = c.rng.permutation(have)[:min(have, take - 2)]
            if len(some) > 1 and h == 0:
                some = some[1:]
            slots = c.rng.permutation(take)[:len(some)]    # in any order, with gaps
            pages[b, h, slots] = some
            seen[b].append(np.concatenate([np.arange(p * page, min(n, (p + 1) * page)) for p in some] + [np.zeros(0, int)]))
    pages[0, 0][pages[0, 0] < 0] = columns + 9             # outside the table: none
    out, lse = c.cache.attend(q.cuda(), ints(lengths), c.table, pages=torch.from_numpy(pages).cuda(), return_lse=True)
    c.check_attention(q, out, lse, group, seen=seen)


def test_attention_over_selected_pages_is_attention_over_all_of_them(lpq):
    c = Case(lpq, 2, 128, 16, [200, 37])
    q = c.queries(4)
    pages = c.cache.select(q.cuda(), ints(c.lengths), c.table, 13, 0, 1)
    out, lse = c.cache.attend(q.cuda(), ints(c.lengths), c.table, pages=pages, return_lse=True)
    c.check_attention(q, out, lse, 4)


def test_attention_masks_and_missing_pages(lpq):
    c = Case(lpq, 1, 64, 16, [100, 40], "f16", seed=2)
    q = c.queries(2)
    # every code outside the lengths set to the largest: what is masked must not count
    c.cache.v.fill_(127)
    c.cache.k.fill_(127)
    c.cache.write(torch.cat(c.k).cuda(), torch.cat(c.v).cuda(), ints([0, 0]), c.table, ints(c.starts.tolist()))
    out, lse = c.cache.attend(q.cuda(), ints(c.lengths), c.table, return_lse=True)
    c.check_attention(q, out, lse, 2)
    table = c.table.clone()
    table[0, 2], table[1, 0] = -1, c.cache.pages + 100
    dead = [np.arange(100) // 16 == 2, np.arange(40) // 16 == 0]
    out, lse = c.cache.attend(q.cuda(), ints(c.lengths), table, return_lse=True)
    c.check_attention(q, out, lse, 2, dead=dead)
    table[1] = -1
    out, lse = c.cache.attend(q.cuda(), ints(c.lengths), table, return_lse=True)
    assert not out[1].any() and torch.isneginf(lse[1]).all() and torch.isfinite(out).all()
    out, lse = c.cache.attend(q.cuda(), ints([-5, 0]), c.table, return_lse=True)
    assert not out.any() and torch.isneginf(lse).all()
    # lengths beyond the table end with it
    a = c.cache.attend(q.cuda(), ints([7 * 16, 7 * 16]), c.table)
    b = c.cache.attend(q.cuda(), ints([10 ** 9, 7 * 16]), c.table)
    assert torch.equal(a, b)


def test_attention_of_queries_that_are_not_finite_or_zero(lpq):
    c = Case(lpq, 1, 128, 64, [300], "bf16", seed=3)
    q = c.queries(4)
    clean = c.cache.attend(q.cuda(), ints([300]), c.table)
    bad = q.clone()
    bad[0, 0, 1, 5], bad[0, 0, 2, 100] = float("nan"), float("inf")
    out = c.cache.attend(bad.cuda(), ints([300]), c.table)
    assert torch.isnan(out[0, 0, [1, 2]]).all()
    assert torch.equal(out[0, 0, [0, 3]], clean[0, 0, [0, 3]])          # the other rows are not touched
    q.zero_()
    out, lse = c.cache.attend(q.cuda(), ints([300]), c.table, return_lse=True)
    c.check_attention(q, out, lse, 4)                                    # the mean of the values
    q = c.queries(4, strength=300.0)                                     # one token takes all
    out, lse = c.cache.attend(q.cuda(), ints([300]), c.table, return_lse=True)
    c.check_attention(q, out, lse, 4)


@pytest.mark.parametrize("order", [1, -1])
def test_attention_where_the_maximum_keeps_moving(lpq, order):
    """Scores that rise (or fall) along the sequence by far more than the head room of the running maximum."""
    c = Case(lpq, 1, 64, 16, [3000], "f32", seed=4)
    ramp = torch.linspace(-3.5, 3.5, 3000)[:: order].contiguous() if order == 1 else torch.linspace(3.5, -3.5, 3000)
    k = (ramp[:, None] * torch.from_numpy(c.std)[None]).float().add(torch.from_numpy(c.mean).float()).view(3000, 1, 64)
    c.cache.write(k.cuda(), c.v[0].cuda(), ints([0]), c.table, ints([0, 3000]))
    c.kcodes = [plain.codes(k.numpy(), c.kc, False)]
    c.kx = [plain.values(c.kcodes[0], c.kc).astype(np.float64)]
    q = torch.from_numpy((4.0 / c.std).astype(np.float32)).view(1, 1, 1, 64)
    out, lse = c.cache.attend(q.cuda(), ints([3000]), c.table, return_lse=True)
    c.check_attention(q, out, lse, 1)


def test_queries_and_outputs_with_strides_scale_and_parts_joined_by_lse(lpq):
    c = Case(lpq, 2, 72, 16, [150, 90], "f32", seed=6)
    q = c.queries(3, 2)
    wide = torch.zeros(2, 2, 6, 3, 75)
    wide[:, :, :, 1, 2:74] = q
    strided = wide.cuda()[:, :, :, 1, 2:74]
    base = torch.full((2, 6, 2, 80), 5.0, device="cuda")
    out, lse = c.cache.attend(strided, ints(c.lengths), c.table, scale=0.31, out=base.permute(0, 2, 1, 3)[..., 4:76], return_lse=True)
    c.check_attention(q, out, lse, 3, scale=0.31)
    assert (base[..., :4] == 5).all() and (base[..., 76:] == 5).all()
    # attention over two halves of the pages, joined
    pages = torch.arange(10, dtype=torch.int32, device="cuda").expand(2, 2, 10)
    parts = [c.cache.attend(q.cuda(), ints(c.lengths), c.table, pages=p.contiguous(), scale=0.31, return_lse=True)
             for p in (pages[..., :4], pages[..., 4:])]
    both = torch.stack([p[1] for p in parts])
    w = torch.softmax(both, 0)[..., None]
    joined = (w * torch.stack([p[0] for p in parts])).sum(0)
    assert torch.allclose(joined, out, rtol=1e-4, atol=1e-4)


def test_offsets_beyond_32_bits(lpq):
    """A pool of 4.3 GB of keys and as much of values, the sequences on its last and first pages."""
    heads, dim, page = 8, 128, 64
    c = Case(lpq, heads, dim, page, [200, 130], seed=7)
    pages = (1 << 32) // (heads * dim * page) + 40
    f = heads * dim
    quant = [lpq.Quantizer(f, 8).set_params(k.k.reshape(-1), k.sb.reshape(-1), k.se.reshape(-1)) for k in (c.kc, c.vc)]
    big = lpq.KVCache(*quant, heads=heads, page=page, pages=pages)
    assert big.k.numel() > 1 << 32
    table = torch.tensor([[pages - 1, 0, pages - 2, pages - 20], [pages // 2 + 1, pages - 3, 1, -1]], dtype=torch.int32, device="cuda")
    big.write(torch.cat(c.k).cuda(), torch.cat(c.v).cuda(), ints([0, 0]), table, ints(c.starts.tolist()))
    k, v = big.read(ints([0, 0]), table, ints(c.starts.tolist()), 330)
    assert np.array_equal(k.cpu().numpy(), np.concatenate(c.kx).astype(np.float32))
    assert np.array_equal(v.cpu().numpy(), np.concatenate(c.vx).astype(np.float32))
    q = c.queries(4)
    out, lse = big.attend(q.cuda(), ints(c.lengths), table, return_lse=True)
    c.check_attention(q, out, lse, 4)
    got = big.select(q.cuda(), ints(c.lengths), table, 2).cpu().numpy()
    for b in range(2):
        want = plain.select(q[b].float().numpy(), c.kcodes[b], c.kc, page, 2, 0, 1, 4)
        assert got[b].tolist() == want


def test_another_stream_and_a_captured_graph(lpq):
    """A generation step (write, select, attend) on a stream of its own and replayed from a graph."""
    c = Case(lpq, 2, 128, 16, [100, 400], seed=8)
    q, lengths = c.queries(4).cuda(), ints(c.lengths)
    k, v = (torch.stack([r[b][-1] for b in range(2)]).cuda() for r in (c.k, c.v))
    first = lengths - 1

    def step():
        c.cache.write(k, v, first, c.table)
        pages = c.cache.select(q, lengths, c.table, 6, 1, 1)
        return pages, c.cache.attend(q, lengths, c.table, pages=pages), c.cache.attend(q, lengths, c.table)

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for turn in range(3):
        q.copy_(c.queries(4))
        lengths.sub_(turn)
        first.sub_(turn)
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), turn


def test_refusals(lpq):
    c = Case(lpq, 2, 64, 16, [40, 20])
    rows = torch.cat(c.k).cuda()
    first, starts, lengths, q = ints([0, 0]), ints([0, 40, 60]), ints([40, 20]), c.queries(2).cuda()
    def code(fn, *a, **kw):
        with pytest.raises(lpq.LpqError) as e:
            fn(*a, **kw)
        assert str(e.value).count(":") >= 1
        return e.value.code
    cache = c.cache
    quant = lambda d, bits=8: lpq.Quantizer(d, bits).set_params(*[np.full(d, x, np.float32) for x in (0, -1, 1)])
    good = quant(128)
    assert code(lpq.KVCache, good, good, heads=2, page=24, pages=4) == lpq.EINVAL
    assert code(lpq.KVCache, good, good, heads=2, page=512, pages=4) == lpq.EINVAL
    assert code(lpq.KVCache, good, good, heads=2, page=16, pages=0) == lpq.EINVAL
    assert code(lpq.KVCache, good, good, heads=2, page=16, pages=4, packed=True) == lpq.EINVAL     # 8 bits
    assert code(lpq.KVCache, good, quant(130), heads=2, page=16, pages=4) == lpq.EINVAL
    assert code(lpq.KVCache, quant(600), quant(600), heads=2, page=16, pages=4) == lpq.ERANGE      # 300 features
    assert code(lpq.KVCache, lpq.Quantizer(128, 8), good, heads=2, page=16, pages=4) == lpq.ESTATE
    before = cache.k.clone()
    assert code(cache.write, rows, rows, first, c.table) == lpq.EINVAL                             # 60 rows, 2 sequences
    assert code(cache.read, first, c.table, starts, 60,
                out=(rows[:1].expand(60, -1, -1), rows.clone())) == lpq.EINVAL                     # outputs on top of each other
    assert code(cache.select, q, lengths, c.table, 0) == lpq.EINVAL
    assert code(cache.select, q, lengths, c.table, 2, 2, 1) == lpq.EINVAL
    assert code(cache.select, q, lengths, c.table, 2, -1, 1) == lpq.EINVAL
    assert code(cache.select, q[:, :, :3], lengths, c.table, 2) == lpq.EINVAL                      # 3 query heads on 2
    assert code(cache.select, c.queries(20, 7).cuda(), lengths, c.table, 2) == lpq.ERANGE          # 140 query rows
    wide = torch.full((2, 600), -1, dtype=torch.int32, device="cuda")                              # columns enough for a workspace
    assert code(cache.select, q, lengths, wide, 2, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")) == lpq.ERANGE
    assert code(cache.attend, q, lengths, c.table, scale=float("nan")) == lpq.EINVAL
    assert code(cache.attend, q[:, :, :1], lengths, c.table) == lpq.EINVAL
    assert code(cache.attend, q, lengths, c.table, out=torch.empty_like(q[:1]).expand(2, -1, -1, -1)) == lpq.EINVAL
    long = Case(lpq, 1, 64, 16, [3000])
    ql = long.queries(2).cuda()
    assert code(long.cache.attend, ql, ints([3000]), long.table, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")) == lpq.ERANGE
    room = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    assert code(long.cache.attend, ql, ints([3000]), long.table, workspace=room[1:]) == lpq.EINVAL
    long.cache.attend(ql, ints([3000]), long.table, workspace=room)
    for bad in (dict(q=q.cpu()), dict(q=q.double()), dict(q=q[..., :60]), dict(lengths=lengths.long()), dict(lengths=lengths[:1])):
        with pytest.raises(AssertionError):
            cache.attend(bad.get("q", q), bad.get("lengths", lengths), c.table)
    assert torch.equal(before, cache.k)


@pytest.mark.parametrize("scale", [-0.4, 0.0, -0.0, 1e-33, 2.5])
@pytest.mark.parametrize("kind,packed", [("f32", False), ("f16", True), ("bf16", False)])
def test_scales_of_any_sign(lpq, kind, packed, scale):
    c = Case(lpq, 2, 96, 16, [70, 5], kind, packed, seed=11)
    q = c.queries(3, 2, strength=0.3)
    out, lse = c.cache.attend(q.cuda(), ints(c.lengths), c.table, scale=scale, return_lse=True)
    c.check_attention(q, out, lse, 3, scale=scale)


def test_many_small_weights_beside_a_large_one(lpq):
    """30 000 tokens whose weights are 2^-30 to 2^-24 of one token's: together they still move the result."""
    n = 30_000
    c = Case(lpq, 1, 64, 64, [n], "f32", seed=12)
    k = np.broadcast_to(c.mean, (n, 64)) + 0.05 * c.std * c.rng.standard_normal((n, 64))
    k[17] = c.mean + 3.0 * c.std
    k = torch.from_numpy(k.astype(np.float32)).view(n, 1, 64)
    c.cache.write(k.cuda(), c.v[0].cuda(), ints([0]), c.table, ints([0, n]))
    c.kcodes = [plain.codes(k.numpy(), c.kc, False)]
    c.kx = [plain.values(c.kcodes[0], c.kc).astype(np.float64)]
    q = torch.from_numpy((0.8 / c.std).astype(np.float32)).view(1, 1, 1, 64)
    out, lse = c.cache.attend(q.cuda(), ints([n]), c.table, return_lse=True)
    c.check_attention(q, out, lse, 1)


@pytest.mark.parametrize("heads,dim,page,kind,packed", [(3, 64, 128, "bf16", False), (7, 192, 32, "f16", True), (2, 33, 16, "f32", False)])
def test_few_rows_of_many_sequences(lpq, heads, dim, page, kind, packed):
    rng = np.random.default_rng(5)
    lengths = [int(x) for x in rng.integers(0, 12, 150)] + [page, 2 * page + 1]
    before = [int(rng.integers(0, n + 1)) for n in lengths]
    c = Case(lpq, heads, dim, page, lengths, kind, packed, write=False, seed=13)
    for part in (0, 1):
        span = [(0, a) if part == 0 else (a, n) for a, n in zip(before, lengths)]
        k, v = (torch.cat([x[a:e] for x, (a, e) in zip(rows, span)]).cuda() for rows in (c.k, c.v))
        first, starts = [a for a, _ in span], np.concatenate([[0], np.cumsum([e - a for a, e in span])]).tolist()
        c.cache.write(k, v, ints(first), c.table, ints(starts))
        back = c.cache.read(ints(first), c.table, ints(starts), starts[-1])
        for got, codes, consts in ((back[0], c.kcodes, c.kc), (back[1], c.vcodes, c.vc)):
            want = plain.values(np.concatenate([x[a:e] for x, (a, e) in zip(codes, span)]), consts)
            assert np.array_equal(got.cpu().numpy(), want)
    bounds = c.cache.bounds.cpu().numpy()
    for b, n in enumerate(lengths):
        if n == 0:
            continue
        assert np.array_equal(c.stored(b, "k"), c.kcodes[b]) and np.array_equal(c.stored(b, "v"), c.vcodes[b])
        for p in range(-(-n // page)):
            codes = c.kcodes[b][p * page:(p + 1) * page]
            assert np.array_equal(bounds[c.table_np[b, p]], np.stack([codes.min(0), codes.max(0)], 1))


@pytest.mark.parametrize("heads,dim,page,lengths,group,new,kind,packed", [
    (1, 192, 16, [130, 33, 1], 12, 4, "f32", True),
    (1, 256, 128, [500, 128], 16, 2, "f16", False),
    (1, 64, 256, [2000, 0], 40, 1, "f32", True),
    (1, 192, 32, [400], 8, 9, "bf16", False),
    (2, 128, 32, [300, 70], 20, 1, "bf16", True),
    (1, 128, 64, [700, 90], 24, 1, "f32", False),
    (1, 128, 16, [333, 16], 9, 4, "f32", True),
    (1, 256, 16, [260, 40], 6, 3, "f16", True),
    (1, 256, 64, [90, 300], 17, 1, "f32", True),
    (2, 50, 16, [45, 2], 6, 4, "bf16", False),
])
def test_attention_of_many_rows_in_tables_with_room_for_long_sequences(lpq, heads, dim, page, lengths, group, new, kind, packed):
    """What a table has room for decides how a call is shared out, and how many rows go through a tile at a time."""
    c = Case(lpq, heads, dim, page, lengths, kind, packed, seed=14)
    q = c.queries(group, new)
    columns = (1 << 20) // (page * heads * len(lengths))
    table = torch.full((len(lengths), columns), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    out, lse = c.cache.attend(q.cuda(), ints(lengths), table, return_lse=True)
    c.check_attention(q, out, lse, group)
    short, short_lse = c.cache.attend(q.cuda(), ints(lengths), c.table, return_lse=True)
    c.check_attention(q, short, short_lse, group)
