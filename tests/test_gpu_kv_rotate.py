"""Keys and queries turned by the angles of their positions on the way into a key-value cache, on a real MI355X.  Each of the definition's operations is
rounded to binary32, so codes, bounds and turned queries must be equal to the plain definition's (numpy)."""
import numpy as np
import pytest
import torch

import kv_plain as plain
from test_gpu_kv_cache import TYPES, Case, ints, lpq  # noqa: F401  (lpq is a fixture)

pytestmark = pytest.mark.gpu


def table_of_angles(count, rotated, seed=0):
    """cos and sin float32 [count, rotated / 2]; scaled a little, as extended contexts have it."""
    half = rotated // 2
    at = np.arange(count)[:, None] * 10000.0 ** (-np.arange(half) / half)[None]
    scale = 1.0 + 0.1 * (seed % 3)
    return (scale * np.cos(at)).astype(np.float32), (scale * np.sin(at)).astype(np.float32)


def turn(x, cos, sin, at, interleaved):
    """x float32 [n, heads, dim], at [n]: below 0 not turned, beyond the table NaN."""
    half = cos.shape[1]
    first = np.arange(half) * (2 if interleaved else 1)
    second = first + (1 if interleaved else half)
    out = x.astype(np.float32).copy()
    on, off = at >= 0, at >= len(cos)
    c, s = (t[np.clip(at, 0, len(cos) - 1)][:, None] for t in (cos, sin))
    a, b = out[..., first], out[..., second]
    with np.errstate(invalid="ignore", over="ignore"):
        na, nb = a * c - b * s, b * c + a * s
    na[off], nb[off] = np.nan, np.nan
    out[..., first] = np.where(on[:, None, None], na, a)
    out[..., second] = np.where(on[:, None, None], nb, b)
    return out


def equal(got, want):
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))


class Rotated:
    """New rows for a Case's sequences, behind `before` tokens of each, with queries and angles."""

    def __init__(self, c, group, before, added, rotated, interleaved, count=None, positions=None):
        self.c, self.interleaved = c, interleaved
        kind = TYPES[c.kind]
        self.n, f = sum(added), c.heads * c.dim
        draw = lambda width: torch.from_numpy((c.rng.standard_normal((self.n, width)) * np.resize(c.std, width)).astype(np.float32)).to(kind)
        self.k, self.v = (draw(f).view(self.n, c.heads, c.dim) for _ in range(2))
        self.q = draw(f * group).view(self.n, c.heads * group, c.dim)
        self.before, self.added = before, added
        self.first = np.asarray(before, np.int64)
        self.starts = np.concatenate([[0], np.cumsum(added)]).astype(np.int64)
        self.at = np.concatenate([b + np.arange(a) for b, a in zip(before, added)]) if self.n else np.zeros(0, np.int64)
        self.positions = positions(self.at) if positions else None
        self.angle = self.at if self.positions is None else self.positions
        self.cos, self.sin = table_of_angles(count or int(max([0, *self.angle])) + 1, rotated, rotated)

    def call(self, cache, table, starts=True, out=None, q=True, **kw):
        return cache.write_rotated(kw.get("k", self.k.cuda()), kw.get("v", self.v.cuda()), ints(self.first.tolist()), table,
                                   torch.from_numpy(self.cos).cuda(), torch.from_numpy(self.sin).cuda(),
                                   starts=ints(self.starts.tolist()) if starts else None,
                                   positions=None if self.positions is None else ints(self.positions.tolist()),
                                   q=kw.get("queries", self.q.cuda()) if q else None, out=out, interleaved=self.interleaved)

    def turned(self, x):
        return turn(x.float().numpy(), self.cos, self.sin, self.angle, self.interleaved)

    def want_queries(self):
        return torch.from_numpy(self.turned(self.q)).to(self.q.dtype)


SHAPES = [  # heads, dim, page, group, type, packed, rotated, interleaved
    (2, 64, 16, 1, "bf16", False, 64, False),
    (8, 128, 64, 4, "bf16", False, 128, False),
    (3, 100, 32, 2, "f16", True, 100, False),             # halves of 50 features
    (3, 100, 32, 2, "f16", False, 52, True),
    (1, 128, 64, 8, "f32", False, 64, False),             # half of a head
    (2, 33, 16, 3, "f32", True, 32, True),                # an odd feature behind
    (2, 33, 16, 3, "bf16", False, 22, False),             # 11 and 11 and 11
    (1, 192, 64, 5, "bf16", True, 2, False),              # one pair, 1 apart
    (1, 256, 128, 1, "f16", False, 256, True),
    (1, 256, 256, 2, "f32", True, 250, False),
    (5, 80, 16, 6, "bf16", True, 14, True),
    (1, 2, 16, 1, "f32", False, 2, True),
    (2, 7, 16, 2, "f16", False, 6, False),                # 3 and 3 in one run of 8
    (2, 90, 32, 1, "bf16", False, 84, False),
]
LENGTHS = [([0], [1]), ([5, 40, 0, 15], [20, 0, 33, 1]), ([0, 100, 7], [300, 3, 129])]


@pytest.mark.parametrize("before,added", LENGTHS)
@pytest.mark.parametrize("heads,dim,page,group,kind,packed,rotated,interleaved", SHAPES)
def test_codes_bounds_and_queries(lpq, heads, dim, page, group, kind, packed, rotated, interleaved, before, added):
    c = Case(lpq, heads, dim, page, [b + a for b, a in zip(before, added)], kind, packed, seed=dim)
    r = Rotated(c, group, before, added, rotated, interleaved)
    q = r.q.cuda()
    out = r.call(c.cache, c.table, queries=q)
    assert equal(out.cpu(), r.want_queries()) and torch.equal(q.cpu(), r.q)
    kcodes, vcodes = plain.codes(r.turned(r.k), c.kc, packed), plain.codes(r.v.float().numpy(), c.vc, packed)
    for b, (n, m) in enumerate(zip(before, added)):
        rows = slice(int(r.starts[b]), int(r.starts[b + 1]))
        want = np.concatenate([c.kcodes[b][:n], kcodes[rows]])
        assert np.array_equal(c.stored(b, "k"), want)
        assert np.array_equal(c.stored(b, "v"), np.concatenate([c.vcodes[b][:n], vcodes[rows]]))
        got = c.cache.bounds.cpu().numpy()[c.table_np[b, :-(-(n + m) // page)]]
        assert np.array_equal(got, plain.bounds(want, page))
    # without queries, and with them where they lie
    again = Case(lpq, heads, dim, page, c.lengths, kind, packed, seed=dim)
    assert r.call(again.cache, again.table, q=False) is None
    assert torch.equal(again.cache.k, c.cache.k) and torch.equal(again.cache.v, c.cache.v) and torch.equal(again.cache.bounds, c.cache.bounds)
    assert r.call(again.cache, again.table, queries=q, out=q) is q
    assert equal(q.cpu(), r.want_queries())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind,heads,dim,group", [("bf16", 2, 64, 4), ("f32", 3, 50, 1), ("f16", 1, 128, 16)])
def test_one_row_for_each_of_many_sequences(lpq, kind, heads, dim, group, interleaved):
    rng = np.random.default_rng(1)
    before = [int(x) for x in rng.integers(0, 90, 300)]
    c = Case(lpq, heads, dim, 16, [b + 1 for b in before], kind, seed=2)
    r = Rotated(c, group, before, [1] * 300, dim // 2 * 2, interleaved)
    out = r.call(c.cache, c.table, starts=False)
    assert equal(out.cpu(), r.want_queries())
    kcodes = plain.codes(r.turned(r.k), c.kc, False)
    for b in range(0, 300, 7):
        assert np.array_equal(c.stored(b, "k"), np.concatenate([c.kcodes[b][:-1], kcodes[b:b + 1]]))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind,dim,rotated", [("f32", 64, 40), ("bf16", 100, 100), ("f16", 33, 10)])
def test_positions_that_are_given(lpq, kind, dim, rotated, interleaved):
    """Positions of drafted tokens, ones below 0 (not turned) and beyond the angles (NaN, code 0)."""
    before, added = [30, 4], [17, 40]

    def positions(at):
        p = at // 2
        p[[3, 20, 41]] = [-1, -(2 ** 31), 60]
        p[[5, 30]] = [61, 2 ** 31 - 1]
        return p
    c = Case(lpq, 2, dim, 16, [47, 44], kind, seed=3)
    r = Rotated(c, 3, before, added, rotated, interleaved, count=61, positions=positions)
    out = r.call(c.cache, c.table)
    want = r.want_queries()
    assert torch.isnan(want[5]).any() and torch.isnan(want[30]).any() and not torch.isnan(want[[3, 20, 41]]).any()
    assert equal(out.cpu(), want) and torch.equal(out[3].cpu(), r.q[3])
    kcodes = plain.codes(r.turned(r.k), c.kc, False)
    for b in range(2):
        rows = slice(int(r.starts[b]), int(r.starts[b + 1]))
        assert np.array_equal(c.stored(b, "k"), np.concatenate([c.kcodes[b][:before[b]], kcodes[rows]]))


@pytest.mark.parametrize("starts", [[0, 20, 40], [5, 20, 53], [0, 0, 0], [53, 53, 53], [3, 8, 8]])
def test_rows_of_no_sequence_stay_as_they_are(lpq, starts):
    c = Case(lpq, 2, 64, 16, [40, 60], "bf16", seed=4)
    r = Rotated(c, 2, [0, 0], [20, 33], 64, False, count=100)
    r.starts = np.asarray(starts)
    r.angle = np.full(53, -1)
    for b in range(2):
        r.angle[starts[b]:starts[b + 1]] = np.arange(starts[b + 1] - starts[b])
    before = c.cache.k.clone()
    q = r.q.cuda()
    out = r.call(c.cache, c.table, queries=q)
    assert equal(out.cpu(), r.want_queries()) and torch.equal(out.cpu()[r.angle < 0], r.q[r.angle < 0])
    r.call(c.cache, c.table, queries=q, out=q)
    assert equal(q.cpu(), r.want_queries())
    kcodes = plain.codes(r.turned(r.k), c.kc, False)
    for b in range(2):
        got, m = c.stored(b, "k"), starts[b + 1] - starts[b]
        assert np.array_equal(got[:m], kcodes[starts[b]:starts[b + 1]]) and np.array_equal(got[m:], c.kcodes[b][m:])
    if starts[2] == starts[0]:
        assert torch.equal(before, c.cache.k)


def test_sequences_that_begin_below_0_or_have_no_pages(lpq):
    c = Case(lpq, 1, 64, 16, [40, 20], "f32", seed=5)
    r = Rotated(c, 2, [-3, 5], [10, 12], 64, False, count=30)
    table = c.table.clone()
    table[1] = -1
    before = c.stored(1, "k")
    out = r.call(c.cache, table)
    assert equal(out.cpu(), r.want_queries()) and torch.equal(out[:3].cpu(), r.q[:3])      # turned whether or not there is a page
    kcodes = plain.codes(r.turned(r.k), c.kc, False)
    assert np.array_equal(c.stored(0, "k")[:7], kcodes[3:10]) and np.array_equal(c.stored(0, "k")[7:], c.kcodes[0][7:])
    assert np.array_equal(c.stored(1, "k"), before)


def test_special_values(lpq):
    """NaN and infinities turn into what the formula gives, features that are not turned into themselves."""
    c = Case(lpq, 1, 40, 16, [20], "f32", seed=6)
    for interleaved in (False, True):
        r = Rotated(c, 1, [0], [20], 24, interleaved)
        r.q[3, 0, [0, 1, 13, 30]] = torch.tensor([float("nan"), float("inf"), -float("inf"), float("inf")])
        r.q[4] = float("inf")
        r.q[5] = -0.0
        r.k[6, 0, 2] = float("nan")
        out = r.call(c.cache, c.table)
        want = r.want_queries()
        assert equal(out.cpu(), want)
        assert torch.equal(out[:, :, 24:].cpu(), r.q[:, :, 24:])
        assert np.array_equal(c.stored(0, "k"), plain.codes(r.turned(r.k), c.kc, False))


def test_strides(lpq):
    """Keys, values and queries inside one tensor, heads outermost, angles in wider tables, queries turned where they lie."""
    c = Case(lpq, 3, 40, 16, [20, 33], "f16", seed=7)
    r = Rotated(c, 2, [0, 0], [20, 33], 28, False)
    want = r.want_queries()
    r.call(c.cache, c.table)
    other = Case(lpq, 3, 40, 16, [20, 33], "f16", seed=7)
    packed = torch.full((53, 12, 43), 9.0, dtype=torch.float16, device="cuda")
    packed[:, :6, 1:41], packed[:, 6:9, 1:41], packed[:, 9:, 1:41] = r.q.cuda(), r.k.cuda(), r.v.cuda()
    q, k, v = packed[:, :6, 1:41], packed[:, 6:9, 1:41], packed[:, 9:, 1:41]
    wide = torch.full((len(r.cos), 3, 20), 5.0, device="cuda")
    wide[:, 0, :14], wide[:, 1, 1:15] = torch.from_numpy(r.cos).cuda(), torch.from_numpy(r.sin).cuda()
    other.cache.write_rotated(k, v, ints([0, 0]), other.table, wide[:, 0, :14], wide[:, 1, 1:15], starts=ints([0, 20, 53]), q=q, out=q)
    assert torch.equal(other.cache.k, c.cache.k) and torch.equal(other.cache.v, c.cache.v) and torch.equal(other.cache.bounds, c.cache.bounds)
    assert equal(packed[:, :6, 1:41].cpu(), want)
    assert torch.equal(packed[:, 6:9, 1:41].cpu(), r.k) and (packed[:, :, 0] == 9).all() and (packed[:, :, 41:] == 9).all()
    out = torch.full((6, 53, 44), 3.0, dtype=torch.float16, device="cuda")
    r.call(other.cache, other.table, queries=r.q.cuda().permute(1, 0, 2).contiguous().permute(1, 0, 2), out=out[..., 2:42].permute(1, 0, 2))
    assert equal(out[..., 2:42].permute(1, 0, 2).cpu(), want) and (out[..., :2] == 3).all() and (out[..., 42:] == 3).all()


def test_a_generation_step_with_streams_and_graphs(lpq):
    """Rotated rows, attention with a window and over a tree: on another stream and replayed."""
    c = Case(lpq, 2, 128, 16, [200, 90], "bf16", seed=8)
    r = Rotated(c, 4, [180, 70], [6, 6], 128, False, count=400)
    k, v, q = r.k.cuda(), r.v.cuda(), r.q.cuda()
    first, starts, lengths = ints([180, 70]), ints([0, 6, 12]), ints([186, 76])
    cos, sin = torch.from_numpy(r.cos).cuda(), torch.from_numpy(r.sin).cuda()
    tree = torch.ones(6, 6, dtype=torch.bool, device="cuda").tril()
    depth = ints([180, 181, 181, 182, 182, 182, 70, 71, 72, 72, 73, 73])

    def step():
        turned = c.cache.write_rotated(k, v, first, c.table, cos, sin, starts=starts, positions=depth, q=q)
        seen = turned.view(2, 6, 8, 128)
        return turned, c.cache.attend(seen, lengths, c.table, tree=tree), c.cache.attend(seen, lengths, c.table, window=64, sinks=4)

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
    for turn_ in range(3):
        q.mul_(0.9)
        k.mul_(1.1)
        first.add_(turn_)
        depth.add_(turn_)
        lengths.add_(turn_)
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), turn_


def test_refusals(lpq):
    c = Case(lpq, 2, 64, 16, [40, 20], "bf16")
    k, q = torch.cat(c.k).cuda(), c.queries(2, 1)[:, 0].repeat(30, 1, 1).cuda()
    cos = torch.ones(50, 32, device="cuda")
    first, starts = ints([0, 0]), ints([0, 40, 60])

    def call(k=k, v=k, cos=cos, sin=cos, starts=starts, **kw):
        return c.cache.write_rotated(k, v, first, c.table, cos, sin, starts=starts, **kw)

    def code(**kw):
        with pytest.raises(lpq.LpqError) as e:
            call(**kw)
        return e.value.code
    before = c.cache.k.clone()
    assert code(starts=None) == lpq.EINVAL                                           # 60 rows, 2 sequences
    wide = torch.ones(50, 33, device="cuda")
    assert code(cos=wide, sin=wide) == lpq.EINVAL                                    # 66 of 64 features
    assert code(cos=cos[:0], sin=cos[:0]) == lpq.EINVAL
    assert code(cos=cos[:, :0], sin=cos[:, :0]) == lpq.EINVAL
    assert code(q=q[:, :3]) == lpq.EINVAL                                            # 3 query heads on 2
    assert code(q=q, out=torch.empty_like(q[:1]).expand(60, -1, -1)) == lpq.EINVAL
    for bad in (dict(cos=cos.cpu()), dict(cos=cos.double()), dict(sin=cos[:, :31]), dict(sin=cos[:49]), dict(q=q.float()), dict(q=q[:59]),
                dict(q=q, out=q[:, :2]), dict(q=q[..., :63]), dict(positions=ints([0] * 59)), dict(positions=ints([0] * 60).long()), dict(v=k[:59]),
                dict(q=q.cpu()), dict(cos=cos.t().contiguous().t())):
        with pytest.raises(AssertionError):
            call(**bad)
    with pytest.raises(AssertionError):
        call(q=q.requires_grad_())
    assert torch.equal(before, c.cache.k)
    # nothing to do
    none = torch.zeros(0, 3, dtype=torch.int32, device="cuda")
    assert c.cache.write_rotated(k[:0], k[:0], ints([]), none, cos, cos, q=q[:0].detach()).shape == (0, 4, 64)
