"""Attention over a key-value cache where new tokens see less than all that is ahead of them: a window with the first tokens (sinks), or
a tree of drafted tokens.  Against the plain definition in 64 bits, within the bound that kv_plain.py derives for attention."""
import numpy as np
import pytest
import torch

import kv_plain as plain
from test_gpu_kv_cache import TYPES, Case, ints, lpq  # noqa: F401  (lpq is a fixture)

pytestmark = pytest.mark.gpu


def attend(q, kx, vx, group, scale, sees):
    """q [new, q_heads, dim], kx / vx float64 [n, heads, dim], sees bool [new, n] -> o, lse in float64."""
    new, q_heads, dim = q.shape
    o, lse = np.zeros((new, q_heads, dim)), np.full((new, q_heads), -np.inf)
    for j in range(q_heads):
        t = scale * (q[:, j].astype(np.float64) @ kx[:, j // group].T)
        for i in range(new):
            at = np.flatnonzero(sees[i])
            if len(at):
                most = t[i, at].max()
                p = np.exp(t[i, at] - most)
                o[i, j] = p @ vx[at, j // group] / p.sum()
                lse[i, j] = most + np.log(p.sum())
    return o, lse


def window_mask(n, new, window, sinks):
    p = np.arange(n)[None]
    me = n - new + np.arange(new)[:, None]
    return (p <= me) & ((p > me - window) | (p < sinks))


def tree_mask(n, new, tree):
    """tree bool [new, new]; new tokens at positions below 0 see nothing."""
    sees = np.zeros((new, n), bool)
    at = n - new
    for i in range(new):
        if at + i < 0:
            continue
        sees[i, :max(0, at)] = True
        for j in range(new):
            if at + j >= 0:
                sees[i, at + j] = tree[i, j]
    return sees


def random_tree(rng, new, empty=0.0):
    tree = np.zeros((new, new), bool)
    for i in range(new):
        if i:
            tree[i] = tree[rng.integers(max(0, i - 4), i)]
        tree[i, i] = True
    tree[rng.random(new) < empty] = False
    return tree


def check(c, q, out, lse, group, sees, scale=None):
    kind = {v: k for k, v in TYPES.items()}[q.dtype]
    scale = c.dim ** -0.5 if scale is None else scale
    q, out, lse = q.float().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, n in enumerate(c.lengths):
        o, want = attend(q[b], c.kx[b], c.vx[b], group, scale, sees[b])
        err, lerr = plain.attend_bound(q[b], c.kcodes[b], c.vx[b], c.kc, group, scale, kind)
        empty = np.isinf(want)
        assert (out[b][empty] == 0).all() and np.isneginf(lse[b][empty]).all()
        diff = np.abs(out[b] - o)
        assert (diff <= err).all(), (b, n, float((diff - err).max()))
        assert np.isfinite(lse[b][~empty]).all() and (np.abs(lse[b][~empty] - want[~empty]) <= lerr[~empty]).all()


def roomy(c, columns):
    """The case's table with room for long sequences: how a call is shared out goes by that."""
    if not columns:
        return c.table
    table = torch.full((len(c.lengths), columns), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    return table


SHAPES = [  # heads, dim, page, lengths, group, new, type, packed
    (2, 64, 16, [1, 0, 63, 64, 65], 1, 1, "bf16", False),
    (1, 128, 64, [700, 255, 256, 257, 3], 4, 1, "bf16", False),
    (2, 100, 32, [333, 31], 3, 1, "f16", False),
    (1, 192, 16, [130, 33, 1], 12, 4, "f32", True),
    (3, 80, 64, [200, 7], 5, 3, "bf16", True),
    (1, 256, 128, [500, 128], 16, 2, "f16", False),
    (2, 33, 16, [45, 2, 0], 1, 4, "f32", False),          # more new tokens than tokens
    (1, 64, 256, [2000], 40, 1, "f32", True),
    (1, 192, 32, [400, 90], 8, 9, "bf16", False),         # 72 query rows
    (1, 128, 64, [2500, 300], 8, 1, "f16", True),
    (4, 128, 32, [3000], 1, 1, "f32", False),
    (2, 128, 16, [700, 40, 333], 4, 30, "bf16", False),   # row tiles that each have a range of their own
    (1, 64, 32, [900], 5, 101, "f16", True),
    (1, 256, 16, [400], 2, 37, "f32", False),
    (1, 1, 16, [50], 2, 1, "f32", False),
]
WINDOWS = [(1, 0), (7, 3), (64, 0), (100, 1), (250, 17), (700, 64)]


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("heads,dim,page,lengths,group,new,kind,packed", SHAPES)
def test_window(lpq, heads, dim, page, lengths, group, new, kind, packed, window, sinks):
    c = Case(lpq, heads, dim, page, lengths, kind, packed, seed=window)
    q = c.queries(group, new)
    sees = [window_mask(n, new, window, sinks) for n in lengths]
    for columns in (None, 16 * (1 << 14) // page):
        out, lse = c.cache.attend(q.cuda(), ints(lengths), roomy(c, columns), window=window, sinks=sinks, return_lse=True)
        check(c, q, out, lse, group, sees)
        again = c.cache.attend(q.cuda(), ints(lengths), roomy(c, columns), window=window, sinks=sinks)
        assert torch.equal(out, again)


@pytest.mark.parametrize("heads,dim,kind,packed,group,new,window,sinks", [
    (8, 128, "bf16", False, 4, 1, 1500, 4),
    (2, 128, "bf16", False, 8, 5, 2000, 130),
    (1, 64, "f16", True, 16, 3, 3000, 0),
    (3, 192, "f32", True, 2, 2, 1300, 33),
    (1, 256, "bf16", False, 12, 4, 1100, 16),
    (1, 128, "f32", False, 3, 200, 1200, 5),
])
def test_long_windows_in_parts(lpq, heads, dim, kind, packed, group, new, window, sinks):
    """Windows beyond 1024 tokens are split over workgroups and joined, each row tile by itself."""
    lengths = [5000, new, 1203, 0, 2600]
    c = Case(lpq, heads, dim, 32, lengths, kind, packed, seed=3)
    q = c.queries(group, new)
    out, lse = c.cache.attend(q.cuda(), ints(lengths), roomy(c, 4000), window=window, sinks=sinks, return_lse=True)
    check(c, q, out, lse, group, [window_mask(n, new, window, sinks) for n in lengths])


@pytest.mark.parametrize("window", [33, 999, 2000, 4096, 2 ** 31 + 5])
def test_a_window_that_holds_everything_is_none(lpq, window):
    c = Case(lpq, 2, 72, 16, [999, 32], "f16", seed=5)
    q = c.queries(3, 2).cuda()
    want, want_lse = c.cache.attend(q, ints(c.lengths), c.table, return_lse=True)
    got, lse = c.cache.attend(q, ints(c.lengths), c.table, window=window, sinks=7, return_lse=True)
    if window >= 1008:                                    # more than the table has room for
        assert torch.equal(want, got) and torch.equal(want_lse, lse)
    check(c, q.cpu(), got, lse, 3, [window_mask(n, 2, window, 7) for n in c.lengths])


@pytest.mark.parametrize("columns", [None, 4000])
@pytest.mark.parametrize("kind,packed,group,new", [("bf16", False, 4, 1), ("f32", True, 3, 40), ("f16", False, 8, 3)])
def test_what_is_not_seen_does_not_count(lpq, kind, packed, group, new, columns):
    """Other codes at the positions that no row sees, pages missing there: equal bits."""
    c = Case(lpq, 2, 128, 16, [600, 1400], kind, packed, seed=6)
    q, window, sinks = c.queries(group, new).cuda(), 130, 21
    lengths, table = ints(c.lengths), roomy(c, columns)
    want = c.cache.attend(q, lengths, table, window=window, sinks=sinks)
    hidden = table.clone()
    for b, n in enumerate(c.lengths):
        seen = window_mask(n, new, window, sinks).any(0)
        for p in range(-(-n // 16)):
            rows = np.flatnonzero(~seen[p * 16:(p + 1) * 16])
            for pool in (c.cache.k, c.cache.v):
                pool[int(c.table_np[b, p]), :, rows.tolist()] = 119
            if len(rows) == len(seen[p * 16:(p + 1) * 16]):
                hidden[b, p] = (-1, c.cache.pages + 5)[p & 1]
    assert (hidden != table).sum() > 60
    assert torch.equal(want, c.cache.attend(q, lengths, table, window=window, sinks=sinks))
    assert torch.equal(want, c.cache.attend(q, lengths, hidden, window=window, sinks=sinks))


@pytest.mark.parametrize("heads,dim,page,lengths,group,new,kind,packed", SHAPES)
def test_tree(lpq, heads, dim, page, lengths, group, new, kind, packed):
    c = Case(lpq, heads, dim, page, lengths, kind, packed, seed=7)
    q = c.queries(group, new)
    trees = np.stack([random_tree(c.rng, new, 0.2) for _ in lengths])
    sees = [tree_mask(n, new, t) for n, t in zip(lengths, trees)]
    for columns in (None, 16 * (1 << 14) // page):
        out, lse = c.cache.attend(q.cuda(), ints(lengths), roomy(c, columns), tree=torch.from_numpy(trees).cuda(), return_lse=True)
        check(c, q, out, lse, group, sees)


@pytest.mark.parametrize("lengths", [[64], [63, 70], [300, 1, 0, 64 + 33], [1500, 64, 20]])
@pytest.mark.parametrize("kind,packed,dim", [("bf16", False, 128), ("f32", True, 64), ("f16", False, 256)])
def test_trees_without_tokens_ahead_and_shorter_than_their_mask(lpq, lengths, kind, packed, dim):
    """64 drafted tokens, some sequences with fewer: the first rows have no position then.  Rows that name nothing see what is ahead."""
    new = 64
    c = Case(lpq, 1, dim, 16, lengths, kind, packed, seed=8)
    q = c.queries(2, new)
    trees = np.stack([random_tree(c.rng, new, 0.3) for _ in lengths])
    out, lse = c.cache.attend(q.cuda(), ints(lengths), c.table, tree=torch.from_numpy(trees).cuda(), return_lse=True)
    check(c, q, out, lse, 2, [tree_mask(n, new, t) for n, t in zip(lengths, trees)])


@pytest.mark.parametrize("new,group,dim", [(4096, 1, 64), (300, 3, 128), (777, 1, 256)])
def test_large_trees_and_masks_of_any_form(lpq, new, group, dim):
    """Not only ancestors: any mask, up to the largest there is room for."""
    lengths = [new + 37]
    c = Case(lpq, 1, dim, 64, lengths, "bf16", seed=9)
    q = c.queries(group, new)
    mask = c.rng.random((1, new, new)) < 0.4
    out, lse = c.cache.attend(q.cuda(), ints(lengths), c.table, tree=torch.from_numpy(mask).cuda(), return_lse=True)
    check(c, q, out, lse, group, [tree_mask(lengths[0], new, mask[0])])


def test_a_chain_is_causal_and_masks_may_be_shared_or_strided(lpq):
    c = Case(lpq, 2, 96, 32, [400, 90, 1300], "f16", seed=10)
    new = 21
    q = c.queries(4, new).cuda()
    lengths = ints(c.lengths)
    chain = torch.ones(new, new, dtype=torch.bool, device="cuda").tril()
    out, lse = c.cache.attend(q, lengths, c.table, tree=chain, return_lse=True)
    check(c, q.cpu(), out, lse, 4, [window_mask(n, new, n + 1, 0) for n in c.lengths])
    tree = torch.from_numpy(random_tree(c.rng, new)).cuda()
    want = c.cache.attend(q, lengths, c.table, tree=tree)
    assert torch.equal(want, c.cache.attend(q, lengths, c.table, tree=tree.expand(3, -1, -1)))
    wide = torch.ones(new, 5, new + 9, dtype=torch.bool, device="cuda")
    wide[:, 1::2, 4:4 + new] = tree[:, None]
    assert torch.equal(want[:2], c.cache.attend(q[:2], lengths[:2], c.table[:2], tree=wide[:, 1::2, 4:4 + new].permute(1, 0, 2)))
    # what drafted tokens that no row names hold does not count
    alone = torch.zeros(new, new, dtype=torch.bool, device="cuda")
    alone[:, 0] = True
    want = c.cache.attend(q, lengths, c.table, tree=alone)
    for b, n in enumerate(c.lengths):
        for p in range(n - new + 1, n):
            for pool in (c.cache.k, c.cache.v):
                pool[int(c.table_np[b, p // 32]), :, p % 32] = -77
    assert torch.equal(want, c.cache.attend(q, lengths, c.table, tree=alone))


def test_windows_and_trees_over_listed_pages(lpq):
    c = Case(lpq, 2, 64, 16, [300, 77], "f32", seed=11)
    new = 5
    q = c.queries(3, new)
    pages = torch.tensor([[[0, 3, 18, -1, 17], [17, 2, 18, 1, 0]], [[4, 0, 3, -1, -1], [1, 4, 99, 2, -1]]], dtype=torch.int32)
    tree = random_tree(c.rng, new)
    for name, masks in (("window", [window_mask(n, new, 20, 9) for n in c.lengths]), ("tree", [tree_mask(n, new, tree) for n in c.lengths])):
        kw = dict(window=20, sinks=9) if name == "window" else dict(tree=torch.from_numpy(tree).cuda())
        out, lse = c.cache.attend(q.cuda(), ints(c.lengths), c.table, pages=pages.cuda(), return_lse=True, **kw)
        for h in range(2):      # each head has pages of its own
            sees = [m & np.isin(np.arange(n) // 16, pages[b, h].numpy())[None] for b, (n, m) in enumerate(zip(c.lengths, masks))]
            for b in range(2):
                o, want = attend(q[b, :, 3 * h:3 * h + 3].numpy(), c.kx[b][:, h:h + 1], c.vx[b][:, h:h + 1], 3, 64 ** -0.5, sees[b])
                err, lerr = plain.attend_bound(q[b].numpy(), c.kcodes[b], c.vx[b], c.kc, 3, 64 ** -0.5, "f32")
                part = slice(3 * h, 3 * h + 3)
                assert (np.abs(out[b, :, part].double().cpu().numpy() - o) <= err[:, part]).all()
                empty = np.isinf(want)
                got = lse[b, :, part].double().cpu().numpy()
                assert np.isneginf(got[empty]).all() and (np.abs(got[~empty] - want[~empty]) <= lerr[:, part][~empty]).all()


def test_rows_that_are_not_finite_and_rows_that_see_nothing(lpq):
    """A row with a NaN gives NaN where it sees a token, zeros where it sees none; the others do not notice."""
    c = Case(lpq, 1, 128, 16, [3, 200, 0], "bf16", seed=12)
    new = 6
    q = c.queries(2, new)
    tree = np.tril(np.ones((new, new), bool))
    tree[4] = False
    clean = {}
    for bad in (False, True):
        if bad:
            q[:, 1, 0, 3] = float("nan")
            q[:, 4, 1, 5] = float("inf")
        for name, kw in (("window", dict(window=4, sinks=1)), ("tree", dict(tree=torch.from_numpy(tree).cuda()))):
            out, lse = c.cache.attend(q.cuda(), ints(c.lengths), c.table, return_lse=True, **kw)
            if not bad:
                clean[name] = out, lse
                continue
            want, want_lse = (t.clone() for t in clean[name])
            for b, i, h in ((1, 1, 0), (1, 4, 1), (0, 4, 1)):
                if name == "tree" and (b, i) == (0, 4):
                    continue                              # no token ahead and none that it names
                want[b, i, h], want_lse[b, i, h] = float("nan"), float("nan")
            assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(torch.isnan(lse), torch.isnan(want_lse))
            assert torch.equal(out.nan_to_num(), want.nan_to_num())
            assert not out[2].any() and torch.isneginf(lse[2]).all() and not out[0, :3].any()
    # lengths below 0 and beyond the table
    for kw in (dict(window=9, sinks=2), dict(tree=torch.from_numpy(tree).cuda())):
        out, lse = c.cache.attend(clean["tree"][0], ints([-7, 0, -(2 ** 31)]), c.table, return_lse=True, **kw)
        assert not out.any() and torch.isneginf(lse).all()
        room = 13 * 16
        a = c.cache.attend(clean["tree"][0], ints([room] * 3), c.table, **kw)
        b = c.cache.attend(clean["tree"][0], ints([2 ** 31 - 1, room + 1, 10 ** 9]), c.table, **kw)
        assert torch.equal(a, b)


def test_offsets_beyond_32_bits(lpq):
    """A window at the far end of a pool of more than 4 GiB."""
    heads, dim, page = 8, 128, 256
    c = Case(lpq, heads, dim, page, [700], seed=13)
    pages = (1 << 32) // (heads * dim * page) + 8
    quant = [lpq.Quantizer(heads * dim, 8).set_params(k.k.reshape(-1), k.sb.reshape(-1), k.se.reshape(-1)) for k in (c.kc, c.vc)]
    big = lpq.KVCache(*quant, heads=heads, page=page, pages=pages)
    table = torch.tensor([[pages - 1, pages // 2 + 3, pages - 2]], dtype=torch.int32, device="cuda")
    big.write(c.k[0].cuda(), c.v[0].cuda(), ints([0]), table, ints([0, 700]))
    q = c.queries(4, 3)
    out, lse = big.attend(q.cuda(), ints([700]), table, window=300, sinks=5, return_lse=True)
    check(c, q, out, lse, 4, [window_mask(700, 3, 300, 5)])


def test_strides_scale_and_a_given_workspace(lpq):
    c = Case(lpq, 2, 72, 16, [2500, 90], "f32", seed=14)
    q = c.queries(3, 2)
    wide = torch.zeros(2, 2, 6, 3, 75)
    wide[:, :, :, 1, 2:74] = q
    base = torch.full((2, 6, 2, 80), 5.0, device="cuda")
    need = lpq.lib().lpq_kv_attend_masked_workspace_bytes(c.cache._h, 2, 2, 6, c.table.shape[1], 0, 1500, 4, 0)
    assert need > 0
    room = torch.full((need + 512,), 85, dtype=torch.uint8, device="cuda")
    out, lse = c.cache.attend(wide.cuda()[:, :, :, 1, 2:74], ints(c.lengths), c.table, scale=-0.31, out=base.permute(0, 2, 1, 3)[..., 4:76],
                              return_lse=True, window=1500, sinks=4, workspace=room[:need])
    check(c, q, out, lse, 3, [window_mask(n, 2, 1500, 4) for n in c.lengths], scale=-0.31)
    assert (base[..., :4] == 5).all() and (base[..., 76:] == 5).all() and (room[need:] == 85).all()


def test_streams_and_graphs_with_workspaces_of_their_own_and_shared(lpq):
    c = Case(lpq, 2, 128, 16, [1700, 400], seed=15)
    new = 7
    q, lengths = c.queries(4, new).cuda(), ints(c.lengths)
    tree = torch.from_numpy(np.stack([random_tree(c.rng, new) for _ in range(2)])).cuda()
    need = max(lpq.lib().lpq_kv_attend_masked_workspace_bytes(c.cache._h, 2, new, 8, c.table.shape[1], 0, w, 3, t) for w, t in ((1200, 0), (0, 1)))
    room = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step(workspace):
        return (c.cache.attend(q, lengths, c.table, window=1200, sinks=3, workspace=workspace), c.cache.attend(q, lengths, c.table, tree=tree, workspace=workspace),
                c.cache.attend(q, lengths, c.table, window=50))

    want = step(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(None)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graphs = []
    for workspace in (None, room, room):                  # two of them share a workspace, and run one behind the other
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step(workspace)
        graphs.append((graph, got))
    for turn in range(3):
        q.copy_(c.queries(4, new))
        lengths.sub_(turn)
        tree.copy_(torch.from_numpy(np.stack([random_tree(c.rng, new) for _ in range(2)])))
        want = step(None)
        torch.cuda.synchronize()
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, got in graphs:
            assert all(torch.equal(a, b) for a, b in zip(want, got)), turn


def test_refusals(lpq):
    c = Case(lpq, 2, 64, 16, [40, 20])
    new = 3
    q, lengths, tree = c.queries(2, new).cuda(), ints([40, 20]), torch.ones(2, new, new, dtype=torch.bool, device="cuda")

    def code(**kw):
        with pytest.raises(lpq.LpqError) as e:
            c.cache.attend(q, lengths, c.table, **kw)
        return e.value.code
    assert code(sinks=4) == lpq.EINVAL
    assert code(window=8, tree=tree) == lpq.EINVAL
    assert code(window=8, scale=float("inf")) == lpq.EINVAL
    assert code(tree=tree, out=torch.empty_like(q[:1]).expand(2, -1, -1, -1)) == lpq.EINVAL
    many = torch.zeros(1, 5000, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(lpq.LpqError) as e:
        c.cache.attend(many, lengths[:1], c.table[:1], tree=torch.ones(1, 1, dtype=torch.bool, device="cuda").expand(5000, 5000).contiguous())
    assert e.value.code == lpq.ERANGE
    long = Case(lpq, 1, 64, 16, [3000])
    with pytest.raises(lpq.LpqError) as e:
        long.cache.attend(long.queries(2).cuda(), ints([3000]), long.table, window=2000, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == lpq.ERANGE
    for kw in (dict(window=0), dict(window=-3), dict(window=5, sinks=-1), dict(window=5, sinks=2 ** 31), dict(tree=tree.cpu()), dict(tree=tree.byte()),
               dict(tree=tree[:1]), dict(tree=tree[:, :2]), dict(tree=tree.transpose(1, 2)[:, :, :2]), dict(tree=tree.float())):
        with pytest.raises(AssertionError):
            c.cache.attend(q, lengths, c.table, **kw)
    grad = q.float().requires_grad_()
    with pytest.raises(AssertionError):
        c.cache.attend(grad, lengths, c.table, window=4)
