"""How attention over a key-value cache is shared out to workgroups, on a real MI355X: equal runs that cross heads and sequences, parts
of a sequence in many workgroups, many query rows, joins of many rows; and rows read back by workgroups that take several heads."""
import numpy as np
import pytest
import torch

import kv_plain as plain
from test_gpu_kv_cache import TYPES, Case, ints, lpq  # noqa: F401  (lpq is a fixture)

pytestmark = pytest.mark.gpu

RUN = 200      # tiles from which on a workgroup's run goes over to the next pair wherever it ends


def blocks_per_cu(dpad, packed, rows, kind):
    if dpad > 128:
        return 2 if rows == 16 and not (dpad == 256 and kind == "f32") else 1
    if rows == 32:
        return 2
    return 3 if kind == "f32" or (dpad > 64 and (packed or kind == "f16")) else 4


def two_row_tiles(dpad, packed, kind):
    if packed:
        return dpad == 64 or (kind == "bf16" and dpad != 192)
    return dpad < 192 or kind != "f32"


def planned(dim, packed, kind, pairs, rows, tokens):
    """rows of a row tile, row tiles, shares, whether tiles are dealt out, bytes of workspace."""
    dpad = -(-dim // 64) * 64
    tile = 64 if dpad // (2 if packed else 1) <= 64 else 32
    high = 32 if rows > 16 and pairs * tokens > 1 << 19 and two_row_tiles(dpad, packed, kind) else 16
    row_tiles = -(-rows // high)
    grid, tiles = pairs * row_tiles, -(-tokens // tile)
    chip = 256 * blocks_per_cu(dpad, packed, high, kind)
    if not (tokens > 1024 or (grid < 256 and tokens * dpad > 128 * 1024)) or row_tiles >= chip:
        return high, row_tiles, pairs, False, 0
    shares = min(-(-tiles // 4) * pairs, -(-chip // row_tiles))
    if row_tiles > 1:
        shares = -(-shares // 8) * 8
    return high, row_tiles, shares, True, 4 * (2 * shares * row_tiles * high * (dpad + 2) + 2 * pairs)


def mode(lpq, c, columns, group, new):
    """("equal" or "apart", rows of a row tile, row tiles, most parts of a pair) of a call with tables of that many columns."""
    pairs, tokens = c.heads * len(c.lengths), columns * c.page
    plans = {k: planned(c.dim, c.packed, k, pairs, new * group, tokens) for k in TYPES}
    need = lpq.lib().lpq_kv_attend_workspace_bytes(c.cache._h, len(c.lengths), new, c.heads * group, columns, 0)
    assert need == max(p[4] for p in plans.values()), "the plan is another one: bring the cases here in line with it"
    high, row_tiles, shares, dealt, _ = plans[c.kind]
    assert dealt
    tile = 64 if -(-c.dim // 64) * (32 if c.packed else 64) <= 64 else 32
    tiles = [max(1, -(-n // tile)) for n in c.lengths]
    run = max(4, -(-sum(tiles) * c.heads // shares))
    apart = run < RUN and pairs < shares
    return "apart" if apart else "equal", high, row_tiles, -(-max(tiles) // run)


def call(c, group, new, columns):
    q = c.queries(group, new)
    table = torch.full((len(c.lengths), columns), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    return q, *c.cache.attend(q.cuda(), ints(c.lengths), table, return_lse=True)


def ragged(count, most, seed):
    rng = np.random.default_rng(seed)
    n = [int(x) for x in np.exp(rng.uniform(0, np.log(most + 1), count))]
    n[1::7] = [0] * len(n[1::7])
    return n


@pytest.mark.parametrize("heads,dim,kind,packed,group,new,high", [
    (4, 64, "bf16", False, 1, 1, 16),
    (4, 64, "f16", True, 2, 2, 16),
    (5, 100, "f32", False, 3, 1, 16),
    (3, 128, "bf16", False, 20, 1, 32),
    (3, 128, "bf16", True, 5, 4, 32),
    (3, 64, "f32", True, 17, 1, 32),
    (2, 192, "f16", False, 9, 2, 32),
    (2, 256, "bf16", False, 1, 1, 16),
])
def test_equal_runs_cross_heads_and_sequences(lpq, heads, dim, kind, packed, group, new, high):
    """More (sequence, head) than shares: a workgroup ends one pair that began before its run, has some whole ones and begins another."""
    c = Case(lpq, heads, dim, 16, ragged(-(-1100 // heads), 700, 31), kind, packed, seed=31)
    columns = 2048 // 16
    assert mode(lpq, c, columns, group, new)[:2] == ("equal", high)
    q, out, lse = call(c, group, new, columns)
    c.check_attention(q, out, lse, group)
    assert torch.equal(out, call_again(c, q, columns))


def call_again(c, q, columns):
    table = torch.full((len(c.lengths), columns), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    return c.cache.attend(q.cuda(), ints(c.lengths), table)


@pytest.mark.parametrize("dim,kind,packed", [(64, "bf16", False), (64, "f32", True), (128, "f16", False), (192, "bf16", True),
                                             (192, "f32", False), (256, "f16", True), (256, "f32", False)])
def test_parts_of_many_rows_are_joined(lpq, dim, kind, packed):
    """At least 1024 rows of several parts each."""
    c = Case(lpq, 4, dim, 64, [int(x) for x in np.linspace(1100, 2500, 17)], kind, packed, seed=32)
    dealt, high, row_tiles, parts = mode(lpq, c, c.table.shape[1], 16, 1)
    assert (dealt, high, row_tiles) == ("apart", 16, 1) and parts >= 4 and 17 * 4 * 16 >= 1024
    q, out, lse = call(c, 16, 1, c.table.shape[1])
    c.check_attention(q, out, lse, 16)


@pytest.mark.parametrize("dim,kind,packed,group,new", [(64, "bf16", False, 16, 40), (128, "f32", True, 5, 130), (192, "f16", False, 8, 75)])
def test_many_query_rows_on_few_pairs(lpq, dim, kind, packed, group, new):
    """A part of a prompt: hundreds of new tokens, more pairs than shares of a row tile, some sequences shorter than what is new."""
    c = Case(lpq, 1, dim, 32, ragged(45, 400, 33), kind, packed, seed=33)
    dealt, high, row_tiles, _ = mode(lpq, c, 40, group, new)
    assert (dealt, high) == ("equal", 16) and row_tiles > 32
    q, out, lse = call(c, group, new, 40)
    c.check_attention(q, out, lse, group)


def test_long_runs_of_one_pair(lpq):
    """2048 rows on one head of 52 000 tokens: runs of more than 200 tiles, the pair in eight of them.  Some of the rows are checked."""
    c = Case(lpq, 1, 128, 64, [52_000], "bf16", seed=34)
    dealt, high, row_tiles, parts = mode(lpq, c, c.table.shape[1], 2048, 1)
    assert (dealt, high, row_tiles, parts) == ("equal", 16, 128, 8)
    q, out, lse = call(c, 2048, 1, c.table.shape[1])
    some = np.r_[0:3, 700:703, 1337, 2045:2048]
    c.check_attention(q[:, :, some], out[:, :, some], lse[:, :, some], len(some))


@pytest.mark.parametrize("heads,dim,kind,packed", [(4, 64, "bf16", False), (6, 40, "f16", True), (3, 128, "f32", False)])
def test_rows_of_several_heads_are_read_back_together(lpq, heads, dim, kind, packed):
    """Rows enough that a workgroup takes neighbouring heads and several pages of them (workgroups of 256 threads, 8 features each; 4096 of them)."""
    lengths = [20_001, 0, 17, 20_000]
    c = Case(lpq, heads, dim, 16, lengths, kind, packed, seed=35)
    n, slots = sum(lengths), 256 // (-(-dim // 64) * 8)
    units = -(-n // 16) + len(lengths)
    together = max(h for h in range(1, heads + 1) if heads % h == 0 and h <= slots and slots // h * h * 8 >= slots * 7
                   and (h == 1 or 2 * units * (heads // h) >= 4096))
    assert together > 1
    k, v = c.cache.read(ints([0] * 4), c.table, ints(c.starts.tolist()), n, TYPES[kind])
    for got, codes, consts in ((k, c.kcodes, c.kc), (v, c.vcodes, c.vc)):
        want = torch.from_numpy(np.concatenate([plain.values(q, consts) for q in codes])).to(TYPES[kind])
        assert torch.equal(got.cpu(), want)
    bounds = c.cache.bounds.cpu().numpy()
    for b, m in enumerate(lengths):
        if m:
            assert np.array_equal(bounds[c.table_np[b, :-(-m // 16)]], plain.bounds(c.kcodes[b], 16))


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
def test_small_weights_in_tiles_with_a_large_one(lpq, kind):
    """1000 tokens in one workgroup, one of them with nearly all the weight, the others at 2^-24.5 of it with values at the other end of
    the range.  A wave has 255 of them in tiles of its own with the large one: lost, they would move lse and (float32) the result by several
    times the bound.  The bound: sums of at most 16 matrix instructions and 4 waves, each rounded to 2^-24; a logarithm of 13 to half a unit and one of the
    instruction; the row's offset, 8 roundings of |q| |k|; the score of the small tokens, rounded to 2^-16 of 17, on their share."""
    n, large, heads = 1000, 5, 1
    c = Case(lpq, heads, 64, 64, [n], kind, seed=36)
    depth = 24.5 * np.log(2.0)
    k = np.broadcast_to(c.mean - 2.0 * c.std, (n, 64)).copy()
    k[large] = c.mean + 1e-3 * c.std
    v = np.broadcast_to(0.1 * c.mean + 3.0 * c.std, (n, 64)).copy()
    v[large] = 0.1 * c.mean - 3.0 * c.std
    k, v = (torch.from_numpy(x.astype(np.float32)).to(TYPES[kind]).view(n, 1, 64) for x in (k, v))
    c.cache.write(k.cuda(), v.cuda(), ints([0]), c.table, ints([0, n]))
    kcodes, vcodes = plain.codes(k.float().numpy(), c.kc, False), plain.codes(v.float().numpy(), c.vc, False)
    kx, vx = plain.values(kcodes, c.kc).astype(np.float64), plain.values(vcodes, c.vc).astype(np.float64)
    q = torch.from_numpy((1.0 / c.std).astype(np.float32)).view(1, 1, 1, 64).to(TYPES[kind])
    qd = q.double().numpy()[0]
    scale = float(np.float32(depth / (qd[0] @ (kx[large] - kx[0]).T).item()))
    o, lse = plain.attend(qd, kx, vx, 1, scale)
    seen = np.ones(n, bool)
    seen[(np.arange(n) // 64 % 4 == 0) & (np.arange(n) != large)] = False        # the small ones of the wave with the large one
    assert (~seen).sum() == 255
    lost_o, lost_lse = plain.attend(qd, kx, vx, 1, scale, dead=~seen)
    unit, share = 2.0 ** -24, n * 2.0 ** -24.5
    offset = abs(scale) * (np.abs(qd[0]) @ (np.abs(c.kc.k) + c.kc.s).T).item()
    lse_bound = 20 * unit + 1.5 * 2.0 ** -20 * np.log(2.0) + 8 * unit * offset + 17 * 2.0 ** -16 * share
    size = np.abs(vx).max(0)[0]
    bound = plain.UNIT[kind] * size + 24 * unit * 2 * size + (17 * 2.0 ** -16 + 2.0 ** -11) * share * 2 * size
    got, got_lse = c.cache.attend(q.cuda(), ints([n]), c.table, scale=scale, return_lse=True)
    assert abs(lost_lse - lse).max() > 2 * lse_bound
    assert np.abs(got_lse[0].double().cpu().numpy() - lse).max() <= lse_bound
    if kind == "f32":
        assert (np.abs(lost_o - o)[0, 0] > 2 * bound).all()
    assert (np.abs(got[0].double().cpu().numpy() - o)[0, 0] <= bound).all()


@pytest.mark.parametrize("dim,kind,packed,group", [(128, "bf16", False, 16384), (256, "f32", True, 4096 + 5), (192, "f16", False, 8192)])
def test_row_tiles_that_fill_the_chip_take_no_workspace(lpq, dim, kind, packed, group):
    """Some of the rows are checked.  (The size that the library names is enough for queries of any type, this call's takes none.)"""
    c = Case(lpq, 1, dim, 64, [1500, 90], kind, packed, seed=37)
    q = c.queries(group)
    out, lse = c.cache.attend(q.cuda(), ints(c.lengths), c.table, return_lse=True, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    some = np.r_[0:3, 700:703, group - 5:group]
    c.check_attention(q[:, :, some], out[:, :, some], lse[:, :, some], len(some))
