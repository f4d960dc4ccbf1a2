"""Key-value cache on a real MI355X at the edges of what a caller may pass."""
import numpy as np
import pytest
import torch

import kv_plain as plain
from test_gpu_kv_cache import TYPES, Case, ints, lpq  # noqa: F401  (lpq is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("starts", [[0, 20, 40], [5, 20, 53], [0, 0, 0], [53, 53, 53], [3, 8, 8]])
def test_rows_of_no_sequence_are_dropped_and_read_back_as_zeros(lpq, starts, packed):
    """More rows than the sequences have, at the end or ahead of the first: a caller with rows for the most there can be."""
    c = Case(lpq, 3, 40, 16, [20, 53], "f16", packed)
    n = 53
    rows = [np.zeros((n, 3, 40)) for _ in range(2)]
    for b in range(2):
        for out, held in zip(rows, (c.kx, c.vx)):
            out[starts[b]:starts[b + 1]] = held[b][:starts[b + 1] - starts[b]]
    into = [torch.full((n, 3, 40), 7.0, dtype=torch.float16, device="cuda") for _ in range(2)]
    c.cache.read(ints([0, 0]), c.table, ints(starts), n, out=into)
    for got, want in zip(into, rows):
        assert torch.equal(got.cpu(), torch.from_numpy(want).to(torch.float16))
    # the same rows written leave what the sequences hold as it is
    other = Case(lpq, 3, 40, 16, [20, 53], "f16", packed, write=False)
    given = [torch.full((n, 3, 40), 9.0, dtype=torch.float16) for _ in range(2)]
    for b in range(2):
        for out, held in zip(given, (c.k, c.v)):
            out[starts[b]:starts[b + 1]] = held[b][:starts[b + 1] - starts[b]]
    other.cache.k.fill_(3)
    other.cache.write(*(x.cuda() for x in given), ints([0, 0]), other.table, ints(starts))
    pool = other.cache.k.cpu().numpy()
    written = np.zeros(pool.shape[0] * 16, bool)
    for b in range(2):
        at = np.arange(starts[b + 1] - starts[b])
        written[other.table_np[b][at // 16] * 16 + at % 16] = True
    assert (pool.transpose(0, 2, 1, 3).reshape(len(written), -1)[~written] == 3).all()


def test_rows_without_any_sequence_are_refused(lpq):
    c = Case(lpq, 3, 40, 16, [20], "f16")
    none, rows = torch.zeros(0, 3, dtype=torch.int32, device="cuda"), c.k[0][:4].cuda()
    for call in (lambda: c.cache.read(ints([]), none, ints([0]), 4), lambda: c.cache.write(rows, rows, ints([]), none, ints([0]))):
        with pytest.raises(lpq.LpqError) as e:
            call()
        assert e.value.code == lpq.EINVAL


def test_a_list_without_pages_is_refused(lpq):
    c = Case(lpq, 2, 64, 16, [40, 20])
    with pytest.raises(AssertionError):
        c.cache.attend(c.queries(2).cuda(), ints(c.lengths), c.table, pages=torch.zeros(2, 2, 0, dtype=torch.int32, device="cuda"))


def test_queries_that_require_a_gradient_are_refused(lpq):
    c = Case(lpq, 2, 64, 16, [40, 20], "f32")
    q = c.queries(2).cuda()
    want = c.cache.attend(q, ints(c.lengths), c.table)
    q.requires_grad_()
    with pytest.raises(AssertionError):
        c.cache.attend(q, ints(c.lengths), c.table)
    with torch.no_grad():
        assert torch.equal(c.cache.attend(q, ints(c.lengths), c.table), want)


@pytest.mark.parametrize("room", [None, 1 << 12, 1 << 20])
@pytest.mark.parametrize("group,kind,packed", [(2, "bf16", False), (3, "f16", True), (12, "f32", False)])
def test_rows_that_see_no_token_are_zeros_whatever_the_query_holds(lpq, group, kind, packed, room):
    """Places of a batch without a sequence often hold whatever was in memory; room: tokens that the tables have columns for."""
    c = Case(lpq, 2, 64, 16, [0, 40, 2, 30, 0, 700], kind, packed, seed=3)
    q = c.queries(group, 4)
    table = c.table
    if room:
        table = torch.full((len(c.lengths), room // 16), -1, dtype=torch.int32, device="cuda")
        table[:, :c.table.shape[1]] = c.table
    table = table.clone()
    table[3] = -1                                    # tokens, but no page that holds them
    dead = [np.full(n, b == 3) for b, n in enumerate(c.lengths)]
    lengths = list(c.lengths)
    lengths[4] = -7
    clean, clean_lse = c.cache.attend(q.cuda(), ints(lengths), table, return_lse=True)
    c.check_attention(q, clean, clean_lse, group, dead=dead)
    empty = torch.isneginf(clean_lse)
    bad = q.clone()
    bad[0], bad[3, :, ::2], bad[4] = float("nan"), float("inf"), float("nan")
    bad[2, 0, :], bad[2, 1, 0, 5], bad[2, 3, 1, 2] = -float("inf"), float("nan"), float("nan")
    bad[5, 2, 1, 7] = float("inf")
    out, lse = c.cache.attend(bad.cuda(), ints(lengths), table, return_lse=True)
    assert empty[0].all() and empty[3].all() and empty[4].all() and empty[2, :2].all() and not empty[2, 2:].any()
    assert not out[empty].any() and torch.isneginf(lse[empty]).all()
    spoiled = ~torch.isfinite(bad).all(-1).cuda() & ~empty
    assert spoiled.sum() == 2
    assert torch.isnan(out[spoiled]).all() and torch.isnan(lse[spoiled]).all()
    rest = ~spoiled & ~empty
    assert torch.equal(out[rest], clean[rest]) and torch.equal(lse[rest], clean_lse[rest])


def with_keys(c, k):
    """The first sequence of the case with keys k [n, heads, dim] (numpy) instead of its own."""
    k = torch.from_numpy(np.ascontiguousarray(k, np.float32)).to(TYPES[c.kind])
    n = len(k)
    c.cache.write(k.cuda(), c.v[0].cuda(), ints([0]), c.table[:1], ints([0, n]))
    c.kcodes[0] = plain.codes(k.float().numpy(), c.kc, c.packed)
    c.kx[0] = plain.values(c.kcodes[0], c.kc).astype(np.float64)


@pytest.mark.parametrize("n", [300, 9000])
@pytest.mark.parametrize("kind,packed,strength,scale", [
    ("bf16", False, 1e6, None), ("bf16", True, 1e7, None), ("f32", False, 3e7, None), ("f32", True, 1e9, None), ("f32", False, 1e25, None),
    ("f16", False, 1e3, 1e6), ("f16", True, 1e3, -1e30), ("bf16", False, 1e30, 1.0), ("f32", False, 1e37, 1.0), ("bf16", False, 1e36, 1e30)])
def test_one_token_or_two_alike_take_all(lpq, kind, packed, strength, scale, n):
    """Scores far beyond those at which a float holds whole numbers.  Two tokens with the same keys have the same integer product and
    share the weight; every other token is behind by more than what is rounded, so the result is their values' mean to a few
    roundings: of the sum, the half step, the step and the offset, and to the type."""
    c = Case(lpq, 1, 64, 64, [n], kind, packed, seed=21)
    assert c.dim == 64
    sign = np.where(c.rng.random(64) < 0.5, -1.0, 1.0)
    q = (strength / c.std * sign).astype(np.float32).reshape(1, 1, 1, 64)
    q = torch.from_numpy(np.concatenate([q, 0.5 * q], 2)).to(TYPES[kind])
    by = c.dim ** -0.5 if scale is None else float(np.float32(scale))
    toward = np.sign(by) * sign * c.std
    k = c.mean + 0.5 * c.std * c.rng.standard_normal((n, 64))
    k[[n // 3, n - 5]] = c.mean + 2.0 * toward
    with_keys(c, k.reshape(n, 1, 64))
    qf = q.float().numpy()[0, 0].astype(np.float64)
    t = by * (c.kx[0][:, 0, None] * qf[None]).sum(2)                            # [n, rows]; equal tokens have equal sums
    ranked = np.sort(t, 0)
    e = abs(by) * np.abs(qf * c.kc.s[0]).max(1) / (2 * 16319) * np.abs(c.kcodes[0][:, 0]).sum(1).max()
    assert (ranked[-1] == ranked[-2]).all() and (ranked[-2] - ranked[-3] > 4 * e + 1000).all()
    want = 0.5 * (c.vx[0][n // 3, 0] + c.vx[0][n - 5, 0])
    out, lse = c.cache.attend(q.cuda(), ints([n]), c.table, scale=scale, return_lse=True)
    size = np.maximum(np.abs(c.vx[0][n // 3, 0]), np.abs(c.vx[0][n - 5, 0])) + 256 * c.vc.s[0]
    assert (np.abs(out[0, 0].double().cpu().numpy() - want) <= (plain.UNIT[kind] + 8 * 2.0 ** -24) * size).all()
    want_lse = t.max(0) + np.log(2.0)
    inside = np.abs(want_lse) < 1e38
    total = np.abs(by) * (np.abs(qf) @ np.abs(c.kx[0][:, 0]).max(0))
    assert (np.abs(lse[0, 0].double().cpu().numpy() - want_lse) <= e + 2.0 ** -19 * total + 1e-5)[inside].all()


def scaled_case(lpq, factor, *args, **kw):
    """A case whose key features are `factor` (a number or one per feature) times as wide and as far out."""
    c = Case(lpq, *args, write=False, **kw)
    bits, f = c.kc.bits, c.heads * c.dim
    c.std, c.mean = c.std * factor, c.mean * factor
    width = 4.0 if bits == 8 else 2.5
    ranges = [x.astype(np.float32) for x in (c.mean, c.mean - width * c.std, c.mean + width * c.std)]
    c.kc = plain.Constants(*ranges, bits, c.heads)
    values = lpq.Quantizer(f, bits).set_params(*(x.reshape(-1) for x in (c.vc.k, c.vc.sb, c.vc.se)))
    c.cache = lpq.KVCache(lpq.Quantizer(f, bits).set_params(*ranges), values, heads=c.heads, page=c.page, pages=c.cache.pages, packed=c.packed)
    c.k = [torch.from_numpy((c.rng.standard_normal((n, f)) * c.std + c.mean).astype(np.float32)).to(TYPES[c.kind]).view(n, c.heads, c.dim)
           for n in c.lengths]
    c.kcodes = [plain.codes(x.float().numpy(), c.kc, c.packed) for x in c.k]
    c.kx = [plain.values(x, c.kc).astype(np.float64) for x in c.kcodes]
    c.cache.write(torch.cat(c.k).cuda(), torch.cat(c.v).cuda(), ints([0] * len(c.lengths)), c.table, ints(c.starts.tolist()))
    return c


@pytest.mark.parametrize("lengths", [[300, 1, 0], [5000]])
@pytest.mark.parametrize("kind,packed,factor,size", [("f32", False, 1e4, 1e37), ("bf16", False, 1e4, 1e37), ("f32", True, 1e4, 2e37),
                                                     ("f32", False, 1.0, 1e-33), ("bf16", False, 1.0, 3e-36), ("f32", True, 1.0, 1e-38)])
def test_queries_whose_products_with_the_steps_are_very_large_or_small(lpq, kind, packed, factor, size, lengths):
    """Finite queries q with q s beyond binary32, or far below 1, at a scale that makes the scores ordinary numbers."""
    c = scaled_case(lpq, factor, 1, 64, 64, lengths, kind, packed, seed=22)
    q = torch.from_numpy((c.rng.standard_normal((len(lengths), 2, 3, 64)) * size).astype(np.float32)).to(TYPES[kind])
    scaled = q.double().numpy() * c.kc.s[0].astype(np.float64)
    assert torch.isfinite(q).all() and (np.abs(scaled).max() > 3.5e38 if factor > 1 else np.abs(scaled).max() < 1e-30)
    scale = float(np.float32(2.0 / (np.sqrt((c.std ** 2).sum()) * size)))
    assert 0 < scale < 3e38
    out, lse = c.cache.attend(q.cuda(), ints(lengths), c.table, scale=scale, return_lse=True)
    c.check_attention(q, out, None, 3, scale=scale)
    for b, n in enumerate(lengths):                  # the bound of lse holds sums of |q| |k| that float32 does not
        qb = q[b].double().numpy()
        want = plain.attend(qb, c.kx[b], c.vx[b], 3, scale)[1]
        bound = plain.attend_bound(qb, c.kcodes[b], c.vx[b], c.kc, 3, scale, kind)[1]
        got, seen = lse[b].double().cpu().numpy(), np.isfinite(want)
        assert np.isfinite(bound).all() and (np.abs(got[seen] - want[seen]) <= bound[seen]).all() and np.isneginf(got[~seen]).all()


@pytest.mark.parametrize("spread", [20.0, 100.0])
@pytest.mark.parametrize("kind,packed", [("f16", False), ("f16", True), ("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
def test_features_of_very_different_sizes(lpq, kind, packed, spread):
    """One key feature far wider than the others, queries that do not make up for it, scores of standard deviation 8: what a query loses
    where its row is held to a number of bits of its largest entry.  Root mean square error over the rows against 64 bits.

    16-bit results: relative to what rounding the exact result to the type costs (u / sqrt(3) or less of each value).  Weights in fp16 have
    an error of the same kind and, for float16, of at most the same size: a factor of sqrt(2) there, 1.01 for bfloat16; a query's own
    rounding may add a third of the result's to bfloat16 (1.05) and nothing that shows to float16.  float32: no further off than
    scores, weights and sums in float32 of the same keys and values."""
    factor = np.ones(256)
    factor[[5, 128 + 77]] = spread
    c = scaled_case(lpq, factor, 2, 128, 64, [4000, 1500], kind, packed, seed=23)
    q = c.rng.standard_normal((2, 1, 2, 4, 128))
    q *= 8.0 * 128 ** 0.5 / np.sqrt((c.std ** 2).reshape(2, 1, 128).sum(2, keepdims=True))
    q = torch.from_numpy(q.reshape(2, 1, 8, 128).astype(np.float32)).to(TYPES[kind])
    out = c.cache.attend(q.cuda(), ints(c.lengths), c.table).double().cpu().numpy()
    exact = np.stack([plain.attend(q[b].float().numpy(), c.kx[b], c.vx[b], 4, 128 ** -0.5)[0] for b in range(2)])
    if kind == "f32":
        least, factor = np.zeros_like(exact), 1.0
        for b in range(2):
            for j in range(8):
                t = (torch.from_numpy(c.kx[b][:, j // 4]).float() @ q[b, 0, j]) * 128 ** -0.5
                least[b, 0, j] = (torch.softmax(t, 0) @ torch.from_numpy(c.vx[b][:, j // 4]).float()).double().numpy()
    else:
        least, factor = torch.from_numpy(exact).to(TYPES[kind]).double().numpy(), {"f16": 1.42, "bf16": 1.1}[kind]
    off, most = (np.sqrt(((x - exact) ** 2).mean()) for x in (out, least))
    print(f"error {off:.3e}, of the reference form {most:.3e}")
    assert off <= factor * most


@pytest.mark.parametrize("room", [16, 4096])
@pytest.mark.parametrize("kind,packed", [("f32", False), ("f32", True), ("f16", False), ("bf16", False), ("bf16", True)])
def test_a_token_alone_comes_out_as_it_reads_back(lpq, kind, packed, room):
    """Also where its offset and its code nearly cancel: the same bits as read() gives."""
    c = Case(lpq, 5, 100, 16, [1] * 60, kind, packed, seed=24)
    table = torch.full((60, room // 16), -1, dtype=torch.int32, device="cuda")
    table[:, :1] = c.table
    out = c.cache.attend(c.queries(3).cuda(), ints(c.lengths), table)
    want = c.cache.read(ints([0] * 60), c.table, dtype=TYPES[kind])[1]
    assert torch.equal(out, want.repeat_interleave(3, 1).view(out.shape))


@pytest.mark.parametrize("n", [1, 20, 33])
def test_fewer_rows_than_the_sequences_have(lpq, n):
    c = Case(lpq, 3, 40, 16, [20, 53], "f16")
    k, v = c.cache.read(ints([0, 0]), c.table, ints([0, 20, 73]), n, TYPES["f16"])
    for got, held in ((k, c.kx), (v, c.vx)):
        assert torch.equal(got.cpu(), torch.from_numpy(np.concatenate(held)[:n]).to(torch.float16))
    other = Case(lpq, 3, 40, 16, [20, 53], "f16", write=False)
    other.cache.write(torch.cat(other.k)[:n].cuda(), torch.cat(other.v)[:n].cuda(), ints([0, 0]), other.table, ints([0, 20, 73]))
    k, _ = other.cache.read(ints([0, 0]), other.table, ints([0, 20, 73]), n, TYPES["f16"])
    assert torch.equal(k.cpu(), torch.from_numpy(np.concatenate(c.kx)[:n]).to(torch.float16))
