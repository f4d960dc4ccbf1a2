"""A decoder layer on codes from end to end: projections by Linear8, keys and queries turned on the way into the cache, attention with a window or
over a tree of drafted tokens, and the projection back.  Each step against float64 on what the step before gave, so that bounds do not pile up."""
import numpy as np
import pytest
import torch

import kv_plain as plain
from test_gpu_kv_cache import lpq  # noqa: F401  (a fixture)
from test_gpu_kv_masked import attend, random_tree, tree_mask, window_mask

pytestmark = pytest.mark.gpu

HEADS, GROUP, DIM, WIDTH, PAGE = 2, 3, 64, 200, 16
UNIT = 2.0 ** -8                                             # bfloat16: largest relative rounding error


def linear_is(layer, x, y, w):
    """Codes off by half a step in both factors: sum |x| sb / 2 + |w| sa / 2 + d sa sb / 4, in 64 bits; then a rounding."""
    x, w, y = x.double().cpu(), w.double().cpu(), y.double().cpu()
    sa, sb = x.abs().amax(1, keepdim=True) / 127, w.abs().amax(1) / 127
    want = x @ w.t()
    bound = (x.abs().sum(1, keepdim=True) * sb + w.abs().sum(1) * sa + x.shape[1] * sa * sb / 2) / 2 * (1 + 1e-5)
    assert ((y - want).abs() <= bound + UNIT * (want.abs() + bound)).all()


def turned(x, at):
    """Pairs half a head apart, angles of positions `at`, in 64 bits."""
    half = DIM // 2
    angle = torch.as_tensor(at, dtype=torch.float64)[:, None] * 10_000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x.double().cpu().split(half, -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("way", ["window", "tree"])
def test_a_layer(lpq, way, packed):
    from paper_2110_08919_amd import decode
    g = torch.Generator().manual_seed(5)
    rng = np.random.default_rng(5)
    f, old, new = HEADS * DIM, [90, 7, 0], 6
    # queries, keys, values
    w_in, w_out = torch.randn((GROUP + 2) * f, WIDTH, generator=g).bfloat16(), torch.randn(WIDTH, GROUP * f, generator=g).bfloat16() * 0.1
    first, last = lpq.Linear8(w_in.cuda()), lpq.Linear8(w_out.cuda())
    quant, constants = [], []
    for spread in (30.0, 20.0):
        k, width = torch.zeros(f), torch.full((f,), 3.0 * spread)
        quant.append(lpq.Quantizer(f, 4 if packed else 8).set_params(k, -width, width))
        constants.append([t.reshape(HEADS, DIM) for t in quant[-1].get_params()])
    cache = lpq.KVCache(*quant, heads=HEADS, page=PAGE, pages=24, packed=packed)
    table = torch.arange(24, dtype=torch.int32, device="cuda").view(3, 8)
    cos, sin = decode.angles(200, DIM)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    tree = random_tree(rng, new)
    depth = np.array([int(tree[i].sum()) - 1 for i in range(new)])

    def project(count):
        x = torch.randn(count, WIDTH, generator=g).bfloat16().cuda()
        y = first(x)
        linear_is(first, x, y, w_in)
        q, k, v = y.split([GROUP * f, f, f], 1)
        return q.view(count, -1, DIM), k.view(count, HEADS, DIM), v.view(count, HEADS, DIM)

    def add(at, counts, positions=None):
        q, k, v = project(sum(counts))
        where = np.concatenate([np.arange(a, a + n) for a, n in zip(at, counts)]) if positions is None else positions
        out = cache.write_rotated(k, v, ints(at), table, cos, sin, starts=ints(np.cumsum([0] + counts).tolist()), q=q,
                                  positions=None if positions is None else ints(positions.tolist()))
        want = turned(q, where)
        # angles to 2^-25 of 1, three roundings to binary32, one to the type
        size = torch.cat([q.double().cpu().abs()[..., :DIM // 2] + q.double().cpu().abs()[..., DIM // 2:]] * 2, -1)
        assert ((out.double().cpu() - want).abs() <= UNIT * want.abs() + 5 * 2.0 ** -24 * size).all()
        kt = turned(k, where)
        rk, rv = cache.read(ints(at), table, ints(np.cumsum([0] + counts).tolist()), sum(counts))
        for got, t, (mean, _, _, m) in ((rk, kt, constants[0]), (rv, v.double().cpu(), constants[1])):
            step = 1.0 / torch.as_tensor(m).double()
            inside = t.abs() <= 3.0 * (30.0 if got is rk else 20.0) - step
            assert ((got.double().cpu() - t).abs() <= step * 0.5001 + 1e-4)[inside].all()
        return out, rk.double().cpu().numpy(), rv.double().cpu().numpy()

    _, rk, rv = add([0, 0, 0], old)
    drafted = np.concatenate([[a + d for d in depth] for a in old]) if way == "tree" else None
    q, nk, nv = add(old, [new] * 3, drafted)
    lengths = [a + new for a in old]
    kw = dict(tree=torch.from_numpy(tree).cuda()) if way == "tree" else dict(window=30, sinks=2)
    o = cache.attend(q.view(3, new, HEADS * GROUP, DIM), ints(lengths), table, **kw)
    begin = np.cumsum([0] + old)
    for b, n in enumerate(lengths):
        kx, vx = np.concatenate([rk[begin[b]:begin[b + 1]], nk[b * new:(b + 1) * new]]), np.concatenate([rv[begin[b]:begin[b + 1]], nv[b * new:(b + 1) * new]])
        sees = tree_mask(n, new, tree) if way == "tree" else window_mask(n, new, 30, 2)
        rows = q.view(3, new, HEADS * GROUP, DIM)[b].float().cpu().numpy()
        want, _ = attend(rows, kx, vx, GROUP, DIM ** -0.5, sees)
        kc = type("Constants", (), dict(s=1.0 / np.asarray(constants[0][3], np.float64), k=np.asarray(constants[0][0], np.float64)))
        codes = np.rint((kx - kc.k) / kc.s - 0.5)
        err, _ = plain.attend_bound(rows, codes, vx, kc, GROUP, DIM ** -0.5, "bf16")
        assert (np.abs(o[b].double().cpu().numpy() - want) <= err).all()
    y = last(o.view(3, new, -1))
    linear_is(last, o.reshape(3 * new, -1), y.view(3 * new, WIDTH), w_out)


def test_the_decoder_with_codes_rotation_and_a_window():
    from paper_2110_08919_amd import decode
    g = torch.Generator().manual_seed(0)
    prompts = [torch.randint(500, (n,), generator=g).tolist() for n in (150, 1, 37)]
    # the cache's bounds are those of the decoder without these: its codes are not coarser
    for more in (dict(rotate=True), dict(window=20, sinks=2), dict(rotate=True, window=20)):
        shape = decode.Shape(layers=2, width=256, heads=6, kv_heads=2, dim=48, vocabulary=500, page=16, **more)
        for codes in (False, True):
            d = decode.Decoder(shape, prompts, 12, codes=codes)
            assert max(d.errors(0)) < 0.06 and max(d.errors(0)) < 0.06
            tokens = [d.step(0).tolist() for _ in range(5)]
            assert all(0 <= t < 500 for row in tokens for t in row) and d.lengths.tolist() == [157, 8, 44]


def test_command_with_codes_rotation_and_a_window(capsys):
    from paper_2110_08919_amd import decode
    r = decode.main(["--prompt", "600", "--conversations", "2", "--steps", "3", "--pages", "0", "--layers", "2", "--codes", "--rotate", "--window", "100"])
    assert "tokens/s" in capsys.readouterr().out and max(r["all_pages"]) < 0.06
