"""Linear layers on 8-bit codes against their definition: codes and sums are whole numbers and have to be equal; the products with the
scales are roundings to binary32 in a stated order, computed here on the CPU."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def make(m, d, kind, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, d, generator=g) * torch.exp(torch.randn(m, 1, generator=g)) * scale
    return x.to(TYPES[kind])


def codes_of(x):
    """Codes (int64) and scales (float32) of rows, by the definition."""
    x = x.float().numpy()
    most = np.abs(x).max(1, keepdims=True)
    with np.errstate(all="ignore"):
        up = np.where(most < np.float32(2.0 ** -100), np.float32(2.0 ** 60), np.float32(1)).astype(np.float32)
        by = np.where(most > 0, np.float32(127) / (most * up), np.float32(0)).astype(np.float32)
        codes = np.rint((x * up) * by)
        scales = (most / np.float32(127))[:, 0]
    bad = ~np.isfinite(most[:, 0])
    codes[bad] = 0
    scales[bad] = np.nan
    return torch.from_numpy(codes.astype(np.int64)), torch.from_numpy(scales.astype(np.float32))


def rows_of(codes):
    """Rows with their ends behind feature d."""
    return codes.blocks.permute(0, 3, 1, 2, 4).flatten(2).flatten(0, 1)[:codes.n]


def product_of(a, sa, b, sb, bias, dtype):
    """fl(fl(fl(sum) sa) sb) [+ bias] to dtype."""
    sums = a.double() @ b.double().t()                       # exact: below 2^53
    y = sums.float() * sa[:, None] * sb
    return (y if bias is None else y + bias).to(dtype)


def same(got, want):
    got = got.cpu()
    assert got.shape == want.shape and got.dtype is want.dtype
    both = torch.isnan(got) & torch.isnan(want)
    assert torch.equal(torch.where(both, torch.zeros_like(got), got), torch.where(both, torch.zeros_like(want), want))


# ------------------------------------------------------------------------------ rows ----
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,d", [(1, 1), (3, 7), (5, 127), (2, 128), (9, 513), (4, 2048), (3, 2049), (2, 8200), (3, 16_385), (2, 40_001), (1, 131_072)])
def test_rows_to_codes(kind, n, d):
    from paper_2110_08919_amd import lpq
    x = make(n, d, kind, 7 * d + n)
    got = lpq.encode_rows(x.cuda())
    codes, scales = codes_of(x)
    stride = (d + 127) // 128 * 128
    assert got.codes.shape == (n, d) and got.n == n and got.d == d
    assert torch.equal(got.codes.cpu().long(), codes)
    blocks = got.blocks.cpu()
    assert blocks.shape == ((n + 15) // 16, stride // 64, 4, 16, 16)
    for i, k in ((0, 0), (n - 1, d - 1), (n // 2, d // 3)):
        assert blocks.flatten()[(i // 16 * (stride // 64) + k // 64) * 1024 + k % 64 // 16 * 256 + i % 16 * 16 + k % 16] == codes[i, k]
    assert not rows_of(got)[:, d:].any()
    assert torch.equal(got.scales.cpu(), scales)
    assert torch.equal(got.float().cpu(), codes.float() * scales[:, None])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_rows_of_any_size_and_rows_that_are_not_finite(kind):
    from paper_2110_08919_amd import lpq
    x = make(12, 300, kind, 3).float()
    for i, size in enumerate((0.0, 1e-40, 1e-38, 1e-33, 2.0 ** -100, 1e-20, 1e20, 3e37)):
        x[i] *= size / x[i].abs().max().clamp(min=1e-30) if size else 0.0
    x[8, 77], x[9, 0], x[10, 299] = float("inf"), float("nan"), -float("inf")
    x = x.to(TYPES[kind])
    got = lpq.encode_rows(x.cuda())
    codes, scales = codes_of(x)
    assert torch.equal(got.codes.cpu().long(), codes)
    same(got.scales, scales)
    assert codes[1].abs().max() == 127 and torch.isnan(scales[8:11]).all() and scales[0] == 0
    w = make(40, 300, kind, 4)
    layer = lpq.Linear8(w.cuda())
    b, sb = codes_of(w)
    y = layer(x.cuda())
    # the roundings of the definition, with the scales' exponents taken apart so that nothing leaves binary32 on the way
    sa_m, sa_e = np.frexp(scales.numpy())
    sb_m, sb_e = np.frexp(sb.numpy())
    t = (codes.double() @ b.double().t()).float().numpy() * sa_m[:, None] * sb_m
    want = torch.from_numpy(np.ldexp(t.astype(np.float64), sa_e[:, None] + sb_e).astype(np.float32)).to(TYPES[kind])
    same(y, want)
    assert torch.isnan(y[8:11]).all() and not torch.isnan(y[:8]).any() and not y[0].any()


def test_scales_whose_products_pass_the_range_of_binary32():
    """Sums of large rows times their scale would be infinite, times the channel's small scale they are not; and the other way round."""
    from paper_2110_08919_amd import lpq
    x, w = torch.full((2, 4000), 1e37), torch.full((70, 4000), 1e-35)
    x[1], w[35:] = 1e-30, 1e33
    y = lpq.Linear8(w.cuda())(x.cuda()).cpu().double()
    want = x.double() @ w.double().t()
    # constant rows: codes 127; two scales and their products, 5 roundings in all (denormals: half their step more)
    assert (torch.isfinite(y) == (want < 3.4e38)).all()
    few = torch.isfinite(y)
    assert ((y - want).abs()[few] <= 6 * 2.0 ** -24 * want[few] + 2.0 ** -149).all()


def test_rows_with_strides_at_odd_places():
    from paper_2110_08919_amd import lpq
    for kind in TYPES:
        whole = make(9, 700, kind, 11).cuda()
        x = whole[1:8, 3:556]
        got, want = lpq.encode_rows(x), lpq.encode_rows(x.contiguous())
        assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales)
        one = whole[2:3, 5:300].expand(6, -1)
        assert torch.equal(lpq.encode_rows(one).codes, lpq.encode_rows(one.contiguous()).codes)


# -------------------------------------------------------------------------- products ----
SIZES = [(1, 1, 1), (1, 64, 64), (1, 1000, 4096), (1, 257, 16_384), (1, 40, 20_000), (2, 100, 129), (3, 129, 65), (4, 2000, 500), (5, 333, 4100),
         (8, 96, 2048), (9, 31, 2000), (15, 17, 1000), (17, 100, 300), (31, 300, 130), (33, 1111, 700), (48, 333, 1025), (64, 65, 128), (65, 200, 257),
         (96, 128, 640), (100, 1300, 77), (127, 129, 513), (128, 128, 128), (129, 127, 100), (130, 515, 1000), (200, 64, 16_384), (256, 256, 64),
         (257, 300, 8200), (300, 700, 1111), (600, 1000, 300), (513, 2100, 200), (1500, 400, 130)]


@pytest.mark.parametrize("m,n,d", SIZES)
@pytest.mark.parametrize("kind,with_bias", [("bf16", False), ("f16", True), ("f32", True)])
def test_layer(m, n, d, kind, with_bias):
    from paper_2110_08919_amd import lpq
    x, w = make(m, d, kind, m), make(n, d, kind, n + 1, 0.1)
    bias = torch.randn(n, generator=torch.Generator().manual_seed(d)) if with_bias else None
    layer = lpq.Linear8(w.cuda(), None if bias is None else bias.cuda())
    assert (layer.d, layer.channels) == (d, n)
    (a, sa), (b, sb) = codes_of(x), codes_of(w)
    same(layer(x.cuda()), product_of(a, sa, b, sb, bias, TYPES[kind]))
    same(lpq.matmul_i8(lpq.encode_rows(x.cuda()), layer.weight, layer.bias, TYPES[kind]), product_of(a, sa, b, sb, bias, TYPES[kind]))


# One product for every way that they go: tokens and channels of a workgroup, parts.
WAYS = [(16, 16, 0, 9, 70, 2100), (16, 32, 0, 13, 4200, 300), (16, 48, 0, 16, 11_003, 260), (16, 64, 0, 10, 13_000, 100),
        (32, 16, 0, 20, 600, 1400), (32, 32, 0, 32, 5001, 520), (32, 48, 0, 17, 12_000, 130), (32, 64, 0, 30, 12_400, 64),
        (48, 16, 0, 35, 500, 1100), (48, 32, 0, 48, 4500, 400), (48, 48, 0, 41, 9000, 770), (48, 64, 0, 33, 12_345, 500),
        (64, 16, 0, 50, 3900, 1000), (64, 32, 0, 64, 8100, 1030), (64, 48, 0, 49, 12_000, 2000), (64, 64, 0, 63, 13_000, 2100),
        (96, 16, 0, 96, 4090, 2000), (96, 32, 0, 66, 8000, 3000), (96, 48, 0, 90, 9000, 4100),
        (128, 16, 0, 128, 4000, 2000), (128, 32, 0, 100, 8000, 3100),
        (64, 64, 1, 129, 333, 200), (64, 64, 1, 500, 900, 64), (128, 128, 1, 2000, 2100, 300), (128, 128, 1, 1111, 4097, 70),
        (256, 256, 1, 3900, 4001, 2600), (64, 64, 2, 4000, 130, 3000), (64, 64, 4, 130, 61, 1500), (64, 64, 7, 130, 60, 2100),
        (64, 64, 16, 131, 59, 6000), (128, 128, 2, 2000, 1001, 16_400), (128, 128, 4, 200, 4099, 8200), (128, 128, 8, 1100, 300, 16_400)]


@pytest.mark.parametrize("rows,channels,parts,m,n,d", WAYS)
def test_every_way_a_product_goes(rows, channels, parts, m, n, d):
    from paper_2110_08919_amd import lpq
    assert lpq.linear8_plan_info(m, n, d)[:3] == [rows, channels, parts]
    for kind in ("bf16", "f32"):
        x, w = make(m, d, kind, m).cuda(), make(n, d, kind, n + 1, 0.1).cuda()
        bias = torch.randn(n, generator=torch.Generator().manual_seed(d)).cuda()
        a, b = lpq.encode_rows(x), lpq.encode_rows(w)
        sums = a.codes.double() @ b.codes.double().t().contiguous()          # whole numbers below 2^53
        want = ((sums.float() * a.scales[:, None]) * b.scales + bias).to(TYPES[kind])
        got = lpq.matmul_i8(a, b, bias, TYPES[kind])
        assert torch.equal(got, want)
        if kind == "bf16":
            out = torch.full((m, n + 3), 5.0, dtype=TYPES[kind], device="cuda")
            assert torch.equal(lpq.Linear8(w, bias)(x, out=out[:, 1:-2]), want)
            assert (out[:, :1] == 5).all() and (out[:, -2:] == 5).all()


@pytest.mark.parametrize("m,n", [(1, 3), (2, 40), (70, 33), (140, 130)])
def test_the_largest_sums(m, n):
    """131 072 products of 127 by 127, and of 127 by -127: the longest rows, near both ends of 32 bits."""
    from paper_2110_08919_amd import lpq
    x, w = torch.ones(m, 131_072), torch.ones(n, 131_072)
    w[n // 2:] = -1.0
    y = lpq.Linear8(w.cuda())(x.cuda()).cpu().double()
    want = x[:, :1].double() * w[:, 0].double() * 131_072
    assert ((y - want).abs() <= 6 * 2.0 ** -24 * 131_072).all()        # scales fl(1 / 127), the sum and two products: 5 roundings


def test_a_row_does_not_depend_on_the_rows_beside_it():
    from paper_2110_08919_amd import lpq
    x, w = make(700, 1500, "bf16", 1).cuda(), make(900, 1500, "bf16", 2).cuda()
    layer = lpq.Linear8(w)
    whole = layer(x)
    for at, count in ((0, 1), (699, 1), (5, 3), (100, 16), (30, 47), (500, 130), (0, 300)):
        assert torch.equal(layer(x[at:at + count]), whole[at:at + count])
    for at, count in ((0, 1), (7, 130), (450, 450)):
        assert torch.equal(lpq.Linear8(w[at:at + count])(x), whole[:, at:at + count])


@pytest.mark.parametrize("m", [1, 3, 40, 100, 300])
def test_shapes_strides_and_what_lies_beside_the_output(m):
    from paper_2110_08919_amd import lpq
    x, w = make(m, 333, "f16", 5).cuda(), make(77, 333, "f16", 6).cuda()
    layer = lpq.Linear8(w)
    want = layer(x)
    assert torch.equal(layer(x.view(1, m, 333)), want.view(1, m, 77)) and torch.equal(layer(x[0]), want[0])
    buffer = torch.full((m + 2, 91), 7.0, dtype=torch.float16, device="cuda")
    out = buffer[1:-1, 5:82]
    assert layer(x, out=out) is out
    assert torch.equal(out, want)
    buffer[1:-1, 5:82] = 7.0
    assert (buffer == 7.0).all()
    wide = torch.zeros(m, 400, dtype=torch.float16, device="cuda")
    wide[:, 9:342] = x
    assert torch.equal(layer(wide[:, 9:342]), want)
    need = lpq.lib().lpq_linear8_workspace_bytes(m, 77, 333)
    space = torch.full((need + 512,), 90, dtype=torch.uint8, device="cuda")
    assert torch.equal(layer(x, workspace=space[256:256 + need]), want)
    assert (space[:256] == 90).all() and (space[256 + need:] == 90).all()


def test_codes_whose_rest_of_a_row_is_not_zero():
    """Bytes behind d count where both operands have some, as the interface says; zeros in one are enough."""
    from paper_2110_08919_amd import lpq
    for m in (1, 40, 200):
        x, w = make(m, 200, "f32", 8), make(150, 200, "f32", 9)
        a, b = lpq.encode_rows(x.cuda()), lpq.encode_rows(w.cuda())
        want = lpq.matmul_i8(a, b, dtype=torch.float32)
        b.blocks[:, 3, 0, :, 8:] = 99
        b.blocks[:, 3, 1:] = -99
        a.blocks[m // 16:, :, :, m % 16:] = 77               # rows behind the last
        b.blocks[150 // 16:, :, :, 150 % 16:] = 55
        assert torch.equal(lpq.matmul_i8(a, b, dtype=torch.float32), want)


def test_no_rows_no_channels():
    from paper_2110_08919_amd import lpq
    layer = lpq.Linear8(make(5, 64, "f32", 1).cuda())
    assert layer(torch.empty(0, 64, device="cuda")).shape == (0, 5)
    assert lpq.encode_rows(torch.empty(0, 64, device="cuda")).n == 0
    none = lpq.Linear8(torch.empty(0, 64, device="cuda"))
    assert none(torch.ones(3, 64, device="cuda")).shape == (3, 0)


@pytest.mark.parametrize("m,n,d", [(1, 500, 700), (40, 500, 700), (200, 300, 4000), (600, 1000, 300)])
def test_another_stream_and_captured_graphs(m, n, d):
    """Two graphs of one layer with inputs of their own, replayed in turn with eager calls between."""
    from paper_2110_08919_amd import lpq
    layer = lpq.Linear8(make(n, d, "bf16", 1).cuda())
    xs = [make(m, d, "bf16", 10 + i).cuda() for i in range(6)]
    wants = [layer(x) for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer(xs[1])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, wants[1])
    fed = [xs[0].clone(), xs[0].clone()]
    graphs, outs = [], []
    for x in fed:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(layer(x))
        graphs.append(g)
    for i in range(6):
        for j in range(2):
            fed[j].copy_(xs[(i + j) % 6])
        for g in graphs:
            g.replay()
        assert torch.equal(layer(xs[5 - i]), wants[5 - i])
        for j in range(2):
            assert torch.equal(outs[j], wants[(i + j) % 6])


def test_refusals():
    from paper_2110_08919_amd import lpq
    w = make(5, 64, "f32", 1).cuda()
    layer = lpq.Linear8(w.clone().requires_grad_())          # a parameter's values, without its gradient
    x = make(3, 64, "f32", 2).cuda()
    with pytest.raises(AssertionError):
        layer(x.clone().requires_grad_())
    with torch.no_grad():
        assert torch.equal(layer(x.clone().requires_grad_()), layer(x))
    for bad in (x[:, :63], x.double(), x.cpu(), x.t()):
        with pytest.raises(AssertionError):
            layer(bad)
    with pytest.raises(AssertionError):
        layer(x, out=torch.empty(3, 5, dtype=torch.float16, device="cuda"))
    with pytest.raises(AssertionError):
        lpq.Linear8(w, torch.zeros(4, device="cuda"))
    with pytest.raises(AssertionError):
        lpq.encode_rows(w.clone().requires_grad_())
    with pytest.raises(lpq.LpqError):
        layer(x, out=torch.empty(1, 5, device="cuda").expand(3, 5))
    with pytest.raises(lpq.LpqError):
        layer(x.repeat(10, 1), workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(AssertionError):
        lpq.matmul_i8(lpq.encode_rows(x), lpq.encode_rows(x[:, :60]))
    bias = torch.ones(5, device="cuda")
    layer = lpq.Linear8(w, bias)
    want = layer(x)
    bias.zero_()
    assert torch.equal(layer(x), want)                       # the layer keeps its own
