"""The work of a decoder layer that runs on codes, beyond keeping and reading a cache, as cases that can be timed.

Four kinds of call, each through the public binding:

    rotate      KVCache.write_rotated: new queries and keys turned by their positions' angles, keys and values into the
                cache as codes; and KVCache.read of the rows just written
    window      KVCache.attend where a token sees its window and the first few tokens (sinks)
    tree        KVCache.attend of drafted tokens that form a tree: each sees the cache and its own ancestors
    linear      Linear8: rows of a model's type to 8-bit codes with a scale for each, their product with 8-bit weights that
                have a scale for each channel, and a bias

The plain form of each kind is in elementary torch operations in float32; `exact` restates the definitions in float64.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
WIDTH = {8: 4.0, 4: 2.5}                    # range of a code in standard deviations to each side
MAX_ROTATED = 24_000 * 8 * 128              # values of keys (or of values) of a call
MAX_SCORES = 32 * 8000 * 32 * 48            # (tokens, query row) pairs of an attention call, padded to the longest sequence
MAX_CODES = 32 * 8000 * 8 * 128             # key codes that it goes over, padded likewise
MAX_PRODUCTS = 8192 ** 3


def _cache_case(name, kind, type_, seqs, lo, hi, heads, dim, page, bits=8, group=1, new=1, new_hi=None, rotated=0,
                interleaved=False, depths=False, window=0, sinks=0):
    return {"name": name, "kind": kind, "type": type_, "seqs": seqs, "lo": lo, "hi": hi, "heads": heads, "dim": dim,
            "page": page, "bits": bits, "group": group, "new": new, "new_hi": new_hi or new, "rotated": rotated,
            "interleaved": interleaved, "depths": depths, "window": window, "sinks": sinks}


def _linear_case(name, type_, rows, features, channels, bias=False):
    return {"name": name, "kind": "linear", "type": type_, "rows": rows, "features": features, "channels": channels,
            "bias": bias}


def listed():
    return [
        # One token of one conversation, far along: all launch latency.
        _cache_case("rotate_one", "rotate", "bf16", 1, 30_000, 30_000, 8, 128, 64, group=4, rotated=128),
        # Drafted trees of 16 conversations: several rows stand at one position, each at its depth in the tree.
        _cache_case("rotate_drafts", "rotate", "f32", 16, 500, 6000, 2, 80, 32, group=6, new=20, rotated=64, depths=True),
        # New prompts of very different lengths, half of each head turned, pairs of neighbours, two codes per byte.
        _cache_case("rotate_prompts", "rotate", "f16", 12, 0, 300, 6, 100, 32, bits=4, group=3, new=37, new_hi=4000,
                    rotated=52, interleaved=True),
        # The first parts of long prompts.
        _cache_case("rotate_large", "rotate", "bf16", 8, 0, 9000, 8, 128, 64, group=4, new=1000, new_hi=5000, rotated=128),
        # The next token of one long conversation.
        _cache_case("window_one", "window", "bf16", 1, 50_000, 50_000, 8, 128, 64, group=4, window=4096, sinks=4),
        # A generation step of many conversations, some shorter than the window.
        _cache_case("window_step", "window", "bf16", 64, 700, 20_000, 8, 128, 64, group=4, window=2000, sinks=20),
        # Parts of prompts of a small model, two codes per byte: each token has a window of its own.
        _cache_case("window_prompt", "window", "f16", 4, 1500, 9000, 4, 96, 32, bits=4, group=4, new=1500, window=600, sinks=1),
        # Trees of 24 drafted tokens are checked for a service's conversations.
        _cache_case("tree_step", "tree", "bf16", 32, 900, 8000, 8, 128, 64, group=4, new=24),
        # One conversation, a larger tree, float32, many query heads on one key head.
        _cache_case("tree_one", "tree", "f32", 1, 5000, 5000, 1, 192, 32, bits=4, group=12, new=60),
        # The projection of one token.
        _linear_case("linear_token", "bf16", 1, 4096, 4096),
        # A generation step of 48 conversations through a wide layer, odd in every size.
        _linear_case("linear_step", "f16", 48, 4100, 11_111, bias=True),
        # A prompt.
        _linear_case("linear_prompt", "bf16", 8192, 8192, 8192),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "window", "window", "tree", "tree", "linear", "linear"])
    type_ = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "linear":
        rows = rng.choice([1, _log_uniform(rng, 1, 128), _log_uniform(rng, 1, 8192)])
        features = _log_uniform(rng, 64, 16_384)
        channels = _log_uniform(rng, 64, max(64, min(32_768, MAX_PRODUCTS // (rows * features))))
        case = _linear_case("", type_, rows, features, channels, bias=rng.random() < 0.4)
        del case["name"]
        return case
    heads, page, group = _log_uniform(rng, 1, 12), rng.choice([16, 32, 64, 128]), rng.choice([1, 2, 4, 5, 8, 12])
    dim = rng.choice([64, 80, 96, 128, 128, 192, 256, rng.randint(33, 255)])
    seqs = _log_uniform(rng, 1, 64)
    case = _cache_case("", kind, type_, seqs, 0, 0, heads, dim, page, bits=rng.choice([8, 8, 4]), group=group)
    del case["name"]
    if kind == "rotate":
        # (queries count too: the largest listed case has four query heads to a key head)
        room = MAX_ROTATED * 6 // (heads * dim * (group + 2))
        depths = rng.random() < 0.2
        new_hi = rng.randint(2, 64) if depths else 1 if rng.random() < 0.3 else max(1, _log_uniform(rng, 2, 5000))
        new_hi = max(1, min(new_hi, room // seqs))
        hi = _log_uniform(rng, 1, 60_000)
        hi = max(1, min(hi, 4 * MAX_ROTATED // (seqs * heads * dim)))
        rotated = rng.choice([dim // 2 * 2, dim // 2 * 2, 2 * rng.randint(1, dim // 2)])
        case.update(lo=rng.randint(0, hi), hi=hi, new=rng.randint(1, new_hi), new_hi=new_hi, rotated=rotated,
                    interleaved=rng.random() < 0.4, depths=depths)
        return case
    if kind == "tree":
        new = _log_uniform(rng, 2, 64)
        room = min(MAX_CODES // (seqs * heads * dim), MAX_SCORES // (seqs * heads * group * new))
        hi = max(new + 1, _log_uniform(rng, new + 1, max(new + 1, min(60_000, room))))
        case.update(lo=rng.randint(new, hi), hi=hi, new=new, new_hi=new)
        return case
    window, sinks = _log_uniform(rng, 1, 5000), rng.choice([0, 1, 4, rng.randint(2, 130)])
    new = rng.choice([1, 1, rng.randint(2, 8), _log_uniform(rng, 2, 2000)])
    while seqs * heads * group * new * (window + sinks + new) > MAX_SCORES or seqs * heads * dim * (window + sinks + new) > MAX_CODES:
        if new > 16:
            new = new // 2
        elif seqs > 1:
            seqs = seqs // 2
        else:
            window = window // 2
    hi = max(new + 1, _log_uniform(rng, new + 1, max(new + 1, min(60_000, 2 * MAX_CODES // (seqs * heads * dim)))))
    case.update(seqs=seqs, lo=rng.randint(new, hi), hi=hi, new=new, new_hi=new, window=window, sinks=sinks)
    return case


# ---------------------------------------------------------------------- sizes and inputs ----
def _spread(lo, hi, count, phase):
    """`count` whole numbers of [lo, hi], the same for every seed."""
    return [lo + int((hi - lo + 0.999) * ((b * 0.6180339887 + phase) % 1.0)) for b in range(count)]


def _lengths(case):
    """Tokens that each sequence holds before the call (rotate), or in all."""
    return _spread(case["lo"], case["hi"], case["seqs"], 0.37)


def _added(case):
    return _spread(case["new"], case["new_hi"], case["seqs"], 0.81)


def _held(case):
    n = _lengths(case)
    return [a + b for a, b in zip(n, _added(case))] if case["kind"] == "rotate" else n


def _generator(seed, b):
    return torch.Generator("cuda").manual_seed(seed * 4099 + b)


def _features(case, seed):
    """Mean and spread of the features of keys and of values: keys have offsets and a few wide features (rotation turns
    pairs of features of like spread into one another)."""
    g = _generator(seed, 4000)
    f = case["heads"] * case["dim"]
    k_mean = 0.5 * torch.randn(f, device="cuda", generator=g)
    k_std = torch.exp(0.4 * torch.randn(f, device="cuda", generator=g))
    k_std = torch.where(torch.rand(f, device="cuda", generator=g) < 0.03, 6.0 * k_std, k_std)
    v_std = torch.exp(0.3 * torch.randn(f, device="cuda", generator=g))
    return k_mean, k_std, torch.zeros_like(v_std), v_std


def _ranges(case, seed):
    """k, S_b, S_e of keys and of values, as calibrating on earlier text gives them."""
    k_mean, k_std, v_mean, v_std = _features(case, seed)
    w = WIDTH[case["bits"]]
    return [(mean, mean - w * std, mean + w * std) for mean, std in ((k_mean, k_std), (v_mean, v_std))]


def _rows(case, seed, b, n):
    """Keys and values [n, heads, dim] of sequence b, in the case's type."""
    k_mean, k_std, v_mean, v_std = _features(case, seed)
    g = _generator(seed, b)
    shape = (n, case["heads"], case["dim"])
    k = torch.randn(n, k_std.numel(), device="cuda", generator=g).mul_(k_std).add_(k_mean)
    v = torch.randn(n, k_std.numel(), device="cuda", generator=g).mul_(v_std).add_(v_mean)
    return k.to(TYPES[case["type"]]).view(shape), v.to(TYPES[case["type"]]).view(shape)


def _queries(case, seed, *shape):
    """[*shape, heads * group, dim]: scores have a standard deviation of about 2."""
    _, k_std, _, _ = _features(case, seed)
    g = _generator(seed, 4001)
    q = torch.randn(*shape, case["heads"], case["group"], case["dim"], device="cuda", generator=g)
    q = 2.0 * q / k_std.view(case["heads"], 1, case["dim"])
    return q.reshape(*shape, -1, case["dim"]).to(TYPES[case["type"]])


def _page_table(case, seed):
    """Pages of the pool in no order: table int32 [seqs, most pages], -1 where a sequence has none, and their number."""
    counts = [-(-n // case["page"]) for n in _held(case)]
    g = torch.Generator().manual_seed(seed)
    order = torch.randperm(max(1, sum(counts)), generator=g, dtype=torch.int32)
    table = torch.full((case["seqs"], max(1, max(counts))), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    return table.cuda(), max(1, sum(counts))


def _angles(case):
    """cos and sin [positions, rotated / 2] float32, of angles in 64 bits."""
    half = case["rotated"] // 2
    turn = 10_000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    at = torch.arange(max(_held(case)) + 1, device="cuda", dtype=torch.float64)[:, None] * turn
    return torch.cos(at).float(), torch.sin(at).float()


def _parents(case, seed):
    """For each sequence the parent (an earlier number) of every drafted token but the first, which has none."""
    g = torch.Generator().manual_seed(seed + 5)
    at = torch.rand(case["seqs"], case["new_hi"], generator=g)
    return [[-1 if i == 0 else max(0, i - 1 - int(float(at[b, i]) ** 2 * min(i, 6))) for i in range(case["new_hi"])]
            for b in range(case["seqs"])]


def _tree(case, seed):
    """bool [seqs, new, new]: which drafted tokens a drafted token sees, itself and its ancestors."""
    out = torch.zeros(case["seqs"], case["new"], case["new"], dtype=torch.bool)
    for b, parents in enumerate(_parents(case, seed)):
        for i, p in enumerate(parents):
            if p >= 0:
                out[b, i] = out[b, p]
            out[b, i, i] = True
    return out.cuda()


def _positions(case, seed):
    """Of each new row, where it is at its depth in the tree; None where rows stand one behind the other."""
    if not case["depths"]:
        return None
    out = []
    for first, added, parents in zip(_lengths(case), _added(case), _parents(case, seed)):
        depth = []
        for i in range(added):
            depth.append(0 if i == 0 else depth[parents[i]] + 1)
        out += [first + d for d in depth]
    return _ints(out)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _matrix(case, seed):
    """Rows with a few wide features and of different sizes, weights with channels of different sizes, and a bias."""
    g = _generator(seed, 0)
    m, d, n = case["rows"], case["features"], case["channels"]
    wide = torch.where(torch.rand(d, device="cuda", generator=g) < 0.01, 8.0, 1.0)
    x = torch.randn(m, d, device="cuda", generator=g).mul_(wide).mul_(torch.exp(0.5 * torch.randn(m, 1, device="cuda", generator=g)))
    w = torch.randn(n, d, device="cuda", generator=g).mul_(torch.exp(0.3 * torch.randn(n, 1, device="cuda", generator=g)) / math.sqrt(d))
    bias = torch.randn(n, device="cuda", generator=g) if case["bias"] else None
    return x.to(TYPES[case["type"]]), w.to(TYPES[case["type"]]), bias


def prepare(case, seed):
    if case["kind"] == "linear":
        x, w, bias = _matrix(case, seed)
        if own:
            from paper_2110_08919_amd import lpq
            return {"case": case, "x": x, "layer": lpq.Linear8(w, bias)}
        codes, scales = _row_codes(w)
        return {"case": case, "x": x, "weight": codes.t().contiguous(), "scales": scales, "bias": bias}
    state = {"case": case, "lengths": _ints(_held(case))}
    state["table"], pool_pages = _page_table(case, seed)
    ranges = _ranges(case, seed)
    if own:
        from paper_2110_08919_amd import lpq
        f = case["heads"] * case["dim"]
        keys, values = (lpq.Quantizer(f, case["bits"]).set_params(*r) for r in ranges)
        state["cache"] = lpq.KVCache(keys, values, heads=case["heads"], page=case["page"], pages=pool_pages,
                                     packed=case["bits"] == 4)
    else:
        shape = (pool_pages, case["heads"], case["page"], case["dim"])
        state["constants"] = [(k, sb, se, _multiplier(sb, se, case["bits"])) for k, sb, se in ranges]
        state["pools"] = [torch.zeros(shape, dtype=torch.int8, device="cuda") for _ in range(2)]
        state["bounds"] = torch.zeros(pool_pages, case["heads"], 2, case["dim"], dtype=torch.int8, device="cuda")
    fresh = []
    for b, n in enumerate(_held(case)):
        k, v = _rows(case, seed, b, n)
        old = _lengths(case)[b]
        if case["kind"] == "rotate":
            fresh.append((k[old:], v[old:]))
        if old:
            _write(state, k[:old], v[:old], _ints([0]), state["table"][b:b + 1], _ints([0, old]), old)
    if case["kind"] == "rotate":
        state["k"], state["v"] = (torch.cat(t) for t in zip(*fresh))
        state["first"] = _ints(_lengths(case))
        state["starts"] = _starts(_added(case))
        state["cos"], state["sin"] = _angles(case)
        state["positions"] = _positions(case, seed)
        state["q"] = _queries(case, seed, state["k"].shape[0])
    else:
        state["q"] = _queries(case, seed, case["seqs"], case["new"])
        state["tree"] = _tree(case, seed) if case["kind"] == "tree" else None
    return state


def _starts(counts):
    """None where every sequence adds one row, else where the rows of each begin."""
    if all(c == 1 for c in counts):
        return None
    total, at = 0, [0]
    for c in counts:
        total += c
        at.append(total)
    return _ints(at)


def _write(state, k, v, first, table, starts, most):
    if own:
        state["cache"].write(k, v, first, table, starts)
    else:
        _plain_write(state, k, v, first, table, starts, most)


# ------------------------------------------------------------------------- the calls ----
def run(state):
    case = state["case"]
    if case["kind"] == "linear":
        return state["layer"](state["x"]) if own else _plain_linear(state)
    if not own:
        return {"rotate": _plain_rotate, "window": _plain_window, "tree": _plain_tree}[case["kind"]](state)
    cache, table = state["cache"], state["table"]
    if case["kind"] == "rotate":
        q = cache.write_rotated(state["k"], state["v"], state["first"], table, state["cos"], state["sin"], starts=state["starts"],
                                positions=state["positions"], q=state["q"], interleaved=case["interleaved"])
        k, v = cache.read(state["first"], table, state["starts"], state["k"].shape[0], TYPES[case["type"]])
        return q, k, v, cache.bounds
    if case["kind"] == "window":
        return cache.attend(state["q"], state["lengths"], table, window=case["window"], sinks=case["sinks"])
    return cache.attend(state["q"], state["lengths"], table, tree=state["tree"])


# ------------------------------------------------------------------ the plain forms ----
def _multiplier(sb, se, bits):
    return (2.0 ** bits / (se.double() - sb.double())).float()


def _codes(case, x, constants):
    """Equation 1 in float32 on [n, heads, dim] -> int8; a packed code is at most 7."""
    k, sb, se, m = (t.view(case["heads"], case["dim"]) for t in constants)
    half = float(2 ** (case["bits"] - 1))
    x = x.float()
    c = torch.floor((x - k) * m).clamp(-half, half)
    c = torch.where(x < sb, torch.full_like(c, -half), torch.where(x > se, torch.full_like(c, half), c))
    return c.clamp(max=half - 1).to(torch.int8)


def _places(case, first, table, starts, rows):
    """Position, page and row inside it of each of `rows` rows."""
    t = torch.arange(rows, device="cuda", dtype=torch.int32)
    if starts is None:
        seq, pos = t.long(), first.long()
    else:
        seq = torch.bucketize(t, starts[1:].contiguous(), right=True)
        pos = first.long()[seq] + (t - starts[seq])
    return pos, table[seq, pos // case["page"]].long(), pos % case["page"]


def _plain_write(state, k, v, first, table, starts, most):
    case, p = state["case"], state["case"]["page"]
    _, page, row = _places(case, first, table, starts, k.shape[0])
    for x, pool, constants in zip((k, v), state["pools"], state["constants"]):
        pool[page, :, row] = _codes(case, x, constants)
    added = 1 if starts is None else (starts[1:] - starts[:-1]).long()
    end = (first.long() + added)[:, None]
    column = first.long()[:, None] // p + torch.arange((most + p - 2) // p + 1, device="cuda")
    column = torch.minimum(column, (end - 1) // p)
    touched = table.gather(1, column).long()
    codes = state["pools"][0][touched]                                   # [seqs, columns, heads, page, dim]
    inside = (column[..., None] * p + torch.arange(p, device="cuda") < end[..., None])[:, :, None, :, None]
    lo = torch.where(inside, codes, 127).amin(3)
    hi = torch.where(inside, codes, -128).amax(3)
    state["bounds"][touched] = torch.stack([lo, hi], 3)


def _turn(case, x, cos, sin):
    """Rows [n, heads, dim] in float32 with pairs of features turned: (a c - b s, b c + a s)."""
    r, x = case["rotated"], x.float()
    if case["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_rotate(state):
    case = state["case"]
    pos, page, row = _places(case, state["first"], state["table"], state["starts"], state["k"].shape[0])
    at = pos if state["positions"] is None else state["positions"].long()
    cos, sin = state["cos"][at][:, None], state["sin"][at][:, None]
    _plain_write(state, _turn(case, state["k"], cos, sin), state["v"], state["first"], state["table"], state["starts"], case["new_hi"])
    out = [_turn(case, state["q"], cos, sin).to(TYPES[case["type"]])]
    for pool, (k, _, _, m) in zip(state["pools"], state["constants"]):
        k, s = k.view(case["heads"], case["dim"]), (1.0 / m).view(case["heads"], case["dim"])
        out.append(((pool[page, :, row].float() + 0.5) * s + k).to(TYPES[case["type"]]))
    return (*out, state["bounds"])


def _attention(state, at, sees):
    """Positions `at` [seqs, tokens] of the cache, `sees` [seqs, new, tokens] which of them a new token sees."""
    case = state["case"]
    b, h, g, d, new, p = case["seqs"], case["heads"], case["group"], case["dim"], case["new"], case["page"]
    columns = (at // p).clamp(0, state["table"].shape[1] - 1)
    pages, rows = state["table"].long().gather(1, columns).clamp(min=0), at % p
    keys, values = (((pool[pages, :, rows].float() + 0.5) * (1.0 / m).view(h, d) + k.view(h, d)).permute(0, 2, 1, 3).contiguous()
                    for pool, (k, _, _, m) in zip(state["pools"], state["constants"]))       # [seqs, heads, tokens, dim]
    q = state["q"].float().view(b, new, h, g, d).permute(0, 2, 4, 1, 3).reshape(b, h, d, new * g)
    scores = torch.matmul(keys, q).view(b, h, -1, new, g).div_(math.sqrt(d))
    scores.masked_fill_(~sees.transpose(1, 2)[:, None, :, :, None], -math.inf)
    most = scores.amax(2, keepdim=True)
    weights = scores.sub_(torch.where(most == -math.inf, torch.zeros_like(most), most)).exp_()
    total = weights.sum(2)                                                                   # [seqs, heads, new, group]
    weights = weights.view(b, h, -1, new * g).transpose(2, 3).contiguous()
    o = torch.matmul(weights, values).view(b, h, new, g, d)
    o = o / torch.where(total == 0, torch.ones_like(total), total)[..., None]
    return o.permute(0, 2, 1, 3, 4).reshape(b, new, h * g, d).to(TYPES[case["type"]])


def _plain_window(state):
    case = state["case"]
    new, window, sinks = case["new"], case["window"], case["sinks"]
    n = state["lengths"].long()[:, None]
    low = (n - new - window + 1).clamp(min=0)                            # the first position that any window reaches
    tail = low + torch.arange(min(window + new - 1, max(_lengths(case))), device="cuda")
    head = torch.arange(sinks, device="cuda").expand(case["seqs"], -1)
    at = torch.cat([head, tail], 1)
    once = torch.cat([head < low, tail < n], 1)                          # sinks inside a window count once
    me = (n - new + torch.arange(new, device="cuda"))[:, :, None]
    at_ = at[:, None]
    sees = once[:, None] & (at_ <= me) & ((at_ > me - window) | (at_ < sinks))
    return _attention(state, at, sees)


def _plain_tree(state):
    case = state["case"]
    n, new = state["lengths"].long(), case["new"]
    at = torch.arange(max(_lengths(case)), device="cuda").expand(case["seqs"], -1)
    drafted = at - (n - new)[:, None]
    within = (drafted >= 0) & (drafted < new)
    mask = state["tree"].gather(2, drafted.clamp(0, new - 1)[:, None].expand(-1, new, -1))
    return _attention(state, at, (drafted < 0)[:, None] | (within[:, None] & mask))


def _row_codes(x):
    """Codes (as float32) and scales of rows: the largest value of a row becomes 127."""
    x = x.float()
    most = x.abs().amax(1, keepdim=True)
    factor = torch.where(most > 0, torch.full_like(most, 127.0) / most, torch.zeros_like(most))
    return torch.round(x * factor), (most / 127.0)[:, 0]


def _plain_linear(state):
    codes, scales = _row_codes(state["x"])
    y = torch.matmul(codes, state["weight"]) * scales[:, None] * state["scales"]
    return (y if state["bias"] is None else y + state["bias"]).to(state["x"].dtype)


# ------------------------------------------------------------------------- the work ----
def work(case):
    """Inputs read once, outputs and changed state written once."""
    e = SIZE[case["type"]]
    if case["kind"] == "linear":
        m, d, n = case["rows"], case["features"], case["channels"]
        return {"bytes": m * d * e + n * d + 4 * n * (2 if case["bias"] else 1) + m * n * e, "flops": 2 * m * n * d}
    h, d, p, g = case["heads"], case["dim"], case["page"], case["group"]
    code = case["bits"] / 8.0
    if case["kind"] == "rotate":
        rows = sum(_added(case))
        pages = sum((a + n - 1) // p - a // p + 1 for a, n in zip(_lengths(case), _added(case)))
        positions = len(set().union(*(range(a, a + n) for a, n in zip(_lengths(case), _added(case)))))
        return {"bytes": int(2 * rows * h * d * (2 * e + code)) + 2 * rows * h * g * d * e + pages * h * 2 * d + 4 * positions * case["rotated"],
                "flops": 10 * rows * h * d + 3 * rows * h * (1 + g) * case["rotated"]}
    new, tokens, seen = case["new"], 0, 0
    for n in _lengths(case):
        if case["kind"] == "tree":
            tokens += n
            seen += new * (n - new) + new * (new + 1) // 4
        else:
            low = max(0, n - new - case["window"] + 1)
            tokens += n - low + min(case["sinks"], low)
            for i in range(new):
                first = max(0, n - new + i - case["window"] + 1)
                seen += n - new + i + 1 - first + min(case["sinks"], first)
    return {"bytes": int(2 * tokens * h * d * code) + 2 * case["seqs"] * new * h * g * d * e, "flops": 4 * seen * h * g * d}


# ------------------------------------------------------------------ the same in 64 bits ----
def _exact_constants(case, seed):
    out = []
    for k, sb, se in _ranges(case, seed):
        m = ((2 ** case["bits"]) / (se.double() - sb.double())).float()
        out.append({"k": k, "sb": sb, "se": se, "m": m, "s": (1.0 / m.double()).float()})
    return out


def _exact_codes(case, x, c):
    """Equation 1 as it is defined: two operations, each rounded to binary32; result in float64."""
    flat = x.reshape(x.shape[0], -1).float()
    bottom, top = -(2.0 ** (case["bits"] - 1)), 2.0 ** (case["bits"] - 1) - 1.0
    t = ((flat.double() - c["k"].double()).float().double() * c["m"].double()).float()
    code = torch.floor(t.double())
    code[flat < c["sb"]] = bottom
    code[flat > c["se"]] = top
    return code.clamp_(bottom, top).view(x.shape)


def _exact_values(case, code, c):
    """(c + 1/2) s + k of the definition, in 64 bits."""
    s, k = (c[n].double().view(case["heads"], case["dim"]) for n in ("s", "k"))
    return (code + 0.5) * s + k


def _exact_turn(case, x, at, rounded):
    """Rows turned, in 64 bits; `rounded`: as keys are, products and sums rounded to binary32 before they are encoded."""
    half = case["rotated"] // 2
    first = torch.arange(half, device="cuda") * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else half)
    cos, sin = (t[at.long()].double()[:, None] for t in _angles(case))
    r = (lambda t: t.float().double()) if rounded else (lambda t: t)
    a, b = x[..., first].double(), x[..., second].double()
    out = x.double()
    out[..., first] = r(r(a * cos) - r(b * sin))
    out[..., second] = r(r(b * cos) + r(a * sin))
    return out


def exact(case, seed):
    if case["kind"] == "linear":
        return _exact_linear(case, seed)
    keys, values = _exact_constants(case, seed)
    if case["kind"] == "rotate":
        return _exact_rotate(case, seed, keys, values)
    h, d, g, new = case["heads"], case["dim"], case["group"], case["new"]
    q = _queries(case, seed, case["seqs"], new).double()
    tree = _tree(case, seed) if case["kind"] == "tree" else None
    out = torch.zeros(case["seqs"], new, h * g, d, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(case)):
        k, v = _rows(case, seed, b, n)
        sees = torch.zeros(new, n, dtype=torch.bool, device="cuda")
        for i in range(new):
            me = n - new + i
            if tree is None:
                sees[i, max(0, me - case["window"] + 1):me + 1] = True
                sees[i, :min(case["sinks"], me + 1)] = True
            else:
                sees[i, :n - new] = True
                sees[i, n - new:] = tree[b, i]
        some = sees.any(0).nonzero()[:, 0]
        sees = sees[:, some]
        k = _exact_values(case, _exact_codes(case, k[some], keys), keys)
        v = _exact_values(case, _exact_codes(case, v[some], values), values)
        for head in range(h * g):
            scores = (q[b, :, head] @ k[:, head // g].t().contiguous()) / math.sqrt(d)
            scores[~sees] = -math.inf
            weights = torch.nan_to_num(torch.softmax(scores, 1))        # a row that sees nothing
            out[b, :, head] = weights @ v[:, head // g].contiguous()
    return out


def _exact_rotate(case, seed, keys, values):
    rows_k, rows_v, at = [], [], []
    table, pool_pages = _page_table(case, seed)
    table = table.cpu()
    bounds = torch.zeros(pool_pages, case["heads"], 2, case["dim"], dtype=torch.int8, device="cuda")
    given = _positions(case, seed)
    taken = 0
    for b, (old, n) in enumerate(zip(_lengths(case), _held(case))):
        k, v = _rows(case, seed, b, n)
        here = torch.arange(old, n, device="cuda") if given is None else given[taken:taken + n - old]
        taken += n - old
        codes = _exact_codes(case, torch.cat([k[:old].double(), _exact_turn(case, k[old:], here, True)]), keys)
        for column, part in enumerate(codes.split(case["page"])):
            bounds[int(table[b, column])] = torch.stack([part.min(0).values, part.max(0).values], 1).to(torch.int8)
        rows_k.append(_exact_values(case, codes[old:], keys))
        rows_v.append(_exact_values(case, _exact_codes(case, v[old:], values), values))
        at.append(here)
    at = torch.cat(at)
    q = _exact_turn(case, _queries(case, seed, at.shape[0]), at, False)
    return q, torch.cat(rows_k), torch.cat(rows_v), bounds


def _exact_linear(case, seed):
    x, w, bias = _matrix(case, seed)
    parts = []
    for t in (x, w):
        t = t.float()
        most = t.abs().max(1).values.double()
        factor = torch.where(most > 0, 127.0 / most, 0.0).float().double()
        parts.append((torch.round((t.double() * factor[:, None]).float().double()), (most / 127.0).float().double()))
    (a, sa), (b, sb) = parts
    y = (a @ b.t().contiguous()) * sa[:, None] * sb
    return y if bias is None else y + bias.double()
