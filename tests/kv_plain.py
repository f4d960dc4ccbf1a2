"""The key-value cache's definitions in plain numpy (64 bits; Equation 1 as two operations rounded to
binary32), for the tests of the HIP kernels."""
import numpy as np


class Constants:
    """k, S_b, S_e and what follows from them, float32 [heads, dim]."""

    def __init__(self, k, sb, se, bits, heads):
        shape = (heads, -1)
        self.k, self.sb, self.se = (np.asarray(a, np.float32).reshape(shape) for a in (k, sb, se))
        self.bits = bits
        width = self.se.astype(np.float64) - self.sb.astype(np.float64)
        with np.errstate(divide="ignore"):
            self.m = np.where(width > 0, 2.0 ** bits / width, 0.0).astype(np.float32)
            self.s = np.where(self.m > 0, np.float32(1) / self.m, np.float32(0)).astype(np.float32)


def codes(x, c, packed):
    """x [n, heads, dim] (any float type) -> int codes [n, heads, dim]."""
    x = np.asarray(x, np.float32)
    half = 2 ** (c.bits - 1)
    top = min(half, 7 if packed else 127)
    with np.errstate(invalid="ignore", over="ignore"):
        t = ((x - c.k).astype(np.float32) * c.m).astype(np.float32)
        q = np.clip(np.floor(t), -half, top)
        q = np.where(x > c.se, top, np.where(x < c.sb, -half, q))
    return np.where(np.isnan(t) | (c.m == 0), 0, q).astype(np.int64)


def values(q, c):
    """What codes [..., heads, dim] read back as, in binary32 as defined."""
    return (((q.astype(np.float32) + np.float32(0.5)) * c.s).astype(np.float32) + c.k).astype(np.float32)


def bounds(q, page):
    """[pages, heads, 2, dim] of codes [n, heads, dim]."""
    return np.stack([np.stack([p.min(0), p.max(0)], 1) for p in (q[i:i + page] for i in range(0, len(q), page))])


def select(q, kcodes, c, page, n_select, keep_first, keep_last, group, there=None):
    """q [new, q_heads, dim] float32, kcodes [n, heads, dim] -> list per head of ascending page numbers."""
    new, q_heads, dim = q.shape
    heads = q_heads // group
    n = len(kcodes)
    have = -(-n // page)
    there = np.ones(have, bool) if there is None else there
    out = []
    if have:
        b = bounds(kcodes, page)
    for h in range(heads):
        with np.errstate(over="ignore", invalid="ignore"):
            scaled = (q[:, h * group:(h + 1) * group].reshape(-1, dim).astype(np.float32) * c.s[h]).astype(np.float32)
        scaled[~np.isfinite(scaled)] = 0
        most = np.float32(np.abs(scaled).max())
        f = np.float32(127) / most if most > np.float32(1e-30) else np.float32(0)
        z = np.rint((scaled * f).astype(np.float32)).astype(np.int64)
        up, down = np.maximum(z, 0).sum(0), np.minimum(z, 0).sum(0)
        score = [int((up * b[p, h, 1] + down * b[p, h, 0]).sum()) for p in range(have)]
        kept = [p < keep_first or p >= have - keep_last for p in range(have)]
        ranked = sorted((p for p in range(have) if there[p]), key=lambda p: (not kept[p], 0 if kept[p] else -score[p], p))
        out.append(sorted(ranked[:n_select]))
    return out


def attend(q, kx, vx, group, scale, seen=None, dead=None):
    """q [new, q_heads, dim], kx / vx float64 [n, heads, dim] as they read back -> o, lse in float64.
    seen: positions per head (list of arrays) or None for all; dead: positions that do not exist."""
    new, q_heads, dim = q.shape
    n = len(kx)
    o, lse = np.zeros((new, q_heads, dim)), np.full((new, q_heads), -np.inf)
    for i in range(new):
        for j in range(q_heads):
            h = j // group
            at = np.arange(n) if seen is None else np.asarray(seen[h], np.int64)
            at = at[at <= n - new + i]
            if dead is not None:
                at = at[~dead[at]]
            if len(at) == 0:
                continue
            t = scale * (kx[at, h] @ q[i, j].astype(np.float64))
            p = np.exp(t - t.max())
            o[i, j] = (p[:, None] * vx[at, h]).sum(0) / p.sum()
            lse[i, j] = t.max() + np.log(p.sum())
    return o, lse


UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}      # largest relative rounding error of a type


def attend_bound(q, kcodes, vx, kc, group, scale, kind):
    """Largest error of attention of one sequence: per output [new, q_heads, dim], and of its lse.

    A query row is held as integers of A / Qmax, so a score is off by at most e = scale * A / (2 Qmax) * max_j sum_i |c_ji|
    (plus float32 roundings of it, 6 of 2^-24); a weight by exp(e), its rounding (2^-11, or 2^-22 in two terms) and 2^-22
    of exp2 and the maximum; weights below 2^-31 of the largest may vanish.  Weights off by a factor within 1 +- w move a mean
    by at most 2 w times the spread of what is averaged.  Sums of n terms in float32 add n / 16 + 40 roundings (a matrix
    instruction sums 32 products, then one addition per tile and part).  At the end one rounding to the type."""
    new, q_heads, dim = q.shape
    n = len(kcodes)
    qmax, pround = (2088895, 2.0 ** -22) if kind == "f32" else (16319, 2.0 ** -11)
    err, lerr = np.zeros((new, q_heads, dim)), np.zeros((new, q_heads))
    if n == 0:
        return err, lerr
    for j in range(q_heads):
        h = j // group
        scaled = np.abs(q[:, j].astype(np.float64) * kc.s[h])
        total = np.abs(kcodes[:, h]).sum(1).max()
        e = abs(scale) * scaled.max(1) / (2 * qmax) * total                                     # [new]
        t = abs(scale) * (np.abs(kcodes[:, h]) @ scaled.T).max(0)                               # largest score, [new]
        e = e + 6 * 2.0 ** -24 * t + 2.0 ** -22
        w = np.expm1(e) + pround + n * 2.0 ** -31
        spread = vx[:, h].max(0) - vx[:, h].min(0)
        size = np.abs(vx[:, h]).max(0)
        err[:, j] = 2 * w[:, None] * spread + (n / 16 + 40) * 2.0 ** -24 * (size + spread) + UNIT[kind] * size
        lerr[:, j] = w + (n / 16 + 40) * 2.0 ** -24 + 8 * 2.0 ** -24 * (t + 30 + abs(scale) * (np.abs(q[:, j]) @ np.abs(kc.k[h])))
    return err, lerr
