"""A small decoder that generates text tokens from a quantised key-value cache: an example of KVCache in use.

    python -m paper_2110_08919_amd.decode [--prompt 4000 --steps 32 --pages 16 ...]

A stack of attention layers with random weights reads prompts of different lengths with ordinary attention, learns each
layer's quantizers from the prompt's keys and values (Section 3.2 of the paper, mean +- 4 sigma per feature), writes
them into the layer's cache and generates tokens: per token and layer one write, one selection of pages and one
attention over them (or, with --pages 0, over all).  Beside the tokens per second it prints how far the
cache's attention is from attention over the unquantised keys and values, and from it over all pages.

With --codes the projections are 8-bit codes as well (a scale for each row and channel), with --rotate queries and keys are turned by their
positions' angles on the way into the cache, and --window N has a token see the last N positions and the first 4.  Pages are not selected then: they are
ranked over a whole conversation, and the window would mask most of those picked.
"""
from __future__ import annotations

import argparse
import time
from dataclasses import dataclass

import torch

from . import lpq


@dataclass
class Shape:
    layers: int = 4
    width: int = 1024
    heads: int = 16        # query heads
    kv_heads: int = 4
    dim: int = 128         # features of a head
    vocabulary: int = 8000
    page: int = 64
    rotate: bool = False   # queries and keys are turned by their positions' angles
    window: int = 0        # positions that a token sees up to its own, 0: all
    sinks: int = 4         # with a window: first positions that it sees as well


def angles(positions: int, dim: int):
    """cos and sin [positions, dim / 2] float32, of angles in 64 bits."""
    turn = 10_000.0 ** (-torch.arange(dim // 2, device="cuda", dtype=torch.float64) / (dim // 2))
    at = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * turn
    return torch.cos(at).float(), torch.sin(at).float()


def turned(x: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor):
    """Rows x [n, heads, dim] at positions 0 on, features paired with those half a head further."""
    a, b = x.float().chunk(2, -1)
    c, s = cos[:len(x), None], sin[:len(x), None]
    return torch.cat([a * c - b * s, b * c + a * s], -1).to(x.dtype)


class Layer:
    """Projections, and the layer's cache once the prompt is known."""

    def __init__(self, shape: Shape, g: torch.Generator, dtype, codes: bool = False):
        def weight(*size):
            w = (torch.randn(*size, device="cuda", generator=g) / size[0] ** 0.5).to(dtype)
            return lpq.Linear8(w.t().contiguous()) if codes else w
        self.shape = shape
        self.wq = weight(shape.width, shape.heads * shape.dim)
        self.wkv = weight(shape.width, 2 * shape.kv_heads * shape.dim)
        self.wo = weight(shape.heads * shape.dim, shape.width)
        self.cache = None

    @staticmethod
    def times(x: torch.Tensor, w):
        return w(x) if isinstance(w, lpq.Linear8) else x @ w

    def project(self, x: torch.Tensor):
        """Queries, keys and values of rows x [n, width]."""
        s = self.shape
        q = self.times(x, self.wq).view(-1, s.heads, s.dim)
        k, v = self.times(x, self.wkv).view(-1, 2, s.kv_heads, s.dim).unbind(1)
        return q, k, v

    def out(self, o: torch.Tensor):
        return self.times(o, self.wo)

    def make_cache(self, k: torch.Tensor, v: torch.Tensor, pages: int, packed: bool):
        """Quantizers from the prompts' keys and values [n, kv_heads, dim], and an empty cache."""
        f = self.shape.kv_heads * self.shape.dim
        quantizers = [lpq.Quantizer(f, 4 if packed else 8).calibrate(t.reshape(-1, f).float(), "gauss", "per_feature", 2.5 if packed else 4.0)
                      for t in (k, v)]
        self.cache = lpq.KVCache(*quantizers, heads=self.shape.kv_heads, page=self.shape.page, pages=pages, packed=packed)


def causal_attention(q, k, v, window=0, sinks=0):
    """q [n, heads, dim], k / v [n, kv_heads, dim] of one prompt, in float32; window 0: none."""
    n, heads, dim = q.shape
    group = heads // k.shape[1]
    out = torch.empty_like(q)
    keep = torch.ones(n, n, dtype=torch.bool, device=q.device).tril()
    if window:
        keep &= torch.ones_like(keep).triu(1 - window) | (torch.arange(n, device=q.device) < sinks)
    for h in range(heads):
        scores = q[:, h].float() @ k[:, h // group].float().t().contiguous() / dim ** 0.5
        out[:, h] = (torch.softmax(scores.masked_fill(~keep, -float("inf")), 1) @ v[:, h // group].float()).to(q.dtype)
    return out


class Decoder:
    def __init__(self, shape: Shape, prompts, steps: int, packed: bool = False, dtype=torch.bfloat16, seed: int = 0,
                 codes: bool = False):
        g = torch.Generator("cuda").manual_seed(seed)
        self.shape, self.dtype = shape, dtype
        self.embedding = torch.randn(shape.vocabulary, shape.width, device="cuda", generator=g).to(dtype)
        self.layers = [Layer(shape, g, dtype, codes) for _ in range(shape.layers)]
        lengths = [len(p) for p in prompts]
        counts = [-(-(n + steps) // shape.page) for n in lengths]
        table = torch.full((len(prompts), max(counts)), -1, dtype=torch.int32)
        at = 0
        for b, c in enumerate(counts):
            table[b, :c] = torch.arange(at, at + c)
            at += c
        self.table, self.lengths = table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")
        starts = torch.tensor([0] + lengths, dtype=torch.int32).cumsum(0).int().cuda()
        first = torch.zeros_like(self.lengths)
        xs = [self.embedding[torch.as_tensor(p, device="cuda")] for p in prompts]
        self.seen = dict(window=shape.window, sinks=shape.sinks) if shape.window else {}
        self.angles = angles(max(lengths) + steps, shape.dim) if shape.rotate else None
        self.kept = []                                   # unquantised keys and values of each layer and prompt, to compare with
        for layer in self.layers:
            rows = [layer.project(self._norm(x)) for x in xs]
            k, v = (torch.cat([r[i] for r in rows]) for i in (1, 2))
            layer.make_cache(torch.cat([turned(r[1], *self.angles) for r in rows]) if shape.rotate else k, v, at, packed)
            if shape.rotate:
                layer.cache.write_rotated(k, v, first, self.table, *self.angles, starts=starts)
                rows = [(turned(r[0], *self.angles), turned(r[1], *self.angles), r[2]) for r in rows]
            else:
                layer.cache.write(k, v, first, self.table, starts)
            self.kept.append([[r[1], r[2]] for r in rows])
            xs = [x + layer.out(causal_attention(*r, **self.seen).flatten(1)) for x, r in zip(xs, rows)]
        self.tokens = self._next(torch.stack([x[-1] for x in xs]))

    @staticmethod
    def _norm(x):
        return (x.float() * torch.rsqrt(x.float().pow(2).mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def _next(self, x):
        return (self._norm(x) @ self.embedding.t().contiguous()).argmax(-1)

    def step(self, pages: int, watch=None):
        """One token for every conversation; pages > 0: attention over that many selected pages of each head (without a window only)."""
        assert not (pages and self.shape.window), "pages are ranked over all tokens: with a window, select none"
        if watch is None:
            self.kept = None                             # this step's keys and values are not kept
        x = self.embedding[self.tokens]
        first = self.lengths.clone()
        self.lengths += 1
        for i, layer in enumerate(self.layers):
            q, k, v = layer.project(self._norm(x))
            if self.angles:
                q = layer.cache.write_rotated(k, v, first, self.table, *self.angles, q=q)
                if watch is not None:
                    k = torch.cat([turned(t[None], *(a[n:n + 1] for a in self.angles)) for t, n in zip(k, first.tolist())])
            else:
                layer.cache.write(k, v, first, self.table)
            q = q.unsqueeze(1)
            chosen = layer.cache.select(q, self.lengths, self.table, pages, keep_first=1, keep_last=1) if pages else None
            o = layer.cache.attend(q, self.lengths, self.table, pages=chosen, **self.seen)
            if watch is not None:
                watch(i, q, k, v, o)
            x = x + layer.out(o.flatten(1))
        self.tokens = self._next(x)
        return self.tokens

    def errors(self, pages: int):
        """One step, with the relative error of each layer's attention against attention over the unquantised keys and
        values of all tokens that it sees: [layers] (root mean square over conversations, heads and features).  Before any step() only."""
        assert self.kept is not None, "the keys and values of an earlier step were not kept"
        out = []

        def watch(i, q, k, v, o):
            want = []
            for b, (ks, vs) in enumerate(self.kept[i]):
                ks, vs = torch.cat([ks, k[b:b + 1]]), torch.cat([vs, v[b:b + 1]])
                self.kept[i][b] = [ks, vs]
                group = q.shape[2] // ks.shape[1]
                scores = (ks.float().permute(1, 0, 2) @ q[b, 0].float().view(ks.shape[1], group, -1).transpose(1, 2).contiguous())
                if self.seen:
                    at = torch.arange(len(ks), device=ks.device)
                    scores[:, (at <= len(ks) - 1 - self.shape.window) & (at >= self.shape.sinks)] = -float("inf")
                w = torch.softmax(scores / q.shape[-1] ** 0.5, 1).transpose(1, 2).contiguous()
                want.append((w @ vs.float().permute(1, 0, 2).contiguous()).flatten(0, 1))
            want = torch.stack(want)
            out.append(((o[:, 0].float() - want).pow(2).mean().sqrt() / want.pow(2).mean().sqrt()).item())
        self.step(pages, watch)
        return out


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--prompt", type=int, default=4000, help="tokens of the longest prompt")
    parser.add_argument("--conversations", type=int, default=4)
    parser.add_argument("--steps", type=int, default=32)
    parser.add_argument("--pages", type=int, default=None, help="pages a head looks at per token, 16 by default (none with a window); 0: all")
    parser.add_argument("--packed", action="store_true", help="4-bit codes, two per byte")
    parser.add_argument("--layers", type=int, default=4)
    parser.add_argument("--codes", action="store_true", help="projections on 8-bit codes")
    parser.add_argument("--rotate", action="store_true", help="queries and keys turned by their positions' angles")
    parser.add_argument("--window", type=int, default=0, help="positions a token sees up to its own, and the first 4; 0: all")
    a = parser.parse_args(argv)
    if a.pages and a.window:
        parser.error("--pages with --window: pages are ranked over all tokens, not those of the window")
    if a.pages is None:
        a.pages = 0 if a.window else 16
    shape = Shape(layers=a.layers, rotate=a.rotate, window=a.window)
    g = torch.Generator().manual_seed(1)
    lengths = [max(1, a.prompt * (b + 1) // a.conversations) for b in range(a.conversations)]
    prompts = [torch.randint(shape.vocabulary, (n,), generator=g).tolist() for n in lengths]
    d = Decoder(shape, prompts, a.steps + 4, packed=a.packed, codes=a.codes)
    result = {"all_pages": d.errors(0)}
    if a.pages:
        result["selected_pages"] = d.errors(a.pages)
    d.step(a.pages)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        d.step(a.pages)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    codes = sum(2 * layer.cache.k.numel() for layer in d.layers)
    print(f"{a.conversations} conversations of {lengths} tokens, {shape.layers} layers of {shape.kv_heads} x {shape.dim} keys, "
          f"{codes / 1e6:.1f} MB of codes ({'4' if a.packed else '8'} bits)")
    for what, e in result.items():
        print(f"attention over {what.replace('_', ' ')}: relative error per layer " + " ".join(f"{x:.4f}" for x in e))
    print(f"{a.steps} steps: {t / a.steps * 1e3:.3f} ms per step, {a.steps * a.conversations / t:.0f} tokens/s")
    return result


if __name__ == "__main__":
    main()
