"""A small decoder that generates text tokens from a quantised key-value cache: an example of KVCache in use.

    python -m paper_2110_08919_amd.decode [--prompt 4000 --steps 32 --pages 16 ...]

A stack of attention layers with random weights reads prompts of different lengths with ordinary attention, learns each
layer's quantizers from the prompt's keys and values (Section 3.2 of the paper, mean +- 4 sigma per feature), writes
them into the layer's cache and generates tokens: per token and layer one write, one selection of pages and one
attention over them (or, with --pages 0, over all).  Beside the tokens per second it prints how far the
cache's attention is from attention over the unquantised keys and values, and from it over all pages.
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


class Layer:
    """Projections, and the layer's cache once the prompt is known."""

    def __init__(self, shape: Shape, g: torch.Generator, dtype):
        def weight(*size):
            return (torch.randn(*size, device="cuda", generator=g) / size[0] ** 0.5).to(dtype)
        self.shape = shape
        self.wq = weight(shape.width, shape.heads * shape.dim)
        self.wkv = weight(shape.width, 2 * shape.kv_heads * shape.dim)
        self.wo = weight(shape.heads * shape.dim, shape.width)
        self.cache = None

    def project(self, x: torch.Tensor):
        """Queries, keys and values of rows x [n, width]."""
        s = self.shape
        q = (x @ self.wq).view(-1, s.heads, s.dim)
        k, v = (x @ self.wkv).view(-1, 2, s.kv_heads, s.dim).unbind(1)
        return q, k, v

    def make_cache(self, k: torch.Tensor, v: torch.Tensor, pages: int, packed: bool):
        """Quantizers from the prompts' keys and values [n, kv_heads, dim], and an empty cache."""
        f = self.shape.kv_heads * self.shape.dim
        quantizers = [lpq.Quantizer(f, 4 if packed else 8).calibrate(t.reshape(-1, f).float(), "gauss", "per_feature", 2.5 if packed else 4.0)
                      for t in (k, v)]
        self.cache = lpq.KVCache(*quantizers, heads=self.shape.kv_heads, page=self.shape.page, pages=pages, packed=packed)


def causal_attention(q, k, v):
    """q [n, heads, dim], k / v [n, kv_heads, dim] of one prompt, in float32."""
    n, heads, dim = q.shape
    group = heads // k.shape[1]
    out = torch.empty_like(q)
    keep = torch.ones(n, n, dtype=torch.bool, device=q.device).tril()
    for h in range(heads):
        scores = q[:, h].float() @ k[:, h // group].float().t().contiguous() / dim ** 0.5
        out[:, h] = (torch.softmax(scores.masked_fill(~keep, -float("inf")), 1) @ v[:, h // group].float()).to(q.dtype)
    return out


class Decoder:
    def __init__(self, shape: Shape, prompts, steps: int, packed: bool = False, dtype=torch.bfloat16, seed: int = 0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.shape, self.dtype = shape, dtype
        self.embedding = torch.randn(shape.vocabulary, shape.width, device="cuda", generator=g).to(dtype)
        self.layers = [Layer(shape, g, dtype) for _ in range(shape.layers)]
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
        self.kept = []                                   # unquantised keys and values of each layer and prompt, to compare with
        for layer in self.layers:
            rows = [layer.project(self._norm(x)) for x in xs]
            k, v = (torch.cat([r[i] for r in rows]) for i in (1, 2))
            layer.make_cache(k, v, at, packed)
            layer.cache.write(k, v, first, self.table, starts)
            self.kept.append([[r[1], r[2]] for r in rows])
            xs = [x + causal_attention(*r).flatten(1) @ layer.wo for x, r in zip(xs, rows)]
        self.tokens = self._next(torch.stack([x[-1] for x in xs]))

    @staticmethod
    def _norm(x):
        return (x.float() * torch.rsqrt(x.float().pow(2).mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def _next(self, x):
        return (self._norm(x) @ self.embedding.t().contiguous()).argmax(-1)

    def step(self, pages: int, watch=None):
        """One token for every conversation; pages > 0: attention over that many selected pages of each head."""
        if watch is None:
            self.kept = None                             # this step's keys and values are not kept
        x = self.embedding[self.tokens]
        first = self.lengths.clone()
        self.lengths += 1
        for i, layer in enumerate(self.layers):
            q, k, v = layer.project(self._norm(x))
            layer.cache.write(k, v, first, self.table)
            q = q.unsqueeze(1)
            chosen = layer.cache.select(q, self.lengths, self.table, pages, keep_first=1, keep_last=1) if pages else None
            o = layer.cache.attend(q, self.lengths, self.table, pages=chosen)
            if watch is not None:
                watch(i, q, k, v, o)
            x = x + o.flatten(1) @ layer.wo
        self.tokens = self._next(x)
        return self.tokens

    def errors(self, pages: int):
        """One step, with the relative error of each layer's attention against attention over the unquantised keys and
        values of all tokens: [layers] (root mean square over conversations, heads and features).  Before any step() only."""
        assert self.kept is not None, "the keys and values of an earlier step were not kept"
        out = []

        def watch(i, q, k, v, o):
            want = []
            for b, (ks, vs) in enumerate(self.kept[i]):
                ks, vs = torch.cat([ks, k[b:b + 1]]), torch.cat([vs, v[b:b + 1]])
                self.kept[i][b] = [ks, vs]
                group = q.shape[2] // ks.shape[1]
                scores = (ks.float().permute(1, 0, 2) @ q[b, 0].float().view(ks.shape[1], group, -1).transpose(1, 2).contiguous())
                w = torch.softmax(scores / q.shape[-1] ** 0.5, 1).transpose(1, 2).contiguous()
                want.append((w @ vs.float().permute(1, 0, 2).contiguous()).flatten(0, 1))
            want = torch.stack(want)
            out.append(((o[:, 0].float() - want).pow(2).mean().sqrt() / want.pow(2).mean().sqrt()).item())
        self.step(pages, watch)
        return out


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--prompt", type=int, default=4000, help="tokens of the longest prompt")
    a.add_argument("--conversations", type=int, default=4)
    a.add_argument("--steps", type=int, default=32)
    a.add_argument("--pages", type=int, default=16, help="pages a head looks at per token; 0: all")
    a.add_argument("--packed", action="store_true", help="4-bit codes, two per byte")
    a.add_argument("--layers", type=int, default=4)
    a = a.parse_args(argv)
    shape = Shape(layers=a.layers)
    g = torch.Generator().manual_seed(1)
    lengths = [max(1, a.prompt * (b + 1) // a.conversations) for b in range(a.conversations)]
    prompts = [torch.randint(shape.vocabulary, (n,), generator=g).tolist() for n in lengths]
    d = Decoder(shape, prompts, a.steps + 4, packed=a.packed)
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
