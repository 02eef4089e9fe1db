"""Decoding on the kept tokens of pruned scenes, as a language model's layer does.

    python -m paper_2608_13226_gb300.decode_kept [--scenes 8] [--keep 0.15] [--steps 64]
                                                 [--cache bf16|e4m3] [--heads 28] [--kv-heads 4]

Long-video scenes are pruned (coverprune_lite_select), the kept features gathered
and projected, and their keys appended to a paged cache, rotated at the kept
tokens' own indices in the scene (coverprune_cache_append).  Every further token
is then one projection, one append with its query's rotation and one attention
over the cache (coverprune_decode_attention).  Weights are random: what is shown is the
path and what pruning saves, the cache's size and the attention's time beside
those of the unpruned scenes.
"""
from __future__ import annotations

import argparse
import math
from dataclasses import dataclass

import torch

import paper_2608_13226_gb300 as cp
from paper_2608_13226_gb300 import scenes

PAGE = 16


@dataclass
class Layer:
    """Projections of one attention layer, and the speeds of its rotation."""
    heads: int
    kv_heads: int
    width: int
    qkv: torch.Tensor   # [D, (heads + 2 kv_heads) width]
    out: torch.Tensor   # [heads width, D]
    freq: torch.Tensor

    def project(self, x):
        """Queries, keys and values [rows, heads, width] of rows x [rows, D], views of one product."""
        y = (x @ self.qkv).view(x.shape[0], self.heads + 2 * self.kv_heads, self.width)
        return y[:, :self.heads], y[:, self.heads:-self.kv_heads], y[:, -self.kv_heads:]


def make_layer(D, heads, kv_heads, width=128, seed=0, context=1.0):
    """Random weights; context > 1 stretches the rotation to contexts so many times longer."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def weight(a, b):
        return (torch.randn(a, b, generator=g, device="cuda") / math.sqrt(a)).bfloat16()

    freq = cp.coverprune_rotary_frequencies(width, 1e6, stretch="turns" if context > 1 else "none",
                                            factor=context, original=32768.0)
    return Layer(heads, kv_heads, width, weight(D, (heads + 2 * kv_heads) * width),
                 weight(heads * width, D), freq)


class Cache:
    """A paged cache of one layer, with room for `keys` of each sequence."""

    def __init__(self, layer: Layer, sequences: int, keys: int, dtype=torch.bfloat16, scale=0.05):
        width = -(-keys // PAGE)
        shape = (sequences * width, PAGE, layer.kv_heads, layer.width)
        raw = torch.uint8 if dtype == torch.float8_e4m3fn else dtype
        self.k, self.v = (torch.zeros(shape, dtype=raw, device="cuda").view(dtype) for _ in "kv")
        self.table = torch.randperm(sequences * width, device="cuda").int().view(sequences, width)
        self.lens = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        # an 8-bit element stands for scale times its value
        self.scale = torch.full((layer.kv_heads,), scale, device="cuda") if raw == torch.uint8 else None
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws = None

    @property
    def bytes(self):
        return 2 * self.k.numel() * self.k.element_size()

    def append(self, layer, q, k, v, starts=None, pos=None):
        """Keys and values into the cache; the turned queries."""
        r = cp.coverprune_cache_append(k, v, self.k, self.v, self.table, self.lens, starts=starts, pos=pos,
                                       inv_freq=layer.freq, q=q, k_scale=self.scale, v_scale=self.scale,
                                       status=self.status)
        self.lens = r["lens"]
        return r["q"]

    def attend(self, q):
        r = cp.coverprune_decode_attention(q, self.k, self.v, self.table, self.lens, k_scale=self.scale,
                                           v_scale=self.scale, ws=self.ws, status=self.status)
        self.ws = r["ws"]
        return r["out"]


def fill(layer, cache, feats, pos):
    """The prompt: feats [B, K, D] of tokens at pos int64 [B, K]."""
    B, K, _ = feats.shape
    q, k, v = layer.project(feats.reshape(B * K, -1))
    starts = torch.arange(0, B * K + 1, K, dtype=torch.int32, device="cuda")
    cache.append(layer, None, k, v, starts=starts, pos=pos.reshape(-1))


def step(layer, cache, x, pos):
    """One new token a sequence: x [B, D] at pos int64 [B]; the layer's output [B, D]."""
    q, k, v = layer.project(x)
    q = cache.append(layer, q, k, v, pos=pos)
    return cache.attend(q).flatten(1) @ layer.out


def decode(layer, cache, x, pos, steps):
    """`steps` tokens, each the normalised output of the one before; the last one's output."""
    for i in range(steps):
        x = step(layer, cache, x, pos + i)
        x = x / x.float().norm(dim=1, keepdim=True).bfloat16()
    return x


def _ms(f, n):
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    a.record()
    f(n)
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) / n


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--scenes", type=int, default=8)
    p.add_argument("--keep", type=float, default=0.15)
    p.add_argument("--steps", type=int, default=64)
    p.add_argument("--cache", choices=("bf16", "e4m3"), default="bf16")
    p.add_argument("--heads", type=int, default=28)
    p.add_argument("--kv-heads", type=int, default=4)
    a = p.parse_args(argv)
    made = [scenes.make_scene(scenes.CONFIGS["long_video"], i) for i in range(a.scenes)]
    feats = torch.stack([torch.from_numpy(s["feats"]).bfloat16() for s in made]).cuda()
    pos = torch.stack([torch.from_numpy(s["pos"]) for s in made]).cuda()
    frame = torch.stack([torch.from_numpy(s["frame"]) for s in made]).cuda()
    B, N, D = feats.shape
    K = cp.coverprune_budget(a.keep, N)
    kept = cp.coverprune_lite_select(feats, pos, frame, K)["kept"]
    rows = cp.coverprune_gather(feats, pos, frame, kept)[0]
    layer = make_layer(D, a.heads, a.kv_heads)
    dtype = torch.bfloat16 if a.cache == "bf16" else torch.float8_e4m3fn
    every = torch.arange(N, device="cuda").expand(B, N).contiguous()
    x = feats[:, 0] / feats[:, 0].float().norm(dim=1, keepdim=True).bfloat16()
    at = torch.full((B,), N, device="cuda")
    for name, f, where in (("kept", rows, kept), ("all", feats, every)):
        cache = Cache(layer, B, f.shape[1] + 2 * a.steps, dtype)
        fill(layer, cache, f, where)
        decode(layer, cache, x, at, a.steps)  # the first pass of everything
        ms = _ms(lambda n: decode(layer, cache, x, at, n), a.steps)
        q = torch.randn(B, a.heads, layer.width, device="cuda").bfloat16()
        att = _ms(lambda n: [cache.attend(q) for _ in range(n)], 200)
        assert int(cache.status) == 0
        print(f"{name:5s} {f.shape[1]:6d} tokens a scene  cache {cache.bytes / 1e6:8.1f} MB  "
              f"attention {1e3 * att:7.1f} us  layer {1e3 * ms:7.1f} us a token")


if __name__ == "__main__":
    main()
