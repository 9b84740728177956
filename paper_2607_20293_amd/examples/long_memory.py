"""A policy conditioned on a long memory, denoised with a refresh lattice.

Each query has a memory of its own length (history, image patches, language).
Its tokens pass through the layers once: norm, rotation and write of their keys
and values into the paged cache (`evo.qkv_write`), then their own causal
attention (`evo.chunk_attention`).  The reverse steps then work on the action
chunk alone: its tokens lie behind the memory, write their keys and values over
the step before's, and attend to memory and chunk.  A layer's two residuals are
computed where the lattice says so and added from their cache elsewhere (Eq. 1).

The steps of a chunk are recorded once into a HIP graph and replayed for every
set of queries of the same lattice.

    python -m paper_2607_20293_amd.examples.long_memory [--queries 16] [--memory 2000] [--format int8]

prints one JSON line.  Weights and inputs are synthetic.
"""
from __future__ import annotations

import argparse
import json

import torch

from paper_2607_20293_amd import evo

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
FORMATS = {"fp32": torch.float32, "bf16": torch.bfloat16, "int8": torch.int8, "fp8": torch.float8_e4m3fn}
EPS = 1e-6


class MemoryPolicy:
    """Layers of attention and feed-forward with synthetic weights, and the
    caches of `lengths` memories (tokens of each query)."""

    def __init__(self, lengths, chunk=16, layers=4, heads=4, kv_heads=4, dh=64, ff=1024, dtype="bf16", fmt="bf16", seed=0,
                 page=64, device="cuda"):
        self.lengths, self.chunk, self.layers = list(lengths), chunk, layers
        self.heads, self.kv_heads, self.dh, self.d = heads, kv_heads, dh, heads * dh
        self.dtype, self.device = DTYPES[dtype], torch.device(device, torch.cuda.current_device())
        g = torch.Generator().manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn((rows, cols), generator=g) * rows ** -0.5).to(self.dtype).to(self.device)
        wide = (heads + 2 * kv_heads) * dh
        self.qkv = [weight(self.d, wide) for _ in range(layers)]
        self.out = [weight(heads * dh, self.d) for _ in range(layers)]
        self.up = [weight(self.d, ff) for _ in range(layers)]
        self.down = [weight(ff, self.d) for _ in range(layers)]
        self.gains = [tuple((1 + 0.1 * torch.randn(dh, generator=g)).to(self.device) for _ in range(2)) for _ in range(layers)]

        n = len(self.lengths)
        counts = [-(-(t + chunk) // page) for t in self.lengths]
        wide = max(counts)
        table = torch.zeros((n, wide), dtype=torch.int32)
        at = 0
        for s, c in enumerate(counts):
            table[s, :c] = torch.arange(at, at + c)
            at += c
        self.table = table.to(self.device)
        self.caches = [evo.KVCache.empty(at, kv_heads, dh, page, FORMATS[fmt], self.device) for _ in range(layers)]
        self.rope = evo.rope_table(max(self.lengths) + chunk, dh, device=self.device)

        def ints(v):
            return torch.tensor(v, dtype=torch.int32, device=self.device)
        cu = [0]
        for t in self.lengths:
            cu.append(cu[-1] + t)
        self.cu, self.zero = ints(cu), ints([0] * n)
        self.held, self.total = ints(self.lengths), ints([t + chunk for t in self.lengths])

    @staticmethod
    def _norm(x):
        f = x.float()
        return (f * torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)).to(x.dtype)

    def _attention(self, layer, x, starts, lengths, cu, most, causal):
        """The attention's residual of tokens x [rows][d]."""
        hq, hk = self.heads, self.kv_heads
        y = (self._norm(x) @ self.qkv[layer]).unflatten(1, (hq + 2 * hk, self.dh))
        cache = self.caches[layer]
        q = evo.qkv_write(cache, self.table, starts, y[:, :hq], y[:, hq:hq + hk], y[:, hq + hk:], self.rope,
                          *self.gains[layer], EPS, "halves", cu, most)
        a, _ = evo.chunk_attention(q, cache, self.table, lengths, cu, most, causal=causal)
        return a.flatten(1) @ self.out[layer]

    def _forward(self, layer, x):
        return torch.nn.functional.silu(self._norm(x) @ self.up[layer]) @ self.down[layer]

    def write_memory(self, tokens):
        """tokens [sum of lengths][d], the queries' memories one after another."""
        x = tokens
        for i in range(self.layers):
            x = x + self._attention(i, x, self.zero, self.held, self.cu, max(self.lengths), True)
            x = x + self._forward(i, x)

    def denoise(self, noise, lattice):
        """noise [steps + 1][queries][chunk][d]: the first is the chunk the
        steps start from; lattice [layers][steps] of truth values, its first
        step all true.  Returns the chunk after the last step."""
        x = noise[0].flatten(0, 1)
        held = [[None, None] for _ in range(self.layers)]
        steps = noise.shape[0] - 1
        for t in range(steps):
            y = x
            for i in range(self.layers):
                if lattice[i][t]:
                    held[i][0] = self._attention(i, y, self.held, self.total, None, None, False)
                y = y + held[i][0]
                if lattice[i][t]:
                    held[i][1] = self._forward(i, y)
                y = y + held[i][1]
            keep = 0.9
            x = keep * x + (1 - keep) * y + 0.1 * noise[t + 1].flatten(0, 1)
        return x.unflatten(0, (len(self.lengths), self.chunk))

    def record(self, noise, lattice):
        """(graph, chunk): denoise() of what `noise` and the caches hold at each
        replay."""
        side = torch.cuda.Stream(self.device)
        side.wait_stream(torch.cuda.current_stream(self.device))
        with torch.cuda.stream(side):
            self.denoise(noise, lattice)
        torch.cuda.current_stream(self.device).wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = self.denoise(noise, lattice)
        return graph, out


def lattice_every(layers, steps, every):
    return [[t % every == 0 for t in range(steps)] for _ in range(layers)]


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--queries", type=int, default=16)
    p.add_argument("--memory", type=int, default=2000, help="tokens of the longest memory")
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--every", type=int, default=4, help="refresh every so many steps")
    p.add_argument("--dtype", choices=sorted(DTYPES), default="bf16")
    p.add_argument("--format", choices=sorted(FORMATS), default=None, help="of the cache (default: the dtype)")
    a = p.parse_args(argv)
    if a.queries < 1 or a.memory < 1 or a.steps < 1 or a.every < 1:
        p.error("queries, memory, steps and every are at least 1")
    lengths = [max(1, a.memory - a.memory * s // (2 * a.queries)) for s in range(a.queries)]
    pol = MemoryPolicy(lengths, dtype=a.dtype, fmt=a.format or a.dtype)
    g = torch.Generator(device=pol.device).manual_seed(1)
    tokens = torch.randn((sum(lengths), pol.d), generator=g, device=pol.device).to(pol.dtype)
    noise = torch.randn((a.steps + 1, a.queries, pol.chunk, pol.d), generator=g, device=pol.device).to(pol.dtype)
    lattice = lattice_every(pol.layers, a.steps, a.every)
    pol.write_memory(tokens)
    graph, out = pol.record(noise, lattice)
    marks = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    marks[0].record()
    pol.write_memory(tokens)
    marks[1].record()
    graph.replay()
    marks[2].record()
    torch.cuda.synchronize()
    print(json.dumps({"queries": a.queries, "memory_tokens": sum(lengths), "cache": a.format or a.dtype, "steps": a.steps,
                      "refreshed_steps": sum(lattice[0]), "finite": bool(torch.isfinite(out).all()),
                      "write_memory_ms": round(marks[0].elapsed_time(marks[1]), 3),
                      "denoise_ms": round(marks[1].elapsed_time(marks[2]), 3)}), flush=True)


if __name__ == "__main__":
    main()
