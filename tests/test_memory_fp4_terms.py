"""The softmax's terms of bf16 calls over 4-bit caches have twice bf16's bits where a
sequence has few rows to a key/value head or few positions, whatever else the call holds:
against the definition in 64 bits, with a bound that terms of bf16's own 8 bits break
(shown on the CPU)."""
import numpy as np
import pytest
import torch

from oracle import evo_memory as M
from paper_2607_20293_amd import evo
from tests.gpu_util import device, say
from tests.memory_util import EPS16, EPS32, f64, i32, table_for

FP4, BF16 = torch.float4_e2m1fn_x2, torch.bfloat16
SCALE = 0.125

# up to 8 rows to a key/value head, few workgroups and enough to fill the device; any
# number of rows over up to 64 positions
CALLS = [  # rows, lengths, heads, kv_heads, dh
    ([1], [1], 4, 4, 64), ([1], [40], 2, 2, 32), ([2], [250], 8, 2, 64), ([1, 1, 1], [64, 3, 300], 4, 4, 64),
    ([8], [200], 2, 2, 128), ([1], [600], 4, 4, 64), ([3], [1000], 4, 2, 32), ([1], [900], 8, 1, 128),
    ([1] * 96, [1 + 37 * s % 250 for s in range(96)], 12, 12, 64), ([1] * 34, [700 - 19 * s for s in range(34)], 32, 8, 128),
    ([2, 1] * 20, [1300 - 60 * (s % 7) for s in range(40)], 8, 8, 32), ([7] * 70, [5 + s for s in range(70)], 4, 4, 64),
    ([17], [30], 8, 2, 32), ([40, 300], [64, 7], 2, 2, 64), ([150], [60], 2, 2, 128), ([60, 1], [3, 64], 4, 1, 128)]


class Small:
    """A call whose scores are exact up to their last few roundings: small whole
    numbers as queries, powers of two as the keys' scales."""

    def __init__(self, rows, lengths, heads, kv_heads, dh, seed):
        gen, rng = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
        self.rows, self.lengths, self.heads = rows, lengths, heads
        self.tab, pages = table_for(lengths, 64, 2, rng)
        self.k = torch.randint(0, 256, (pages, kv_heads, 64, dh // 2), generator=gen, dtype=torch.uint8)
        self.v = torch.randint(0, 256, (pages, kv_heads, dh // 2, 64), generator=gen, dtype=torch.uint8)
        self.ks = torch.full((pages, kv_heads, 64), 0.5)
        # values' scales up to half a step of bf16 off it
        self.vs = (1 + 2.0 ** -8 * (0.2 + 0.78 * torch.rand(self.ks.shape, generator=gen))) * 2.0 ** torch.randint(-2, 3, self.ks.shape,
                                                                                                                      generator=gen)
        self.q = torch.randint(-3, 4, (sum(rows), heads, dh), generator=gen).to(BF16)

    def parts(self):
        """(scores [heads][rows][keys], values' codes and scales by query head
        [heads][keys][dh] and [heads][keys]) of each sequence."""
        k, v = M.e2m1_of_bytes(self.k.numpy(), 3), M.e2m1_of_bytes(self.v.numpy(), 2)
        at = 0
        for s, (n, length) in enumerate(zip(self.rows, self.lengths)):
            j = np.arange(length)
            page, slot = self.tab[s][j // 64], j % 64
            group = self.heads // k.shape[1]
            keys, values = (np.repeat(x.swapaxes(0, 1), group, 0) for x in (k[page, :, slot] * 0.5, v[page, :, :, slot]))
            scale = np.repeat(f64(self.vs)[page, :, slot].T, group, 0)
            yield SCALE * (f64(self.q[at:at + n]).swapaxes(0, 1) @ keys.swapaxes(1, 2)), values, scale
            at += n

    def reference(self):
        """(outputs, bounds).  A term is off by 2^-16 of itself, or its exponential's
        2^-22, its exponent (EPS32 of the score a few times) and the sums of as many
        terms as there are keys; the output is rounded once, by half a step of its size."""
        outs, bounds = [], []
        for z, v, scale in self.parts():
            p = np.exp(z - z.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            v = v * scale[..., None]
            out, size, keys = p @ v, p @ np.abs(v), z.shape[-1]
            near = size * (2.0 ** -16 + 2.0 ** -22 + 16 * EPS32 * np.max(np.abs(z)) + 2 * (keys + 64) * EPS32)
            half_step = EPS16 * 2.0 ** np.floor(np.log2(np.maximum(np.abs(out) + near, 1e-30)))
            outs.append(out.swapaxes(0, 1))
            bounds.append((near + half_step).swapaxes(0, 1))
        return np.concatenate(outs), np.concatenate(bounds)

    def rounded(self, bits16):
        """The outputs of terms, with the value's scale in them, of 8 significant bits
        or of twice as many."""
        def half(x):
            return torch.from_numpy(x).to(BF16).double().numpy()
        outs = []
        for z, v, scale in self.parts():
            p = np.exp(z - z.max(-1, keepdims=True))
            t = p * scale[:, None]
            held = half(t) if not bits16 else half(t) + half(t - half(t))
            outs.append(half(held @ v / p.sum(-1, keepdims=True)).swapaxes(0, 1))
        return np.concatenate(outs)

    def run(self, dev):
        cache = evo.KVCache(self.k.to(dev).view(FP4), self.v.to(dev).view(FP4), self.ks.to(dev), self.vs.to(dev))
        cu = i32(np.concatenate([[0], np.cumsum(self.rows)]), dev)
        return evo.chunk_attention(self.q.to(dev), cache, i32(self.tab, dev), i32(self.lengths, dev), cu, max(self.rows), scale=SCALE)[0]


@pytest.mark.parametrize("i", range(len(CALLS)))
def test_the_bound_tells_16_bits_from_8(i):
    call = Small(*CALLS[i], seed=i)
    want, bound = call.reference()
    assert np.all(np.abs(call.rounded(True) - want) <= bound)
    assert np.mean(np.abs(call.rounded(False) - want) > bound) > 0.01


@pytest.mark.gpu
@pytest.mark.parametrize("i", range(len(CALLS)))
def test_terms_of_16_bits(i):
    dev = device()
    say(f"[gpu] terms of rows {CALLS[i]}")
    call = Small(*CALLS[i], seed=i)
    want, bound = call.reference()
    err = np.abs(f64(call.run(dev)) - want)
    share = np.max(err / np.maximum(bound, 1e-300))
    print(f"  {share:.3f} of the bound; with terms of 8 bits {np.max(np.abs(call.rounded(False) - want) / np.maximum(bound, 1e-300)):.3f}", flush=True)
    assert share <= 1
