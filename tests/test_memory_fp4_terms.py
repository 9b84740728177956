"""The softmax's terms of small bf16 calls over 4-bit caches have twice bf16's bits:
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

# up to 8 rows to a key/value head, and few enough workgroups not to fill the device
CALLS = [  # rows, lengths, heads, kv_heads, dh
    ([1], [1], 4, 4, 64), ([1], [40], 2, 2, 32), ([2], [250], 8, 2, 64), ([1, 1, 1], [64, 3, 300], 4, 4, 64),
    ([8], [200], 2, 2, 128), ([1], [600], 4, 4, 64), ([3], [1000], 4, 2, 32), ([1], [900], 8, 1, 128)]


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
        """(queries, keys, values) of each sequence."""
        k, v = (M.e2m1_of_bytes(x.numpy(), axis) for x, axis in ((self.k, 3), (self.v, 2)))
        at = 0
        for s, (n, length) in enumerate(zip(self.rows, self.lengths)):
            yield f64(self.q[at:at + n]), *M.gather(k, v, f64(self.ks), f64(self.vs), self.tab, s, length), s
            at += n

    def reference(self):
        """(outputs, bounds).  A term is off by 2^-16 of itself, or its exponential's
        2^-22, its exponent (EPS32 of the score a few times) and the sums of as many
        terms as there are keys; the output is rounded once,
        by half a step of its size."""
        outs, bounds = [], []
        for q, k, v, _ in self.parts():
            out, _ = M.attend(q, k, v, 0, SCALE)
            size, _ = M.attend(q, k, np.abs(v), 0, SCALE)
            z = np.max(np.sum(np.abs(q), -1)) * np.max(np.abs(k), initial=0) * SCALE
            outs.append(out)
            near = size * (2.0 ** -16 + 2.0 ** -22 + 16 * EPS32 * z + 2 * (len(k) + 64) * EPS32)
            half_step = EPS16 * 2.0 ** np.floor(np.log2(np.maximum(np.abs(out) + near, 1e-30)))
            bounds.append(near + half_step)
        return np.concatenate(outs), np.concatenate(bounds)

    def rounded(self, bits16):
        """The outputs of terms, with the value's scale in them, of 8 significant bits
        or of twice as many."""
        def half(x):
            return torch.from_numpy(x).to(BF16).double().numpy()
        outs = []
        for q, k, v, s in self.parts():
            place = [M.place(self.tab, 64, s, j) for j in range(len(k))]
            scale = np.stack([f64(self.vs)[pg, :, sl] for pg, sl in place])      # [keys][kv_heads]
            group = self.heads // k.shape[1]
            out = np.zeros(q.shape)
            for i in range(q.shape[0]):
                for h in range(self.heads):
                    z = SCALE * (k[:, h // group] @ q[i, h])
                    p = np.exp(z - np.max(z))
                    t = p * scale[:, h // group]
                    held = half(t) if not bits16 else half(t) + half(t - half(t))
                    out[i, h] = (held / scale[:, h // group]) @ v[:, h // group] / np.sum(p)
            outs.append(half(out))
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
def test_terms_of_small_calls(i):
    dev = device()
    say(f"[gpu] terms of rows {CALLS[i]}")
    call = Small(*CALLS[i], seed=i)
    want, bound = call.reference()
    err = np.abs(f64(call.run(dev)) - want)
    share = np.max(err / np.maximum(bound, 1e-300))
    print(f"  {share:.3f} of the bound; with terms of 8 bits {np.max(np.abs(call.rounded(False) - want) / np.maximum(bound, 1e-300)):.3f}", flush=True)
    assert share <= 1
