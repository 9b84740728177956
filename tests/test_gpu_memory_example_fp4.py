"""The long-memory example with 4-bit caches against the oracle in 64 bits, with
weights in the dtype and in 4 bits: what its caches hold, its attention over what they
hold, and the chunk."""
import numpy as np
import pytest
import torch

from oracle import evo_memory as M
from paper_2607_20293_amd import evo
from tests.gpu_util import device, say
from tests.memory_util import EPS16, EPS32, f64, i32
from tests.test_gpu_memory_example import _norm, _oracle

pytestmark = pytest.mark.gpu

LENGTHS, CHUNK = [70, 1, 45], 5


def _policy(dtype, weights):
    from paper_2607_20293_amd.examples.long_memory import MemoryPolicy
    dev = device()
    pol = MemoryPolicy(LENGTHS, chunk=CHUNK, layers=2, heads=4, kv_heads=2, dh=32, ff=64, dtype=dtype, fmt="fp4", seed=5,
                       device=dev.type, weights=weights)
    gen = torch.Generator().manual_seed(6)
    tokens = torch.randn((sum(LENGTHS), pol.d), generator=gen).to(pol.dtype).to(dev)
    noise = torch.randn((4, len(LENGTHS), CHUNK, pol.d), generator=gen).to(pol.dtype).to(dev)
    return pol, tokens, noise


def _read(pol, layer, lengths):
    """Keys and values of each query as the layer's cache holds them."""
    n = sum(lengths)
    cu = i32(np.concatenate([[0], np.cumsum(lengths)]), pol.device)
    k, v = (f64(t) for t in evo.cache_read(pol.caches[layer], pol.table, pol.zero, n, torch.float32, cu, max(lengths)))
    at = np.cumsum(lengths)[:-1]
    return list(zip(np.split(k, at), np.split(v, at)))


def _heads(pol, layer, x, start):
    w, pos = f64(pol.qkv[layer]), start + np.arange(len(x))
    y = (_norm(x) @ w).reshape(len(x), pol.heads + 2 * pol.kv_heads, pol.dh)
    q, k = (M.norm_rope(t, f64(g), f64(pol.rope), pos, "halves", 1e-6)
            for t, g in zip((y[:, :pol.heads], y[:, pol.heads:pol.heads + pol.kv_heads]), pol.gains[layer]))
    return q, k, y[:, pol.heads + pol.kv_heads:]


def _attend(pol, layer, q, held, start, causal):
    return M.attend(q, *held, start, pol.dh ** -0.5, causal=causal)[0].reshape(len(q), -1) @ f64(pol.out[layer])


def _half_step(x, off):
    """Half a step of the codes of rows x that are up to `off` off."""
    s = (np.max(np.abs(x), -1, keepdims=True) + off) / 6
    y = (np.abs(x) + off) / s
    return s * np.where(y < 2, 0.25, np.where(y < 4, 0.5, 1.0)) + off


# Off: a residual's 8 roundings and as many by way of the first layer, each of a row of
# at most 128 terms (fp32: 16 sums of EPS32 a term; bf16: independent roundings of 0.6
# EPS16 in the mean square, 2.4 EPS16 of 16, four times that), of the largest value of
# a row, whose codes' scale is off by as much.
OFF = {"fp32": 16 * 128 * EPS32, "bf16": 4 * 2.4 * EPS16}


@pytest.mark.parametrize("weights", [None, "4bit"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_caches_and_attention_of_the_example(dtype, weights):
    """Each layer from what the caches before it hold, so that only its own codes'
    rounding is between it and the oracle, and none of it in its attention."""
    pol, tokens, noise = _policy(dtype, weights)
    pol.write_memory(tokens)
    x, x64 = noise[0].flatten(0, 1), f64(noise[0])
    memories = np.split(f64(tokens), np.cumsum(LENGTHS)[:-1])
    for layer in range(pol.layers):
        worst = 0
        held = _read(pol, layer, LENGTHS)
        for s, n in enumerate(LENGTHS):
            q, k, v = _heads(pol, layer, memories[s], 0)
            for got, want in zip(held[s], (k, v)):
                off = OFF[dtype] * np.max(np.abs(want), -1, keepdims=True)
                worst = max(worst, np.max(np.abs(got - want) / _half_step(want, off)))
            y = memories[s] + _attend(pol, layer, q, held[s], 0, True)
            h = _norm(y) @ f64(pol.up[layer])
            memories[s] = y + h / (1 + np.exp(-h)) @ f64(pol.down[layer])
        got = f64(pol._attention(layer, x, pol.held, pol.total, None, None, False)).reshape(x64.shape)
        all_held = _read(pol, layer, [n + CHUNK for n in LENGTHS])
        want, swapped, forgotten = [], [], []
        for s, n in enumerate(LENGTHS):
            q, k, v = _heads(pol, layer, x64[s], n)
            for g, w in zip(all_held[s], (k, v)):
                off = OFF[dtype] * np.max(np.abs(w), -1, keepdims=True)
                worst = max(worst, np.max(np.abs(g[n:] - w) / _half_step(w, off)))
            want.append(_attend(pol, layer, q, all_held[s], n, False))
            swapped.append(_attend(pol, layer, q, all_held[s - 1], n, False))
            forgotten.append(_attend(pol, layer, q, [t[n:] for t in all_held[s]], n, False))
        top = np.max(np.abs(want))
        err = np.max(np.abs(got - np.stack(want))) / top
        wrong = [np.max(np.abs(np.stack(t) - np.stack(want))) / top for t in (swapped, forgotten)]
        say(f"[gpu] example {dtype}, fp4, weights {weights}, layer {layer}: codes {worst:.3f} of half a step, attention {err:.6f} of "
            f"{OFF[dtype]:.6f}; another memory {wrong[0]:.3f}, none {wrong[1]:.3f}")
        assert worst <= 1 and err <= OFF[dtype] < min(wrong)


# The chunk keeps 0.9 of itself at each of 3 steps and takes 0.1 of what the layers
# make: 3 roundings a step of values of its own size, and 0.1 of the layers' error, held
# to 30 roundings a step of values 1.5 times as large.  Codes of rows whose largest value is some
# 2.3 deviations: 2.6 units of the scale to a deviation, of which 0.56, 0.31 and 0.13 meet steps of 0.5, 1
# and 2, off by 0.28 units in the mean square, 0.107 of a deviation, for keys and for
# values in both layers: 0.214 of a residual half of the chunk's size at most, and four times that.
@pytest.mark.parametrize("weights", [None, "4bit"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_chunk_of_the_example(dtype, weights):
    from paper_2607_20293_amd.examples.long_memory import lattice_every
    pol, tokens, noise = _policy(dtype, weights)
    lattice = lattice_every(2, 3, 2)
    pol.write_memory(tokens)
    got = f64(pol.denoise(noise, lattice))
    want = _oracle(pol, tokens, noise, lattice)
    top = np.max(np.abs(want))
    bound = 3 * ((3 + 4.5) * EPS16 + 0.1 * 0.75 * 4 * 0.214)
    err, last = np.max(np.abs(got - want)) / top, np.max(np.abs(f64(noise[0]) - want)) / top
    say(f"[gpu] chunk of the example {dtype}, fp4, weights {weights}: {err:.5f} of {bound:.5f}; the noise itself {last:.3f}")
    assert err <= bound < last
