"""The long-memory example held to bounds that a wrong policy does not meet: its
attention over memory and chunk, and the chunk itself, against the oracle in 64
bits; and oracles with a mistake planted, which have to miss the bounds."""
import numpy as np
import pytest
import torch

from oracle import evo_memory as M
from tests.gpu_util import device, say
from tests.memory_util import EPS16, EPS32, f64
from tests.test_gpu_memory_example import _norm, _oracle

pytestmark = pytest.mark.gpu

LENGTHS, CHUNK = [70, 1, 45], 5


def _policy(dtype, fmt):
    from paper_2607_20293_amd.examples.long_memory import MemoryPolicy
    dev = device()
    pol = MemoryPolicy(LENGTHS, chunk=CHUNK, layers=2, heads=4, kv_heads=2, dh=32, ff=64, dtype=dtype, fmt=fmt, seed=5,
                       device=dev.type)
    gen = torch.Generator().manual_seed(6)
    tokens = torch.randn((sum(LENGTHS), pol.d), generator=gen).to(pol.dtype).to(dev)
    noise = torch.randn((4, len(LENGTHS), CHUNK, pol.d), generator=gen).to(pol.dtype).to(dev)
    return pol, tokens, noise


def _attention(pol, tokens, x, last, shift=0, causal=False, forget=False, swap=False):
    """The residual that layer `last`'s attention adds to the chunks x, after the
    memories have passed through the layers up to it.  The other arguments are
    mistakes: the chunk's positions shifted, its tokens' future hidden, the
    memory left out, another query's memory used."""
    w = {n: [f64(t) for t in getattr(pol, n)] for n in ("qkv", "out", "up", "down")}
    gains, table = [[f64(g) for g in pair] for pair in pol.gains], f64(pol.rope)
    hq, hk = pol.heads, pol.kv_heads

    def heads(i, x, start):
        y = (_norm(x) @ w["qkv"][i]).reshape(len(x), hq + 2 * hk, pol.dh)
        pos = start + np.arange(len(x))
        q, k = (M.norm_rope(t, g, table, pos, "halves", 1e-6) for t, g in zip((y[:, :hq], y[:, hq:hq + hk]), gains[i]))
        return q, k, y[:, hq + hk:]

    def attend(i, q, k, v, start, causal):
        return M.attend(q, k, v, start, pol.dh ** -0.5, causal=causal)[0].reshape(len(q), -1) @ w["out"][i]
    held, at = [], 0
    for n in pol.lengths:
        y = f64(tokens[at:at + n])
        at += n
        for i in range(last):
            y = y + attend(i, *heads(i, y, 0), 0, True)
            h = _norm(y) @ w["up"][i]
            y = y + h / (1 + np.exp(-h)) @ w["down"][i]
        held.append(heads(last, y, 0)[1:])
    out = []
    for s, n in enumerate(pol.lengths):
        q, k, v = heads(last, x[s * CHUNK:(s + 1) * CHUNK], max(0, n - shift))
        if not forget:
            k, v = (np.concatenate(p) for p in zip(held[s - 1 if swap else s], (k, v)))
        out.append(attend(last, q, k, v, len(k) - CHUNK, causal))
    return np.concatenate(out)


# A residual passes 8 roundings (norm, projection, rotation, cache of keys and of
# values, terms, attention's output, its projection), and as many more by way of
# the memory's pass through the first layer.  bf16: independent ones of at most
# EPS16, 0.6 EPS16 in the mean square, which the products' sums average as they
# average the values: 16 of them 2.4 EPS16, held to four times that.  An int8
# code is off by 1/254 of its row's largest value, some 2.2 deviations: 0.5% in
# the mean square, for keys and for values and in both layers; an fp8 code by 2.6%
# of its own value: 1% and 5.2% beside it, four times those.  fp32: 16 sums of at
# most 128 terms.
@pytest.mark.parametrize("dtype,fmt,bound", [
    ("fp32", "fp32", 16 * 128 * EPS32), ("bf16", "bf16", 4 * 2.4 * EPS16), ("bf16", "int8", 4 * (2.4 * EPS16 + 0.01)),
    ("bf16", "fp8", 4 * (2.4 * EPS16 + 0.052)), ("fp32", "fp8", 4 * 0.052)])
@pytest.mark.parametrize("layer", [0, 1])
def test_attention_over_memory_and_chunk(dtype, fmt, bound, layer):
    pol, tokens, noise = _policy(dtype, fmt)
    pol.write_memory(tokens)
    x = noise[0].flatten(0, 1)
    got = f64(pol._attention(layer, x, pol.held, pol.total, None, None, False))
    want = _attention(pol, tokens, f64(x), layer)
    top = np.max(np.abs(want))
    err = np.max(np.abs(got - want)) / top
    wrong = {name: np.max(np.abs(_attention(pol, tokens, f64(x), layer, **kw) - want)) / top
             for name, kw in (("shifted", dict(shift=1)), ("causal", dict(causal=True)), ("forgotten", dict(forget=True)),
                              ("swapped", dict(swap=True)))}
    say(f"[gpu] attention of the example {dtype} cache {fmt} layer {layer}: {err:.5f} of {bound:.5f}; mistakes "
        + ", ".join(f"{k} {v:.3f}" for k, v in wrong.items()))
    assert err <= bound
    if fmt == "fp8":  # (a shift by one position is smaller than what codes of 4 bits may do)
        del wrong["shifted"]
    assert all(v > bound for v in wrong.values()), wrong


# The chunk keeps 0.9 of itself at each of 3 steps and takes 0.1 of what the
# layers make: 3 roundings a step of values of its own size, and 0.1 of the
# layers' error, held to 30 roundings a step of values 1.5 times as large; 16-bit
# and 8-bit caches add 0.1 of the bound above for a residual half of that size.
@pytest.mark.parametrize("dtype,fmt,bound", [
    ("fp32", "fp32", 3 * (3 + 4.5) * 128 * EPS32), ("bf16", "bf16", 3 * (3 + 4.5) * EPS16),
    ("bf16", "int8", 3 * ((3 + 4.5) * EPS16 + 0.1 * 0.75 * 4 * 0.01)),
    ("bf16", "fp8", 3 * ((3 + 4.5) * EPS16 + 0.1 * 0.75 * 4 * 0.052))])
def test_chunk(dtype, fmt, bound):
    from paper_2607_20293_amd.examples.long_memory import lattice_every
    pol, tokens, noise = _policy(dtype, fmt)
    lattice = lattice_every(2, 3, 2)
    pol.write_memory(tokens)
    got = f64(pol.denoise(noise, lattice))
    want = _oracle(pol, tokens, noise, lattice)
    top = np.max(np.abs(want))
    err = np.max(np.abs(got - want)) / top
    last = np.max(np.abs(f64(noise[0]) - want)) / top
    every = np.max(np.abs(_oracle(pol, tokens, noise, lattice_every(2, 3, 1)) - want)) / top
    say(f"[gpu] chunk of the example {dtype} cache {fmt}: {err:.5f} of {bound:.5f}; the noise itself {last:.3f}, "
        f"every step refreshed {every:.4f}")
    assert err <= bound < 0.2
    assert last > bound
    if dtype == "fp32":
        assert every > bound
