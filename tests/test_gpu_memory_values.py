"""GPU parity of chunk attention over values near the end of the floats' range,
and with scores far beyond it for an exponential."""
import numpy as np
import pytest
import torch

from oracle import evo_memory as M
from paper_2607_20293_amd import evo
from tests.gpu_util import device, say
from tests.memory_util import DTYPES, EPS16, EPS32, FORMATS, f64, i32

pytestmark = pytest.mark.gpu


def _cache_of(dev, fmt, dtype, k, v, size=64):
    """A cache that was written with k and v [keys][heads][dh], its table, and
    what it holds in 64 bits."""
    n, heads, dh = k.shape
    cache = evo.KVCache.empty(-(-n // size), heads, dh, size, FORMATS[fmt], dev)
    order = np.random.default_rng(23).permutation(cache.n_pages).astype(np.int32)[None]
    tab = i32(order, dev)
    evo.cache_write(cache, tab, i32([0], dev), k.to(DTYPES[dtype]).to(dev), v.to(DTYPES[dtype]).to(dev))
    arr = [f64(t) if t is not None else None for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    return cache, tab, M.gather(*arr, order, 0, n)


@pytest.mark.parametrize("dtype,fmt", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "int8"), ("bf16", "fp8"), ("fp32", "fp8")])
@pytest.mark.parametrize("rows,dh,split", [(3, 64, 1), (3, 64, 0), (40, 128, 1), (200, 64, 1), (300, 128, 1)])
def test_large_values(dtype, fmt, rows, dh, split):
    """Values of 1e37 whose weights sum to 1: the later half of the blocks holds
    scores 7 powers of 2 above the first half's."""
    dev, keys = device(), 1024
    say(f"[gpu] large values {dtype} over {fmt}: {rows} rows, dh {dh}")
    gen = torch.Generator().manual_seed(24)
    j = torch.arange(keys)
    z = torch.where(j % 64 == 5, torch.where(j < keys // 2, 0.0, 4.75), -40.0)
    k = torch.zeros(keys, 1, dh)
    k[:, 0, 0] = z
    v = 1e37 * (1 + torch.rand((keys, 1, dh), generator=gen))
    cache, tab, (kk, vv) = _cache_of(dev, fmt, dtype, k, v)
    q = torch.zeros(rows, 1, dh)
    q[:, 0, 0] = 1
    q = q.to(DTYPES[dtype]).to(dev)
    out, lse = evo.chunk_attention(q, cache, tab, i32([keys], dev), scale=1.0, max_length=split)
    want, want_lse = M.attend(f64(q), kk, vv, 0, 1.0)
    # scores of one product; terms, sums over 16 keys and the output's rounding
    assert np.max(np.abs(f64(out) - want)) <= 2e37 * (64 * EPS32 + (2.1 * EPS16 if dtype == "bf16" else 0))
    assert np.max(np.abs(f64(lse) - want_lse)) <= 64 * EPS32 * 8


@pytest.mark.parametrize("dtype,fmt", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "int8"), ("fp32", "fp8")])
@pytest.mark.parametrize("rows,dh", [(3, 64), (40, 64), (200, 64), (300, 128)])
@pytest.mark.parametrize("size", [3e2, 1e4, 3e5])
def test_large_scores(dtype, fmt, rows, dh, size):
    """Scores far beyond 2^32: the largest takes all, and the sum's logarithm
    is that score."""
    dev, keys = device(), 700
    say(f"[gpu] large scores {dtype} over {fmt}: {rows} rows, dh {dh}, size {size:g}")
    gen = torch.Generator().manual_seed(25)
    k, v = torch.randn((keys, 2, dh), generator=gen) * size, torch.randn((keys, 2, dh), generator=gen)
    cache, tab, (kk, vv) = _cache_of(dev, fmt, dtype, k, v)
    q = (torch.randn((rows, 2, dh), generator=gen) * size).to(DTYPES[dtype]).to(dev)
    for scale in (0.125, -0.125):
        z = np.einsum("rhd,khd->rhk", f64(q), kk) * scale
        order = np.sort(z, -1)
        # rows whose second score is further off than products of dh terms in fp32 can move it
        slack = 8 * dh * EPS32 * np.max(np.abs(f64(q)), (1, 2))[:, None] * np.max(np.abs(kk)) * dh * abs(scale)
        clear = order[..., -1] - order[..., -2] > slack + 100
        assert clear.mean() > 0.5
        out, lse = evo.chunk_attention(q, cache, tab, i32([keys], dev), scale=scale)
        best = np.argmax(z, -1)
        want = np.stack([vv[best[:, h], h] for h in range(2)], 1)
        err = np.abs(f64(out) - want)[clear]
        assert np.all(err <= np.abs(want[clear]) * (EPS16 * 2.02 if dtype == "bf16" else 64 * EPS32))
        assert np.all(np.abs(f64(lse) - order[..., -1]) <= 16 * dh * EPS32 * np.abs(f64(q)).max() * np.abs(kk).max() * dh ** 0.5 + slack)


@pytest.mark.parametrize("dtype,fmt", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "int8")])
@pytest.mark.parametrize("rows,dh", [(16, 64), (31, 64), (100, 64), (140, 128)])
def test_large_scores_beside_small_and_none(dtype, fmt, rows, dh):
    """Rows of one wave whose scores are huge, ordinary, and of nothing: each is
    what it is alone."""
    dev, keys = device(), 300
    gen = torch.Generator().manual_seed(28)
    k, v = torch.randn((keys, 1, dh), generator=gen), torch.randn((keys, 1, dh), generator=gen)
    cache, tab, (kk, vv) = _cache_of(dev, fmt, dtype, k, v)
    q = torch.randn((rows, 1, dh), generator=gen)
    q[::3] *= 1e12
    q = q.to(DTYPES[dtype]).to(dev)
    # the first third of the rows lie before all keys
    start = -(rows // 3)
    out, lse = evo.chunk_attention(q, cache, tab, i32([keys], dev), causal=True, starts=i32([start], dev))
    want, want_lse = M.attend(f64(q), kk, vv, start, dh ** -0.5, causal=True)
    none = np.arange(rows) < -start
    assert not f64(out)[none].any() and np.isneginf(f64(lse)[none]).all() and np.isfinite(f64(lse)[~none]).all()
    small = ~none & (np.arange(rows) % 3 != 0)
    # dh products of at most |q| |k|, the terms' and the output's rounding
    dz = 4 * EPS32 * dh * dh ** 0.5 * np.max(np.abs(f64(q)[small])) * np.max(np.abs(kk))
    bound = np.max(np.abs(vv)) * (4 * dz + 4 * (keys + 64) * EPS32 + (1.01 * EPS16 if dtype == "bf16" else 0))
    assert np.max(np.abs(f64(out) - want)[small]) <= bound
    assert np.max(np.abs(f64(lse) - want_lse)[small]) <= 2 * dz + (keys + 64) * EPS32 + 1e-6
    large = ~none & (np.arange(rows) % 3 == 0)
    z = np.einsum("rhd,khd->rhk", f64(q), kk) * dh ** -0.5
    for i in np.nonzero(large)[0]:
        see = z[i, 0, :start + i + 1]
        best = np.argmax(see)
        rest = np.delete(see, best)
        if rest.size and see[best] - np.max(rest) < 8 * dh * EPS32 * dh ** 0.5 * np.max(np.abs(f64(q)[i])) * np.max(np.abs(kk)):
            continue
        err = np.abs(f64(out)[i, 0] - vv[best, 0])
        assert np.all(err <= np.abs(vv[best, 0]) * (EPS16 * 2.02 if dtype == "bf16" else 64 * EPS32)), i
