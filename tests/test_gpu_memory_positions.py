"""GPU parity of chunk attention at far positions."""
import numpy as np
import pytest
import torch

from paper_2607_20293_amd import evo
from tests.gpu_util import device, say
from tests.memory_util import Call, f64, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,fmt,rows,dh", [("bf16", "bf16", 5, 64), ("fp32", "fp32", 3, 32), ("bf16", "int8", 40, 64),
                                               ("bf16", "bf16", 90, 64), ("bf16", "fp8", 140, 128)])
@pytest.mark.parametrize("end", [2 ** 29 + 200, 2 ** 30 - 70, 2 ** 30])
def test_far_positions(dtype, fmt, rows, dh, end):
    """Positions up to 2^30: given starts mean what the cache's end means, and
    a window there sees what it sees near 0."""
    say(f"[gpu] far positions {dtype} over {fmt}: {rows} rows to {end}")
    dev, size = device(), 1024
    c = Call(dev, dtype, fmt, [rows], [512], 2, 2, dh, size=size, seed=22)     # one page of 512 used slots
    pages = c.tensors[0].shape[0]
    base = (end - 1) // size * size - size                 # the last two pages of the table hold the near ones
    tab = torch.zeros((1, 2 ** 30 // size), dtype=torch.int32, device=dev)
    tab[0, base // size] = 1
    tab[0, base // size + 1] = 2 if pages > 2 else 0
    near = i32([[1, 2 if pages > 2 else 0]], dev)
    cache, cu = evo.KVCache(*c.tensors), i32([0, rows], dev)
    kw = dict(cu_rows=cu, max_rows=rows, window=300, max_length=2048, slopes=torch.tensor([0.125, 0.001], device=dev))
    for causal in (True, False):
        want = evo.chunk_attention(c.q, cache, near, i32([end - base], dev), causal=causal, **kw)
        for starts in (None, i32([end - rows], dev)):
            got = evo.chunk_attention(c.q, cache, tab, i32([end], dev), causal=causal, starts=starts, **kw)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (causal, starts)
    # queries that lie behind all keys, and before them: row i then sees i keys
    kw["window"] = 2 ** 30 - end + 200
    got = evo.chunk_attention(c.q, cache, tab, i32([end], dev), causal=True, starts=i32([2 ** 30], dev), **kw)
    want = evo.chunk_attention(c.q, cache, near, i32([end - base], dev), causal=True, starts=i32([2 ** 30 - base], dev), **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    kw["window"] = 2 ** 30
    got = evo.chunk_attention(c.q, cache, near, i32([end - base], dev), starts=i32([-2 ** 30], dev), **kw)
    p, j = -2 ** 30 + np.arange(rows)[:, None], np.arange(end - base)[None]
    seen = (np.abs(p - j) < 2 ** 30).any(1)
    assert np.array_equal(np.isneginf(f64(got[1])).all(1), ~seen)
