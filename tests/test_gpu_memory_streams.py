"""The long-memory operators on a stream other than the caller's current one."""
import numpy as np
import pytest
import torch

from paper_2607_20293_amd import evo
from tests.gpu_util import device
from tests.memory_util import Call, i32

pytestmark = pytest.mark.gpu


def test_memory_released_on_the_current_stream_stays_there():
    """Temporaries of queued work on the current stream are released right
    before a call on a stream that does not wait for that work: neither side's
    results change, and the call's outputs lie elsewhere."""
    dev = device()
    c = Call(dev, "bf16", "int8", [3, 2], [3000, 2000], 4, 2, 64, seed=9, causal=True)
    cache, tab, lens, cu = evo.KVCache(*c.tensors), i32(c.tab, dev), i32(c.lengths, dev), i32(c.cu, dev)
    starts = i32(np.array(c.lengths) - np.array(c.rows), dev)
    x = torch.randn(5, 8, 64, device=dev, dtype=torch.bfloat16)
    table, side = evo.rope_table(4096, 64, device=dev), torch.cuda.Stream(dev)

    def calls(**kw):
        q = evo.qkv_write(cache, tab, starts, x[:, :4], x[:, 4:6], x[:, 6:], table, cu_rows=cu, max_rows=3, **kw)
        out, lse = evo.chunk_attention(q, cache, tab, lens, cu, 3, causal=True, **kw)
        k, v = evo.cache_read(cache, tab, starts, 5, torch.bfloat16, cu, 3, **kw)
        a, b = evo.qk_norm_rope(x[:, :4], x[:, 4:6], i32(range(5), dev), table, **kw)
        return [q, out, lse, k, v, a, b]
    want = [t.clone() for t in calls()]
    big = torch.randn(4096, 4096, device=dev)
    ready = torch.cuda.Event()
    ready.record()
    side.wait_event(ready)
    sizes = [t.numel() * t.element_size() for t in want] + [1 << 14, 1 << 16, 1 << 18]
    for r in range(10):
        for _ in range(3):                                      # some milliseconds of work
            big = torch.tanh(big @ big)
        held = [torch.full((n // 4,), float(r), device=dev) for n in sizes for _ in range(4)]
        kept = [t + 1 for t in held]
        released = {t.data_ptr() for t in held}
        del held
        got = calls(stream=side)
        assert all(t.data_ptr() not in released for t in got)
        torch.cuda.current_stream(dev).wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), r
        assert all(bool((t == r + 1).all()) for t in kept), r
