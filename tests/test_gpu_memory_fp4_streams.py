"""Calls on two streams at once that write neighbouring slots of one page of 4-bit
floats, each ordered behind what made its arguments."""
import pytest
import torch

from paper_2607_20293_amd import evo
from tests.gpu_util import device, say
from tests.test_gpu_memory_fp4 import handle, pool4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_streams_that_write_neighbouring_slots(dtype, dh):
    """A call of a stream of its own waits for nothing by itself: `side` waits for the
    stream that made its arguments."""
    dev, gen = device(), torch.Generator().manual_seed(dh)
    say(f"[gpu] two streams write neighbouring slots {dtype} dh {dh}")
    x = torch.randn((64, 4, dh), generator=gen).to(dtype).to(dev)
    tab = torch.zeros((64, 1), dtype=torch.int32, device=dev)
    order = torch.randperm(64, generator=gen).int().to(dev)
    want, got = ([t.clone() for t in pool4(1, 2, 64, dh, dev, gen)] for _ in range(2))
    evo.cache_write(handle(want), tab, order, x[:, :2], x[:, 2:])
    sides = [torch.cuda.Stream(dev) for _ in range(2)]
    parts = [(tab[:32], order[half::2].contiguous(), x[half::2, :2], x[half::2, 2:]) for half in (0, 1)]
    for side, part in zip(sides, parts):
        side.wait_stream(torch.cuda.current_stream(dev))
        evo.cache_write(handle(got), *part, stream=side)
    for side in sides:
        torch.cuda.current_stream(dev).wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
