"""The long-memory example with weights in 4 bits, whose layers then run the products
and the norms around a block, against the same policy in 64 bits."""
import json

import numpy as np
import pytest
import torch

from tests.gpu_util import device, say
from tests.memory_util import EPS16, EPS32, f64
from tests.test_gpu_memory_example import _oracle

pytestmark = pytest.mark.gpu


def _policy(dtype, fmt):
    from paper_2607_20293_amd.examples.long_memory import MemoryPolicy, lattice_every
    dev = device()
    pol = MemoryPolicy([70, 1, 45], chunk=5, layers=2, heads=4, kv_heads=2, dh=32, ff=64, dtype=dtype, fmt=fmt, device=dev.type,
                       weights="4bit")
    gen = torch.Generator().manual_seed(3)

    def inputs():
        return (torch.randn((116, pol.d), generator=gen).to(pol.dtype).to(dev),
                torch.randn((4, 3, 5, pol.d), generator=gen).to(pol.dtype).to(dev))
    return pol, lattice_every(2, 3, 2), inputs


# The bounds of the example with weights of the dtype: the policy passes the same
# roundings or fewer, and the weights are the values of their codes on both sides.
@pytest.mark.parametrize("dtype,bound", [("fp32", 512 * 100 * EPS32), ("bf16", 4 * 128 ** 0.5 * EPS16)])
def test_policy_of_4_bit_weights(dtype, bound):
    say(f"[gpu] policy over long memories {dtype}, weights in 4 bits")
    pol, lattice, inputs = _policy(dtype, dtype)
    tokens, noise = inputs()
    pol.write_memory(tokens)
    want = _oracle(pol, tokens, noise, lattice)
    err = np.max(np.abs(f64(pol.denoise(noise, lattice)) - want)) / np.max(np.abs(want))
    print(f"  chunk {err / bound:.3f} of its bound", flush=True)
    assert err <= bound


@pytest.mark.parametrize("fmt", ["fp4", "int8", "bf16"])
def test_policy_of_4_bit_weights_replayed(fmt):
    pol, lattice, inputs = _policy("bf16", fmt)
    tokens, noise = inputs()
    pol.write_memory(tokens)
    graph, out = pol.record(noise, lattice)
    for r in range(3):
        for held, new in zip((tokens, noise), inputs()):
            held.copy_(new)
        pol.write_memory(tokens)
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        pol.write_memory(tokens)
        assert torch.equal(replayed, pol.denoise(noise, lattice)) and bool(torch.isfinite(replayed).all()), r


def test_example_of_4_bits_prints_its_line(capsys):
    from paper_2607_20293_amd.examples import long_memory
    device()
    long_memory.main(["--queries", "3", "--memory", "200", "--steps", "4", "--every", "2", "--format", "fp4", "--weights", "4bit"])
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["finite"] and line["weights"] == "4bit" and line["cache"] == "fp4"
