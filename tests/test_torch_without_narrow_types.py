"""CPU test: with a torch that has no 4-bit floats and no power-of-two scales, caches of
the other formats and weights of bytes work as ever."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import torch
for name in ("float4_e2m1fn_x2", "float8_e8m0fnu"):
    if hasattr(torch, name):
        delattr(torch, name)
from paper_2607_20293_amd import evo
from paper_2607_20293_amd.examples import long_memory
evo._device_of = lambda t: t.device
for dtype in (torch.float32, torch.bfloat16, torch.int8, torch.float8_e4m3fn):
    c = evo.KVCache.empty(2, 2, 32, 64, dtype, "cpu")
    assert c.head_dim == 32 and (c.k_scale is None) == (dtype in (torch.float32, torch.bfloat16))
assert evo.KVCache.empty(2, 2, 32, 64, None, "cpu").k.dtype == torch.bfloat16
for bad in (torch.float16, torch.uint8):
    try:
        evo.KVCache.empty(2, 2, 32, 64, bad, "cpu")
    except TypeError:
        continue
    raise SystemExit(f"a cache of {bad}")
w = evo.Weights4(torch.zeros(8, 64, dtype=torch.uint8), torch.zeros(8, 4, dtype=torch.uint8), 32)
assert w.n_out == 8
for bad in (dict(codes=torch.zeros(8, 64)), dict(scales=torch.zeros(8, 4))):
    try:
        evo.Weights4(**{**dict(codes=w.codes, scales=w.scales, n_in=32), **bad})
    except TypeError:
        continue
    raise SystemExit("weights of floats")
assert sorted(long_memory.FORMATS) == ["bf16", "fp32", "fp8", "int8"]
print("fine")
"""


def test_other_formats_need_no_4_bit_floats():
    run = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip().endswith("fine"), run.stderr[-2000:]
