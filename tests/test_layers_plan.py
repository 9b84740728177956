"""CPU tests of how products with 4-bit weights are divided between their kernels:
that the sizes of the GPU tests reach all of them, and what the query refuses."""
import os

import numpy as np
import pytest
import torch

from paper_2607_20293_amd import evo
from tests.test_gpu_layers_tiles import SIZES

BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def built():
    if not os.path.exists(evo.LIB_PATH):
        pytest.skip("library not built")


@pytest.mark.parametrize("dtype,after", [(BF16, {1, 2, 3}), (FP32, {1, 2})])
def test_the_sizes_of_the_tests_reach_every_kernel(dtype, after):
    """Every kernel; of those that stage chunks in LDS, tiles with rows and weight rows
    past the end, and every number of chunks in the last stage; and launches for the
    rows after whole rounds (`after`: kernels that take them)."""
    first, rest, ragged, chunks, parts = set(), set(), set(), set(), {}
    for rows, n_in, n_out in SIZES[dtype]:
        kinds, launches = evo.linear_plan(dtype, rows, n_in, n_out)
        assert sum(n for _, n, _, _, _ in launches) == rows
        for i, (kind, n, tile, wide, k) in enumerate(launches):
            (rest if i else first).add(int(kind))
            parts[int(kind)] = int(k)
            if n % tile and n_out % wide:
                ragged.add(int(kind))
            chunks.add((int(kind), -(-n_in // 128) % int(k)))
    assert first == set(range(kinds)) and ragged == first
    for kind, k in parts.items():
        if 1 < k < 8:
            assert {(kind, c) for c in range(k)} <= chunks, kind
    assert rest >= after, rest


def test_plans_cover_the_rows():
    rng = np.random.default_rng(0)
    for dtype in (BF16, FP32):
        for _ in range(500):
            rows, n_in, n_out = (int(2 ** rng.uniform(0, 20)) for _ in range(3))
            kinds, launches = evo.linear_plan(dtype, rows, n_in, n_out, int(rng.integers(1, 400)))
            assert 1 <= len(launches) <= 2 and sum(launches[:, 1]) == rows and (launches[:, 1] > 0).all()
            assert ((0 <= launches[:, 0]) & (launches[:, 0] < kinds)).all()


def test_the_plan_refuses():
    for args in ((BF16, 0, 8, 8), (BF16, -1, 8, 8), (BF16, 8, 0, 8), (BF16, 8, 8, 0), (FP32, 8, 8, 8, 0), (FP32, (1 << 20) + 1, 8, 8),
                 (FP32, 8, (1 << 20) + 1, 8), (FP32, 8, 8, (1 << 20) + 1)):
        with pytest.raises(RuntimeError):
            evo.linear_plan(*args)
    assert evo.lib().evo_debug_linear_plan(2, 8, 8, 8, 256, None) == -1
    assert evo.lib().evo_debug_linear_plan(evo.EVO_BF16, 8, 8, 8, 256, None) == -1
