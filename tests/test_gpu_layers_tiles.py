"""Products with 4-bit weights at sizes of which tests/test_layers_plan.py checks that
they reach every kernel, in every state of its last tiles and chunks, against the
definition in 64 bits."""
import pytest
import torch

from paper_2607_20293_amd import evo
from tests.gpu_util import device, say
from tests.layers_util import check, linear_reference, random_weights

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")

SIZES = {  # rows, n_in, n_out
    BF16: [(300, 333, 40), (90, 1500, 2101), (64, 4096, 4096), (64, 3970, 4100), (33, 1590, 6300), (30, 2213, 7750), (33, 1335, 7091),
           (2144, 1884, 109), (300, 8192, 8192), (126, 136, 8162), (147, 265, 4740), (1945, 392, 4516), (130, 419, 6786),
           (2079, 547, 385), (1008, 333, 1990), (598, 406, 6725), (2060, 300, 4100)],
    FP32: [(3, 333, 40), (90, 700, 9001), (1950, 391, 493), (1857, 524, 486), (1439, 408, 3442), (1606, 536, 3592), (342, 132, 7622), (2060, 300, 4100)]}


def _call(dtype, rows, n_in, n_out):
    dev, gen = device(), torch.Generator().manual_seed(rows + n_out)
    say(f"[gpu] linear4 {dtype} rows {rows} {n_in} -> {n_out}: {evo.linear_plan(dtype, rows, n_in, n_out)[1].tolist()}")
    x = torch.randn((rows, n_in), generator=gen).to(dtype).to(dev)
    return x, random_weights(n_out, n_in, gen, dev), torch.randn(n_out, generator=gen).to(dev), dev


@pytest.mark.parametrize("dtype,sizes", [(t, s) for t in SIZES for s in SIZES[t]])
def test_linear_tiles(dtype, sizes):
    """Rows and outputs at odd strides; what lies around out keeps its value."""
    rows, n_in, n_out = sizes
    x, w, bias, dev = _call(dtype, *sizes)
    want, bound = linear_reference(x, w, bias, "silu", dtype)
    check(evo.linear4(x, w, bias, "silu"), want, bound, "whole")
    xv = torch.full((rows, n_in + 3), NAN, dtype=dtype, device=dev)[:, 1:n_in + 1]
    xv.copy_(x)
    base = torch.full((rows + 1, n_out + 5), 7.0, dtype=dtype, device=dev)
    check(evo.linear4(xv, w, bias, "silu", out=base[:rows, 2:n_out + 2]), want, bound, "strides")
    assert bool((base[rows] == 7).all()) and bool((base[:, :2] == 7).all()) and bool((base[:, n_out + 2:] == 7).all())


@pytest.mark.parametrize("dtype,sizes", [(t, s) for t in SIZES for s in SIZES[t]])
def test_linear_rows_of_every_tile_do_not_meet(dtype, sizes):
    """A NaN and an infinity stay in their row, a weight that is a NaN in its column."""
    rows, n_in, n_out = sizes
    x, w, _, dev = _call(dtype, *sizes)
    clean = evo.linear4(x, w)
    assert torch.equal(evo.linear4(x, w), clean)
    for bad in (0, rows // 2, rows - 1):
        dirty = x.clone()
        dirty[bad, n_in - 1], dirty[bad, 0] = NAN, INF
        got = evo.linear4(dirty, w)
        keep = torch.arange(rows, device=dev) != bad
        assert torch.equal(got[keep], clean[keep]) and bool(torch.isnan(got[bad]).all())
    for bad, group in ((0, 0), (n_out // 2, n_in // 64), (n_out - 1, (n_in - 1) // 32)):
        held = int(w.scales[bad, group])
        w.scales[bad, group] = 255
        got = evo.linear4(x, w)
        w.scales[bad, group] = held
        keep = torch.arange(n_out, device=dev) != bad
        assert torch.equal(got[:, keep], clean[:, keep]) and bool(torch.isnan(got[:, bad]).all())
