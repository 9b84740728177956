"""Sizes of products with 4-bit weights and of norms around a block that reach every
kernel they are divided between, against the definition in 64 bits."""
import pytest
import torch

from paper_2607_20293_amd import evo
from tests.gpu_util import device, say
from tests.layers_util import NormCall, check, linear_reference, random_weights

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")

SHAPES = [  # rows, n_in, n_out: tiles of 16 rows up to 128 by 256, ragged and with rows that go after whole rounds
    (300, 3, 40), (40, 7, 300), (90, 6, 20000), (64, 4096, 1100), (100, 3000, 4100), (300, 1000, 2300), (700, 520, 1500),
    (600, 260, 2000), (2049, 1000, 1030), (1030, 1030, 4100), (2060, 300, 4100), (4099, 256, 2050)]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_linear_shapes(dtype, rows, n_in, n_out):
    """Rows and outputs at odd strides; what lies around out keeps its value."""
    dev, gen = device(), torch.Generator().manual_seed(rows + n_out)
    say(f"[gpu] linear4 {dtype} rows {rows} {n_in} -> {n_out}")
    w = random_weights(n_out, n_in, gen, dev)
    x = torch.randn((rows, n_in), generator=gen).to(dtype).to(dev)
    bias = torch.randn(n_out, generator=gen).to(dev)
    want, bound = linear_reference(x, w, bias, "gelu", dtype)
    check(evo.linear4(x, w, bias, "gelu"), want, bound, "whole")
    xv = torch.full((rows, n_in + 3), NAN, dtype=dtype, device=dev)[:, 1:n_in + 1]
    xv.copy_(x)
    base = torch.full((rows + 1, n_out + 5), 7.0, dtype=dtype, device=dev)
    check(evo.linear4(xv, w, bias, "gelu", out=base[:rows, 2:n_out + 2]), want, bound, "strides")
    assert bool((base[rows] == 7).all()) and bool((base[:, :2] == 7).all()) and bool((base[:, n_out + 2:] == 7).all())


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,n_in,n_out", [(100, 3000, 4100), (700, 520, 1500), (1030, 1030, 4100), (2060, 300, 4100)])
def test_linear_rows_of_tiles_do_not_meet(dtype, rows, n_in, n_out):
    dev, gen = device(), torch.Generator().manual_seed(3)
    w = random_weights(n_out, n_in, gen, dev)
    x = torch.randn((rows, n_in), generator=gen).to(dtype).to(dev)
    clean = evo.linear4(x, w)
    assert torch.equal(evo.linear4(x, w), clean)
    for bad in (0, rows // 2, rows - 1):
        dirty = x.clone()
        dirty[bad, n_in - 1], dirty[bad, 0] = NAN, INF
        got = evo.linear4(dirty, w)
        keep = torch.arange(rows, device=dev) != bad
        assert torch.equal(got[keep], clean[keep]) and bool(torch.isnan(got[bad]).all())


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_activations_of_extreme_values(dtype):
    """GELU and SiLU of 0, small and large values of either sign, infinities and NaN: one
    weight of 1 passes the rows through."""
    dev = device()
    n = 160
    codes = torch.zeros((1, 64), dtype=torch.uint8, device=dev)
    codes[0, 0] = 2                                       # the value 1
    scales = torch.full((1, 4), 127, dtype=torch.uint8, device=dev)
    w = evo.Weights4(codes, scales, 1)
    x = torch.cat([torch.linspace(-20, 20, n - 9), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 80.0, -80.0, 3e38, INF, NAN])])
    x = x[:, None].to(dtype).to(dev)
    for act in ("silu", "gelu"):
        got, y = evo.linear4(x, w, None, act).double().cpu()[:, 0], x.double().cpu()[:, 0]
        want = y * torch.sigmoid(y) if act == "silu" else y * (0.5 * torch.special.erfc(y * -0.5 ** 0.5))
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and got[-2] == INF
        # fp32: the exponential's and a few more roundings (16, of 2^-24), values below the normal floats lost;
        # bf16: half a step, a hundredth of it for the fit and the fast functions, and from -13 on, where GELU is
        # below 1e-37, what is lost below the normal floats
        fine = torch.isfinite(want)
        rel = 16 * 2.0 ** -24 if dtype == FP32 else 1.01 * 2.0 ** -8
        if act == "gelu" and dtype == FP32:
            # erfc(z) of a rounded z: relative 2 z^2 = x^2 roundings, and the function's own few
            rel = rel + y.abs().clamp(max=20) ** 2 * 2.0 ** -23
        if act == "gelu" and dtype == BF16:
            rel = rel + y.abs().clamp(max=20) ** 2 * 2.0 ** -23
        if act == "silu":
            rel = rel + y.abs().clamp(max=90) * 2.0 ** -23    # the exponential of a rounded argument
        err = (got - want).abs()
        limit = (rel * want.abs() + 1.2e-38 * 2)
        assert bool((err[fine] <= limit[fine]).all()), (act, y[fine][err[fine] > limit[fine]], err[fine][err[fine] > limit[fine]])


NORMS = [(3, 1000), (1501, 1024), (1600, 700), (5, 2049), (40, 4096), (7, 4097), (1800, 5120), (3, 8192), (2, 8193), (9, 16384),
         (300, 12000)]


@pytest.mark.parametrize("rows,d", NORMS)
@pytest.mark.parametrize("stream,block", [(BF16, BF16), (FP32, BF16), (FP32, FP32)])
def test_block_norm_widths(stream, block, rows, d):
    """Rows over a part of a wave up to sixteen waves."""
    for pre, post in (("rms", "layer"), ("layer", "rms")):
        call = NormCall(device(), stream, block, rows, d, pre=pre, post=post, mods=1, seed=d)
        call.check(f"{rows} x {d}, {pre} after {post}")


def test_block_norm_of_no_rows():
    """No rows give none; a modulation of none for some rows is refused."""
    dev = device()
    x, none = torch.randn((4, 64), device=dev), torch.empty((0, 64), device=dev)
    for kw in (dict(y=x, gate=none), dict(scale=none), dict(shift=none)):
        with pytest.raises(ValueError):
            evo.block_norm(x, **kw)
    out, h = evo.block_norm(none, none, gate=x[:1], scale=x[:1])
    assert out.shape == h.shape == (0, 64)
    w = random_weights(16, 64, torch.Generator().manual_seed(1), dev)
    assert evo.linear4(none, w).shape == (0, 16)
