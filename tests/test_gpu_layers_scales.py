"""Products with 4-bit weights whose scales lie at the ends of their range, against
the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2607_20293_amd import evo
from tests.gpu_util import device, say
from tests.layers_util import check, linear_reference, random_weights

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
INF = float("inf")
SIZES = [(3, 256, 48), (3, 8192, 48), (64, 1000, 700), (200, 256, 300), (600, 520, 2000)]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,n_in,n_out", SIZES)
def test_least_scales(rows, n_in, n_out, dtype):
    """2^-127 and its neighbours, the least weight 2^-128: rows around 2^100 bring the
    products to ordinary sizes, so that a weight that counts as 0 is seen.  The bound's
    part for results below the normal floats, 1e-37, is far below them."""
    dev, gen = device(), torch.Generator().manual_seed(rows)
    say(f"[gpu] linear4 {dtype} rows {rows} {n_in} -> {n_out}, least scales")
    w = random_weights(n_out, n_in, gen, dev)
    for byte in (0, 1, 2):
        w.scales[byte::4, :-(-n_in // 32)] = byte
    w.codes[4 % n_out] &= 0x11                              # 0 and the least code alone, of scale 0
    x = (torch.randn((rows, n_in), generator=gen) * 2.0 ** 100).to(dtype).to(dev)
    want, bound = linear_reference(x, w, None, None, dtype)
    tiny = np.arange(n_out) % 4 < 3
    assert np.median(np.abs(want[:, tiny])) > 1e-9
    check(evo.linear4(x, w), want, bound, "least scales")


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,n_in,n_out", SIZES)
def test_largest_scales(rows, n_in, n_out, dtype):
    """Weights up to the largest floats (1.5 * 2^127), of the scales 2^125 to 2^127; a
    weight of 2^128 or more is an infinity of its sign."""
    dev, gen = device(), torch.Generator().manual_seed(rows + 1)
    say(f"[gpu] linear4 {dtype} rows {rows} {n_in} -> {n_out}, largest scales")
    w = random_weights(n_out, n_in, gen, dev)
    groups = -(-n_in // 32)
    w.scales[0::3, :groups] = 252
    w.scales[1::3, :groups] = 253
    w.scales[2::3, :groups] = 254
    w.codes[1::3] &= 0xdd                                   # up to 3
    w.codes[2::3] &= 0xbb                                   # up to 1.5
    x = (torch.randn((rows, n_in), generator=gen) * 2.0 ** -100).to(dtype).to(dev)
    # sums of magnitudes up to 2^135 / 2^100 of x: no result outgrows the floats
    check(evo.linear4(x, w), *linear_reference(x, w, None, None, dtype), "largest scales")
    over = evo.Weights4(torch.zeros_like(w.codes), torch.full_like(w.scales, 254), n_in)
    over.scales[:, groups:] = 0
    for n, code in ((0, 7), (1, 15), (2, 4), (3, 12), (4, 3), (5, 11)):
        over.codes[n, 5] = code << 4                        # weight 11 of row n: 6, -6, 2, -2, 1.5, -1.5
    x[:, 11] = 2.0 ** -100
    got = evo.linear4(x, over).double().cpu()
    assert torch.equal(got[:, :4], torch.tensor([INF, -INF, INF, -INF], dtype=torch.float64).expand(rows, 4))
    assert torch.equal(got[:, 4:6], torch.tensor([1.5, -1.5], dtype=torch.float64).expand(rows, 2) * 2.0 ** 27)
    assert not got[:, 6:].any()
    assert torch.equal(over.values()[:6, 11].cpu(), torch.tensor([INF, -INF, INF, -INF, 1.5 * 2.0 ** 127, -1.5 * 2.0 ** 127]))
