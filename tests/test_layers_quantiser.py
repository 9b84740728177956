"""CPU tests of weights of 64 bits on their way to 4: what 32 bits cannot hold."""
import pytest
import torch

from paper_2607_20293_amd import evo


@pytest.mark.parametrize("value", [1e39, -1e39, 3.4028236e38, 1.7e308])
def test_weights_beyond_32_bits_are_refused(value):
    """Finite in 64 bits, infinite in 32."""
    w = torch.ones((2, 40), dtype=torch.float64)
    w[1, 35] = value
    with pytest.raises(ValueError, match="finite"):
        evo.Weights4.coded(w)


def test_the_largest_weights_of_32_bits():
    """They are above the codes' range (6 * 2^125) and become its end."""
    top = torch.finfo(torch.float32).max
    for dtype in (torch.float32, torch.float64):
        codes, scales = evo.Weights4.coded(torch.tensor([[top, -top, 6 * 2.0 ** 125, 2.0 ** 125]], dtype=dtype))
        assert codes[0, :2].tolist() == [0xf7, 0x27] and scales[0].tolist() == [252, 0, 0, 0]
