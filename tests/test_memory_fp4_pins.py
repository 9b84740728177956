"""CPU tests of the 4-bit cache: the oracle's 4-bit floats, and what the entry
points refuse."""
import numpy as np
import pytest
import torch

from oracle import evo_memory as M
from paper_2607_20293_amd import evo
from tests.test_memory_pins import A, INVALID, UNSUPPORTED, _attend, _cache, _lib, _qkv, _read, _write

FP4 = torch.float4_e2m1fn_x2


def test_4_bit_floats():
    """All sixteen, the nearest of each value between, ties to the even code."""
    grid = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    b = np.arange(256).reshape(16, 16)
    v = M.e2m1_of_bytes(b, 1)
    signed = np.concatenate([grid, -grid])
    assert np.array_equal(v[:, 0::2], signed[b % 16]) and np.array_equal(v[:, 1::2], signed[b // 16])
    assert np.array_equal(M.e2m1_of_bytes(b.T, 0), v.T)
    y = np.concatenate([np.linspace(-6, 6, 4801), (grid[1:] + grid[:-1]) / 2, -(grid[1:] + grid[:-1]) / 2])
    for x, got in zip(y, M.e2m1(y)):
        far = np.abs(grid - abs(x))
        near = np.nonzero(far == far.min())[0]
        want = grid[near[0] if len(near) == 1 else near[near % 2 == 0][0]]
        assert abs(got) == want and (got == 0 or np.sign(got) == np.sign(x)), x


@pytest.mark.parametrize("call", [_write, _read, _qkv, _attend])
def test_refuses_bad_4_bit_caches(call):
    L = _lib()
    for kw, code, word in [(dict(), INVALID, "k_scale"), (dict(k_scale=A), INVALID, "k_scale"),
                           (dict(k_scale=A, v_scale=A + 8), INVALID, "aligned"), (dict(k=A + 4, k_scale=A, v_scale=A), INVALID, "aligned"),
                           (dict(k_scale=A, v_scale=A, head_dim=48), UNSUPPORTED, "head_dim"),
                           (dict(k_scale=A, v_scale=A, page_size=32), UNSUPPORTED, "page_size")]:
        assert call(L, cache=_cache(format=evo.CACHE_FP4, **kw)) == code and word in L.evo_last_error().decode(), kw
    for fmt in (4, 6):
        assert call(L, cache=_cache(format=fmt, k_scale=A, v_scale=A)) == INVALID


def test_4_bit_caches_take_both_types_of_rows():
    """Refused for another reason than their type."""
    L = _lib()
    for dtype in (evo.EVO_FP32, evo.EVO_BF16):
        cache = _cache(format=evo.CACHE_FP4, k_scale=A, v_scale=A)
        assert _write(L, cache=cache, dtype=dtype, starts=None) == INVALID and "starts" in L.evo_last_error().decode()


def test_binding_refuses_4_bit_caches():
    with pytest.raises(ValueError, match="whole elements"):
        evo.KVCache.empty(2, 2, 33, 64, FP4, "cpu")
    with pytest.raises(TypeError):
        evo.KVCache.empty(2, 2, 32, 64, FP4, "cpu")
