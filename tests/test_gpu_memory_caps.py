"""GPU parity of chunk attention with caps of any size."""
import numpy as np
import pytest

from oracle import evo_memory as M
from tests.gpu_util import device, say
from tests.memory_util import EPS16, EPS32, Call, f64

pytestmark = pytest.mark.gpu


def _check_capped(c, cap):
    """Every step of a score (product, scale, quotient by the cap, tanh, cap,
    base 2) rounds relative to the score itself, whatever the cap: dh products
    summed in fp32, 16 more roundings, doubled, and 4 of the distance.  Up to
    caps of 64, bf16 calls may be off by 2^-22 of the cap as well."""
    k, v, ks, vs = c.tensors
    arr = [f64(k), f64(v)] + [None if s is None else f64(s) for s in (ks, vs)]
    out, lse = (f64(t) for t in c.run())
    q, dh = f64(c.q), c.dh
    slopes = None if c.slopes is None else c.slopes.double().numpy()
    for s, (n, length) in enumerate(zip(c.rows, c.lengths)):
        kk, vv = M.gather(*arr, c.tab, s, length)
        x = q[c.cu[s]:c.cu[s + 1]]
        want, want_lse = M.attend(x, kk, vv, length - n, dh ** -0.5, c.kw.get("causal", False), 0, cap, slopes)
        products = np.max(np.abs(x)) * np.max(np.sum(np.abs(kk), -1)) * dh ** -0.5
        far = 0 if slopes is None else np.max(slopes) * length
        dz = 2 * EPS32 * ((dh + 16) * min(products, 1e30) + 4 * far) + (2.0 ** -22 * cap if c.dtype == "bf16" and cap <= 64 else 0)
        top = np.max(np.abs(vv))
        err = np.max(np.abs(out[c.cu[s]:c.cu[s + 1]] - want))
        err_l = np.max(np.abs(lse[c.cu[s]:c.cu[s + 1]] - want_lse))
        bound = top * (4 * (dz + (length + 64) * EPS32) + (EPS16 * 1.01 if c.dtype == "bf16" else 0))
        bound_l = 2 * dz + (length + 64) * EPS32 + 1e-6 + 4 * EPS32 * products
        print(f"  cap {cap:g}: out {err / bound:.3f}, lse {err_l / bound_l:.3f} of their bounds", flush=True)
        assert err <= bound and err_l <= bound_l, cap


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype,fmt,rows,lengths,dh", [
    ("bf16", "bf16", [7, 3], [300, 90], 64), ("bf16", "int8", [20], [200], 32), ("bf16", "fp8", [3], [700], 128),
    ("fp32", "fp32", [9], [150], 64), ("fp32", "fp8", [4], [100], 64),
    ("bf16", "bf16", [100, 30], [260, 70], 64), ("bf16", "fp8", [130], [200], 128)])
def test_any_cap(dtype, fmt, rows, lengths, dh, bias):
    """A cap far above the scores changes nothing, a tiny one leaves the mean
    (or the distances alone)."""
    say(f"[gpu] caps {dtype} over {fmt}: rows {rows} lengths {lengths} dh {dh} bias {bias}")
    for cap in (1e-41, 1e-20, 3.0, 64.0, 65.0, 1e3, 1e5, 1e6, 1e8, 1e30, 3e38):
        c = Call(device(), dtype, fmt, rows, lengths, 2, 2, dh, seed=21, causal=True, bias=bias, cap=cap)
        _check_capped(c, cap)
