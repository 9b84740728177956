"""CPU tests of the layers around the attention: the oracle against torch, the
quantiser, and what the entry points and the binding refuse."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import evo_layers as E
from oracle import evo_memory as M
from paper_2607_20293_amd import evo

INVALID, UNSUPPORTED = -1, -5
A = 0x10000                       # an aligned address; never read: every call below is refused
R = ctypes.byref


def _lib():
    if not os.path.exists(evo.LIB_PATH):
        pytest.skip("library not built")
    return evo.lib()


# ---- oracle ----------------------------------------------------------------
def test_oracle_norms_are_torchs():
    rng = np.random.default_rng(0)
    x, y, g, b = rng.normal(size=(5, 24)), rng.normal(size=(5, 24)), rng.normal(size=24), rng.normal(size=24)
    t = [torch.from_numpy(v) for v in (x, y, g, b)]
    want = torch.nn.functional.layer_norm(t[0], (24,), t[2], t[3], 1e-5).numpy()
    assert np.allclose(E.norm(x, "layer", g, b, 1e-5), want, atol=1e-12)
    want = torch.nn.functional.rms_norm(t[0], (24,), t[2], 1e-5).numpy()
    assert np.allclose(E.norm(x, "rms", g, None, 1e-5), want, atol=1e-12)
    out, h = E.block_norm(x, y, "layer", "rms", None, None, g, None, 2 * np.ones((5, 24)), g[None] + 0 * x, b[None] + 0 * x, 0.5, 1e-5)
    assert np.allclose(out, 0.5 * x + 2 * E.norm(y, "rms", g, None, 1e-5))
    assert np.allclose(h, E.norm(out, "layer", None, None, 1e-5) * (1 + g) + b)
    for act, f in (("silu", torch.nn.functional.silu), ("gelu", torch.nn.functional.gelu), (None, lambda v: v)):
        assert np.allclose(E.activate(x, act), f(t[0]).numpy(), atol=1e-12)


def test_quantiser():
    """Codes and scales are the definition's, at every size a group can have."""
    rng = np.random.default_rng(1)
    m = rng.normal(size=(9, 200)) * np.exp(rng.normal(size=(9, 200)))
    m[0] = 0
    m[1, :32] = 0
    m[2] *= 1e-37
    m[3] *= 1e37
    m[4] = 6.0
    m[5, :7] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, -5]
    m[5, 7:] = 0
    m[6] = np.nextafter(np.float32(6), np.float32(7))
    m[7] = 2.0 ** -149
    m[8] = 3.4e38
    m = m.astype(np.float32)
    codes, scales = evo.Weights4.coded(torch.from_numpy(m))
    assert codes.shape == (9, 128) and scales.shape == (9, 8) and not scales[:, 7].any() and not codes[:, 112:].any()
    want, e = E.quantise(m)
    assert np.array_equal(E.weights4(codes.numpy(), scales.numpy(), 200), want)
    assert np.array_equal(scales.numpy()[want.any(1)], e[want.any(1)])
    assert not codes[0].any()
    for bad in (np.nan, np.inf):
        m[1, 3] = bad
        with pytest.raises(ValueError, match="finite"):
            evo.Weights4.coded(torch.from_numpy(m))
    with pytest.raises(ValueError):
        evo.Weights4.coded(torch.zeros(3))
    with pytest.raises(ValueError):
        evo.Weights4.coded(torch.zeros(3, 3, dtype=torch.int32))
    assert np.array_equal(M.e2m1_of_bytes(np.array([[0x72]], np.uint8), 1), [[1.0, 6.0]])


# ---- refusals --------------------------------------------------------------
def _matrix(**kw):
    d = dict(data=A, row_stride=256)
    d.update(kw)
    return evo.Matrix(**d)


def _linear(L, w=None, dtype=evo.EVO_BF16, n=5, x=None, bias=None, act=0, out=None, **kw):
    d = dict(codes=A, scales=A, n_out=256, n_in=256)
    d.update(kw)
    return L.evo_coded_linear(R(evo.Weights4Desc(**d)), dtype, n, R(x or _matrix()), bias, act, R(out or _matrix()), None)


def test_linear_refuses():
    L = _lib()
    for kw, code, word in [
            (dict(codes=None), INVALID, "NULL"), (dict(scales=None), INVALID, "NULL"), (dict(codes=A + 8), INVALID, "aligned"),
            (dict(n_out=0), INVALID, "weights"), (dict(n_in=-1), INVALID, "weights"), (dict(n_in=(1 << 20) + 1), UNSUPPORTED, "2^20"),
            (dict(n_out=(1 << 20) + 1), UNSUPPORTED, "2^20"), (dict(dtype=2), INVALID, "dtype"), (dict(n=-1), INVALID, "rows"),
            (dict(n=(1 << 20) + 1), UNSUPPORTED, "2^20"), (dict(act=3), INVALID, "activation"), (dict(act=-1), INVALID, "activation"),
            (dict(bias=A + 2), INVALID, "bias"), (dict(x=_matrix(data=None)), INVALID, "x is NULL"),
            (dict(x=_matrix(data=A + 1)), INVALID, "aligned"), (dict(x=_matrix(row_stride=-256)), INVALID, "stride"),
            (dict(out=_matrix(data=None)), INVALID, "out is NULL"), (dict(out=_matrix(row_stride=255)), INVALID, "stride"),
            (dict(out=_matrix(data=A + 2), dtype=evo.EVO_FP32), INVALID, "aligned")]:
        assert _linear(L, **kw) == code and word in L.evo_last_error().decode(), kw
    assert L.evo_coded_linear(None, 1, 1, None, None, 0, None, None) == INVALID
    assert L.evo_coded_linear(R(evo.Weights4Desc(A, A, 4, 4)), 1, 1, None, None, 0, None, None) == INVALID
    assert _linear(L, n=0, x=_matrix(data=None)) == 0      # no rows: nothing to do, nothing read


def _norm(L, n=6, x=None, y=None, x_out=None, h=None, no=(), **kw):
    d = dict(stream_dtype=evo.EVO_BF16, block_dtype=evo.EVO_BF16, d=256, post=1, pre=1, alpha=1.0, eps=1e-6, n_mods=2, gate=_matrix(),
             scale=_matrix(), shift=_matrix())
    d.update(kw)
    t = dict(x=x or _matrix(), y=y or _matrix(), x_out=x_out or _matrix(), h=h or _matrix())
    return L.evo_block_norm(R(evo.BlockNormDesc(**d)), n, *[None if k in no else R(v) for k, v in t.items()], None)


def test_block_norm_refuses():
    L = _lib()
    none = evo.Matrix()
    plain = dict(gate=none, scale=none, shift=none)
    for kw, code, word in [
            (dict(stream_dtype=2), INVALID, "stream_dtype"), (dict(block_dtype=-1), INVALID, "block_dtype"),
            (dict(block_dtype=evo.EVO_FP32), UNSUPPORTED, "bf16"), (dict(d=0), INVALID, "d 0"), (dict(d=16385), UNSUPPORTED, "16384"),
            (dict(post=3), INVALID, "norm"), (dict(pre=-1), INVALID, "norm"), (dict(alpha=float("inf")), INVALID, "alpha"),
            (dict(alpha=float("nan")), INVALID, "alpha"), (dict(eps=-1e-6), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"),
            (dict(eps=float("inf")), INVALID, "eps"), (dict(post=0, post_gain=A), INVALID, "post_gain"),
            (dict(post=0, post_bias=A), INVALID, "post_bias"), (dict(pre=0), INVALID, "scale"),
            (dict(pre=0, pre_gain=A, no=("h",), **plain), INVALID, "pre_gain"), (dict(pre_gain=A + 2), INVALID, "aligned"),
            (dict(n=-1), INVALID, "rows"), (dict(n=1 << 24), UNSUPPORTED, "2^24"), (dict(no=("y",)), INVALID, "without y"),
            (dict(no=("y",), post=0), INVALID, "without y"), (dict(no=("h",)), INVALID, "h is NULL"),
            (dict(pre=0, **plain), INVALID, "h without"), (dict(pre=0, no=("h", "x_out"), **plain), INVALID, "neither"),
            (dict(n_mods=0), INVALID, "n_mods"), (dict(n=5), INVALID, "multiple"), (dict(mod_rows=A, **plain), INVALID, "mod_rows"),
            (dict(mod_rows=A + 2), INVALID, "aligned"), (dict(gate=_matrix(data=A + 1)), INVALID, "gate"),
            (dict(scale=_matrix(row_stride=-1)), INVALID, "scale"), (dict(no=("x",)), INVALID, "x is NULL"),
            (dict(x=_matrix(data=A + 1)), INVALID, "x is not"), (dict(y=_matrix(row_stride=-256)), INVALID, "stride"),
            (dict(x_out=_matrix(row_stride=255)), INVALID, "x_out"), (dict(h=_matrix(row_stride=0)), INVALID, "stride")]:
        assert _norm(L, **kw) == code and word in L.evo_last_error().decode(), (kw, L.evo_last_error())
    assert L.evo_block_norm(None, 1, None, None, None, None, None) == INVALID
    assert _norm(L, n=0, no=("x", "y", "x_out"), post=0, **plain) == 0


# ---- the binding -----------------------------------------------------------
class _Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def library(monkeypatch):
    made = _Library()
    monkeypatch.setattr(evo, "lib", lambda: made)
    monkeypatch.setattr(evo, "_device_of", lambda t: t.device)
    monkeypatch.setattr(evo, "_current_device", lambda: None)
    monkeypatch.setattr(evo, "_current_stream", lambda index: 0)
    return made


def _tensors(dtype=torch.bfloat16):
    x, y, m = (torch.zeros(6, 32, dtype=dtype) for _ in range(3))
    return dict(x=x, y=y, gate=m[:2], scale=m[:2], shift=m[:2], pre_gain=torch.zeros(32), pre_bias=torch.zeros(32),
                post_gain=torch.zeros(32), post_bias=torch.zeros(32), x_out=torch.zeros(6, 32, dtype=dtype),
                h_out=torch.zeros(6, 32, dtype=dtype))


def test_binding_refuses_tensors(library):
    def norm(**kw):
        t = {**_tensors(), **kw}
        return evo.block_norm(t.pop("x"), t.pop("y"), post="rms", **t)
    assert norm()[0].shape == (6, 32)
    for name in _tensors():
        t = _tensors()[name]
        with pytest.raises(TypeError):
            norm(**{name: t.double()})
        with pytest.raises((ValueError, TypeError)):
            norm(**{name: t[..., :31]})
        with pytest.raises(RuntimeError, match=name + ".*gradient"):
            norm(**{name: t.clone().requires_grad_(True)})
        with torch.no_grad():
            norm(**{name: t.clone().requires_grad_(True)})
        if t.dim() == 2:
            with pytest.raises(ValueError, match=name):
                norm(**{name: torch.zeros(*reversed(t.shape), dtype=t.dtype).t()})
    with pytest.raises(ValueError, match="pre and post"):
        norm(pre="batch")
    with pytest.raises(ValueError, match="h_out"):
        norm(pre=None, pre_gain=None, pre_bias=None, scale=None, shift=None)
    with pytest.raises(TypeError):
        norm(mod_rows=torch.zeros(6, dtype=torch.int64))
    with pytest.raises(ValueError):
        evo.block_norm(torch.zeros(6))
    with pytest.raises(TypeError):
        evo.block_norm(torch.zeros(6, 32, dtype=torch.float16))
    with pytest.raises(TypeError):
        evo.block_norm(torch.zeros(6, 32), dtype=torch.float16)


def test_binding_refuses_weights(library):
    codes, scales = torch.zeros(8, 128, dtype=torch.uint8), torch.zeros(8, 8, dtype=torch.uint8)
    w = evo.Weights4(codes, scales, 200)
    x = torch.zeros(3, 200)
    assert evo.linear4(x, w).shape == (3, 8) and evo.linear4(x[:, :], w, torch.zeros(8), "gelu").dtype == torch.float32
    for bad in (dict(n_in=256 + 1), dict(n_in=128), dict(codes=codes[:, :64]), dict(scales=scales[:7]), dict(codes=codes.t())):
        with pytest.raises((ValueError, TypeError)):
            evo.Weights4(**{**dict(codes=codes, scales=scales, n_in=200), **bad})
    for bad in (dict(codes=codes.int()), dict(scales=scales.int()), dict(codes=codes[0])):
        with pytest.raises(TypeError):
            evo.Weights4(**{**dict(codes=codes, scales=scales, n_in=200), **bad})
    for call in (lambda: evo.linear4(x[:, :199], w), lambda: evo.linear4(x.half(), w), lambda: evo.linear4(x[0], w),
                 lambda: evo.linear4(x, w, torch.zeros(7)), lambda: evo.linear4(x, w, torch.zeros(8).double()),
                 lambda: evo.linear4(x, w, activation="relu"), lambda: evo.linear4(x, w, out=torch.zeros(3, 9)),
                 lambda: evo.linear4(x, w, out=torch.zeros(3, 8).bfloat16()), lambda: evo.linear4(torch.zeros(200, 3).t(), w)):
        with pytest.raises((ValueError, TypeError)):
            call()
    for kw in (dict(x=x.clone().requires_grad_(True)), dict(bias=torch.zeros(8, requires_grad=True))):
        with pytest.raises(RuntimeError, match="gradient"):
            evo.linear4(kw.get("x", x), w, kw.get("bias"))


def test_weights_values_and_host_tensors():
    m = torch.randn(7, 150, generator=torch.Generator().manual_seed(0))
    with pytest.raises(TypeError):
        evo.Weights4.of(m)
    codes, scales = evo.Weights4.coded(m)
    w = evo.Weights4.__new__(evo.Weights4)
    w.codes, w.scales, w.n_in = codes, scales, 150
    assert np.array_equal(w.values().double().numpy(), E.weights4(codes.numpy(), scales.numpy(), 150))
    assert float((w.values() - m).abs().max()) <= float(m.abs().max()) / 3


def test_block_norm_rows_of_a_launch():
    """A launch has fewer than 2^32 threads, up to 1024 for a row."""
    L = _lib()
    plain = dict(gate=evo.Matrix(), scale=evo.Matrix(), shift=evo.Matrix())
    wide = _matrix(row_stride=16384)
    for d, n in ((2049, 1 << 23), (4096, 1 << 23), (4097, 1 << 22), (16384, 1 << 22)):
        assert _norm(L, n=n, d=d, x=wide, y=wide, x_out=wide, h=wide, **plain) == UNSUPPORTED
        assert f"up to {n - 1}" in L.evo_last_error().decode()
