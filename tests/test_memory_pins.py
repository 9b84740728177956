"""CPU tests of the long memories: the oracle against independent routines, and
what the entry points refuse (arguments are checked before any device work, so
no GPU is needed)."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import evo_memory as M
from paper_2607_20293_amd import evo


def _lib():
    if not os.path.exists(evo.LIB_PATH):
        pytest.skip("libevo.so not built (run __graft_entry__.build())")
    return evo.lib()


# ---- the oracle ------------------------------------------------------------
@pytest.mark.parametrize("pairs", ["halves", "adjacent"])
def test_rotation_keeps_lengths_and_depends_on_distance(pairs):
    rng = np.random.default_rng(0)
    t = M.rope_table(64, 16)
    q, k = rng.normal(size=(1, 1, 32)), rng.normal(size=(1, 1, 32))

    def dot(i, j):
        a = M.norm_rope(q, None, t, np.array([i]), pairs, None)
        b = M.norm_rope(k, None, t, np.array([j]), pairs, None)
        assert np.isclose(np.linalg.norm(a), np.linalg.norm(q))
        assert np.array_equal(a[..., 16:], q[..., 16:])
        return float(np.sum(a * b))
    assert np.isclose(dot(5, 9), dot(25, 29))
    assert np.isclose(dot(0, 0), float(np.sum(q * k)))
    assert not np.isclose(dot(5, 9), dot(5, 19))


def test_norm_matches_torch():
    rng = np.random.default_rng(1)
    x, g = rng.normal(size=(3, 2, 32)), rng.normal(size=32)
    want = torch.nn.functional.rms_norm(torch.from_numpy(x), (32,), torch.from_numpy(g), 1e-6).numpy()
    assert np.allclose(M.norm_rope(x, g, None, None, "halves", 1e-6), want, rtol=1e-12)


def test_e4m3_matches_torch():
    y = np.concatenate([np.linspace(-448, 448, 30001), 2.0 ** np.linspace(-14, 8.8, 5000), [0.0, 2.0 ** -10, 3 * 2.0 ** -10]])
    y = y.astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(M.e4m3(y), want)


def test_quantise_within_half_a_step():
    rng = np.random.default_rng(2)
    x = rng.normal(size=(50, 64)) * np.exp(rng.normal(size=(50, 1)) * 3)
    x[7] = 0
    c, s = M.quantise(x, "int8")
    assert np.array_equal(c, np.rint(c)) and np.max(np.abs(c)) == 127 and s[7] == 0 and not c[7].any()
    assert np.all(np.abs(c * s[:, None] - x) <= s[:, None] * 0.5 * (1 + 1e-12))
    x[3, 5] = np.nan
    x[4, 5] = np.inf
    for fmt in ("int8", "fp8"):
        c, s = M.quantise(x, fmt)
        assert np.isnan(s[3]) and np.isnan(s[4]) and np.isfinite(s[5]) and np.isfinite(c).all()


@pytest.mark.parametrize("causal", [False, True])
def test_attend_matches_torch(causal):
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(5, 4, 32)), rng.normal(size=(9, 2, 32)), rng.normal(size=(9, 2, 32))
    out, lse = M.attend(q, k, v, 4, 0.2, causal=causal)
    t = [torch.from_numpy(np.repeat(a, r, 1)).transpose(0, 1) for a, r in ((q, 1), (k, 2), (v, 2))]
    mask = torch.from_numpy(np.arange(9)[None] <= np.arange(4, 9)[:, None]) if causal else None
    want = torch.nn.functional.scaled_dot_product_attention(*t, attn_mask=mask, scale=0.2).transpose(0, 1).numpy()
    assert np.allclose(out, want, rtol=1e-10)
    z = torch.matmul(t[0], t[1].transpose(1, 2)) * 0.2
    z = z if mask is None else z.masked_fill(~mask, -np.inf)
    assert np.allclose(lse, torch.logsumexp(z, -1).T.numpy(), rtol=1e-10)


def test_attend_masks_cap_and_bias():
    rng = np.random.default_rng(4)
    q, k, v = rng.normal(size=(4, 1, 32)), rng.normal(size=(10, 1, 32)), rng.normal(size=(10, 1, 32))
    # window and prefix, by listing what each row sees
    out, _ = M.attend(q, k, v, 6, 1.0, causal=True, window=2, prefix=1)
    for i in range(4):
        see = [0, 5 + i, 6 + i]
        w = np.exp(k[see, 0] @ q[i, 0])
        assert np.allclose(out[i, 0], w @ v[see, 0] / w.sum())
    # nothing visible
    out, lse = M.attend(q, k, v, -3, 1.0, causal=True)
    assert not out[:3].any() and np.all(np.isneginf(lse[:3])) and np.allclose(out[3, 0], v[0, 0])
    # a cap far above the scores changes nothing, a small one flattens
    a = M.attend(q, k, v, 6, 0.1, cap=1e6)[0]
    assert np.allclose(a, M.attend(q, k, v, 6, 0.1)[0], atol=1e-8)
    assert np.allclose(M.attend(q, k, v, 6, 1.0, cap=1e-9)[0], v.mean(0)[None], atol=1e-7)
    # a steep bias leaves the row's own position
    a = M.attend(q, k, v, 6, 0.1, slopes=np.array([1e3]))[0]
    assert np.allclose(a[:, 0], v[6:, 0])


# ---- what the entry points refuse ------------------------------------------
A = 0x10000                       # an aligned address; never read: every call below is refused


def _cache(**kw):
    d = dict(k=A, v=A, k_scale=None, v_scale=None, format=evo.CACHE_BF16, n_pages=4, page_size=64, n_kv_heads=2,
             head_dim=64)
    d.update(kw)
    return evo.KVCacheDesc(**d)


def _rows(**kw):
    d = dict(n_seqs=2, n_rows=6, max_rows=3, max_pages=2, cu_rows=None, page_table=A)
    d.update(kw)
    return evo.KVRows(**d)


def _nr(**kw):
    d = dict(rotary_dim=64, pairs=0, n_positions=100, eps=1e-6, q_gain=None, k_gain=None, table=A)
    d.update(kw)
    return evo.NormRope(**d)


def _att(**kw):
    d = dict(dtype=evo.EVO_BF16, n_heads=4, causal=0, window=0, max_length=0, scale=0.125, cap=0.0, lengths=A, starts=None,
             prefix=None, slopes=None)
    d.update(kw)
    return evo.Attention(**d)


def _heads(**kw):
    d = dict(data=A, row_stride=256, head_stride=64)
    d.update(kw)
    return evo.Heads(**d)


R = ctypes.byref


def _write(L, cache=None, rows=None, dtype=evo.EVO_BF16, starts=A, k=None, v=None):
    return L.evo_cache_write(R(cache or _cache()), R(rows or _rows()), dtype, starts, R(k or _heads()), R(v or _heads()), None)


def _read(L, cache=None, rows=None, dtype=evo.EVO_BF16, starts=A, k=None, v=None):
    return L.evo_cache_read(R(cache or _cache()), R(rows or _rows()), dtype, starts, R(k or _heads()), R(v or _heads()), None)


def _qkv(L, cache=None, rows=None, nr=None, dtype=evo.EVO_BF16, n_heads=4, starts=A, q=None, q_out=None):
    return L.evo_qkv_write(R(cache or _cache()), R(rows or _rows()), R(nr or _nr()), dtype, n_heads, starts, R(q or _heads()),
                           R(_heads()), R(_heads()), R(q_out or _heads()), None)


def _rope(L, nr=None, dtype=evo.EVO_BF16, dh=64, n=5, hq=4, hk=2, q=None, positions=A, k_out=None):
    return L.evo_qk_norm_rope(R(nr or _nr()), dtype, dh, n, hq, hk, R(q or _heads()), R(_heads()), positions, R(_heads()),
                              R(k_out or _heads()), None)


def _attend(L, cache=None, rows=None, att=None, q=None, out=None, work=A, size=1 << 40):
    return L.evo_chunk_attention(R(cache or _cache()), R(rows or _rows()), R(att or _att()), R(q or _heads()),
                                 R(out or _heads()), None, work, size, None)


INVALID, UNSUPPORTED = -1, -5

BAD_CACHE = [(dict(k=None), INVALID, "NULL"), (dict(v=None), INVALID, "NULL"), (dict(format=4), INVALID, "format"),
             (dict(format=-1), INVALID, "format"), (dict(format=evo.CACHE_INT8), INVALID, "k_scale"),
             (dict(format=evo.CACHE_FP8, k_scale=A), INVALID, "k_scale"), (dict(k=A + 2), INVALID, "aligned"),
             (dict(format=evo.CACHE_INT8, k_scale=A, v_scale=A + 4), INVALID, "aligned"),
             (dict(page_size=0), INVALID, "page_size"), (dict(page_size=32), UNSUPPORTED, "page_size"),
             (dict(page_size=96), UNSUPPORTED, "page_size"), (dict(page_size=2048), UNSUPPORTED, "page_size"),
             (dict(n_pages=0), INVALID, "pages"), (dict(n_kv_heads=0), INVALID, "heads"),
             (dict(head_dim=0), INVALID, "head_dim"), (dict(head_dim=80), UNSUPPORTED, "head_dim")]
BAD_ROWS = [(dict(n_seqs=0), INVALID, "sequences"), (dict(n_rows=-1), INVALID, "rows"), (dict(max_pages=0), INVALID, "pages"),
            (dict(n_rows=5), INVALID, "cu_rows"), (dict(n_rows=7, cu_rows=A), INVALID, "fit"),
            (dict(page_table=None), INVALID, "page_table"), (dict(max_pages=1 << 26), UNSUPPORTED, "2^30"),
            (dict(n_seqs=1 << 15, max_rows=1 << 16, n_rows=1 << 30, cu_rows=A), UNSUPPORTED, "2^31")]


@pytest.mark.parametrize("call", [_write, _read, _qkv, _attend])
def test_refuses_bad_caches_and_rows(call):
    L = _lib()
    for kw, code, word in BAD_CACHE:
        assert call(L, cache=_cache(**kw)) == code and word in L.evo_last_error().decode(), kw
    for kw, code, word in BAD_ROWS:
        assert call(L, rows=_rows(**kw)) == code and word in L.evo_last_error().decode(), kw


@pytest.mark.parametrize("call", [_write, _read, _qkv])
def test_refuses_types_and_missing_starts(call):
    L = _lib()
    assert call(L, dtype=2) == INVALID and "dtype" in L.evo_last_error().decode()
    assert call(L, dtype=evo.EVO_FP32) == UNSUPPORTED and "bf16 cache" in L.evo_last_error().decode()
    assert call(L, cache=_cache(format=evo.CACHE_FP32)) == UNSUPPORTED
    assert call(L, starts=None) == INVALID and "starts" in L.evo_last_error().decode()


def test_refuses_bad_tensors():
    L = _lib()
    for bad in (dict(data=None), dict(data=A + 1), dict(row_stride=-64)):
        assert _write(L, k=_heads(**bad)) == INVALID
        assert _write(L, v=_heads(**bad)) == INVALID
        assert _read(L, k=_heads(**bad)) == INVALID
        assert _qkv(L, q=_heads(**bad)) == INVALID
        assert _rope(L, q=_heads(**bad)) == INVALID
        assert _attend(L, q=_heads(**bad)) == INVALID
    # outputs may not fold rows or heads onto each other
    for bad in (dict(row_stride=32), dict(head_stride=0)):
        assert _read(L, v=_heads(**bad)) == INVALID
        assert _qkv(L, q_out=_heads(**bad)) == INVALID
        assert _rope(L, k_out=_heads(**bad)) == INVALID
        assert _attend(L, out=_heads(**bad)) == INVALID


def test_refuses_bad_norm_rope():
    L = _lib()
    for kw in (dict(rotary_dim=-16), dict(rotary_dim=24), dict(rotary_dim=80), dict(pairs=2), dict(table=None),
               dict(n_positions=0), dict(table=A + 8), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert _rope(L, nr=_nr(**kw)) == INVALID, kw
        assert _qkv(L, nr=_nr(**kw)) == INVALID, kw
    assert _rope(L, dtype=3) == INVALID and _rope(L, dh=48) == UNSUPPORTED and _rope(L, n=-1) == INVALID
    assert _rope(L, hq=0, hk=0) == INVALID and _rope(L, positions=None) == INVALID
    assert _rope(L, n=1 << 30, hq=4) == UNSUPPORTED
    assert _qkv(L, n_heads=0) == INVALID
    assert _rope(L, n=0) == 0               # no rows: nothing to do, nothing read
    assert _write(L, rows=_rows(n_rows=0, max_rows=0)) == 0


def test_refuses_bad_attention():
    L = _lib()
    for kw in (dict(dtype=7), dict(n_heads=3), dict(n_heads=0), dict(causal=2), dict(window=-1), dict(max_length=-1),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")),
               dict(cap=float("inf")), dict(lengths=None)):
        assert _attend(L, att=_att(**kw)) == INVALID, kw
    assert _attend(L, att=_att(dtype=evo.EVO_FP32)) == UNSUPPORTED
    need = L.evo_chunk_attention_workspace(R(_cache()), R(_rows(max_pages=200)), R(_att()))
    assert need > 0 and need % 4 == 0
    for work, size in ((None, need), (A, need - 1), (A + 4, need)):
        assert _attend(L, rows=_rows(max_pages=200), work=work, size=size) == INVALID
        assert "workspace" in L.evo_last_error().decode()
    assert L.evo_chunk_attention_workspace(R(_cache()), R(_rows(n_rows=0, max_rows=0)), R(_att())) == 0
    assert L.evo_chunk_attention_workspace(R(_cache(head_dim=80)), R(_rows()), R(_att())) == UNSUPPORTED
    for f in (L.evo_cache_write, L.evo_cache_read):
        assert f(None, None, 1, None, None, None, None) == INVALID
    assert L.evo_chunk_attention(None, None, None, None, None, None, None, 0, None) == INVALID
    assert L.evo_qkv_write(None, None, None, 1, 1, None, None, None, None, None, None) == INVALID
    assert L.evo_qk_norm_rope(None, 1, 64, 1, 1, 1, None, None, None, None, None, None) == INVALID


def test_binding_refuses_host_tensors_and_shapes():
    _lib()
    k = torch.zeros(2, 2, 64, 32)
    with pytest.raises(TypeError):
        evo.KVCache(k, k.transpose(2, 3).contiguous())
    with pytest.raises(TypeError):
        evo.qk_norm_rope(torch.zeros(2, 2, 32), torch.zeros(2, 2, 32), None, None)
    t = evo.rope_table(7, 16, device="cpu")
    assert t.shape == (7, 8, 2) and np.allclose(t.numpy(), M.rope_table(7, 16), atol=1e-7)
