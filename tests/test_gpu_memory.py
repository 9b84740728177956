"""GPU parity of the operators over a long memory with the fp64 oracle: norm and
rotation, the paged cache, chunk attention; and where they can go wrong."""
import numpy as np
import pytest
import torch

from oracle import evo_memory as M
from paper_2607_20293_amd import evo
from tests.gpu_util import device, say
from tests.memory_util import DTYPES, EPS16, EPS32, FORMATS, Call, f64, i32, pool, table_for

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


# ---- norm and rotation -----------------------------------------------------
def _rope_bound(want, x, dtype, dh):
    """fp32: dh squares summed (relative dh EPS32, halved by the root), the root,
    the quotient, two products and a sum: each relative to the row's largest
    value; a bf16 result is rounded once more."""
    top = np.max(np.abs(want), -1, keepdims=True) * 2
    return (dh / 2 + 16) * EPS32 * top + (EPS16 * 1.01 * np.abs(want) if dtype == "bf16" else 0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dh,hq,hk,n,rotary,pairs,layout", [
    (64, 4, 4, 16, 64, "halves", "packed"), (64, 4, 4, 1, 64, "adjacent", "packed"), (32, 2, 2, 33, 32, "halves", "plain"),
    (128, 8, 2, 77, 128, "adjacent", "heads_first"), (128, 5, 1, 130, 64, "halves", "odd"), (64, 12, 12, 7, 32, "adjacent", "odd"),
    (32, 3, 1, 65, 16, "halves", "packed"), (64, 1, 1, 300, 0, "halves", "plain"), (128, 32, 8, 40, 96, "halves", "packed"),
    (64, 12, 12, 2050, 64, "halves", "packed"), (128, 1, 1, 4097, 128, "halves", "plain")])
def test_norm_rope(dtype, dh, hq, hk, n, rotary, pairs, layout):
    dev, gen = device(), torch.Generator().manual_seed(dh + n)
    say(f"[gpu] norm and rotation {dtype} dh {dh} rows {n} heads {hq}/{hk} rotary {rotary} {pairs} {layout}")
    pad = 1 if layout == "odd" else 0           # rows that are not aligned
    x = torch.randn((n, (hq + 2 * hk) * dh + pad), generator=gen).to(DTYPES[dtype]).to(dev)
    x = x[:, pad:].unflatten(1, (hq + 2 * hk, dh))
    if layout == "plain":
        x = x.contiguous()
    if layout == "heads_first":
        x = x.transpose(0, 1).contiguous().transpose(0, 1)
    q, k = x[:, :hq], x[:, hq:hq + hk]
    pos = torch.randint(0, 5000, (n,), generator=gen, dtype=torch.int32)
    tab = evo.rope_table(5000, rotary, device=dev) if rotary else None
    gains = [(1 + torch.randn(dh, generator=gen) * 0.3).to(dev) for _ in range(2)]
    cases = [(gains[0], gains[1], 1e-6), (None, gains[1], 1e-3), (None, None, None)]
    for qg, kg, eps in cases:
        got = evo.qk_norm_rope(q, k, pos.to(dev), tab, qg, kg, eps, pairs)
        for t, g, y in zip((q, k), (qg, kg), got):
            want = M.norm_rope(f64(t), None if g is None else f64(g), None if tab is None else f64(tab), pos.numpy(), pairs, eps)
            err = np.abs(f64(y) - want) / _rope_bound(want, f64(t), dtype, dh)
            assert err.max() <= 1, (eps, err.max())
    # in place, and into strided outputs
    q2 = x.clone()
    got2 = evo.qk_norm_rope(q2[:, :hq], q2[:, hq:hq + hk], pos.to(dev), tab, *cases[0], pairs,
                            out=(q2[:, :hq], q2[:, hq:hq + hk]))
    got = evo.qk_norm_rope(q, k, pos.to(dev), tab, *cases[0], pairs)
    assert torch.equal(got2[0], got[0]) and torch.equal(got2[1], got[1]) and torch.equal(q2[:, hq + hk:], x[:, hq + hk:])


def test_norm_rope_marks_positions_outside_the_table():
    dev = device()
    x = torch.randn(4, 2, 64, device=dev)
    pos = torch.tensor([0, -1, 10, 9], dtype=torch.int32, device=dev)
    q, k = evo.qk_norm_rope(x, x[:, :1], pos, evo.rope_table(10, 32, device=dev))
    for y in (q, k):
        assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all() and torch.isfinite(y[0]).all() and torch.isfinite(y[3]).all()


def test_norm_rope_extreme_rows():
    """Rows of zeros stay zeros; rows of tiny and large values keep their norm."""
    dev = device()
    x = torch.zeros(3, 1, 64, device=dev)
    x[1] = 1e-3
    x[2] = 1e15
    y = evo.qk_norm_rope(x, x, torch.zeros(3, dtype=torch.int32, device=dev), None, eps=1e-12)[0]
    assert not y[0].any()
    assert torch.allclose(y[1:], torch.ones_like(y[1:]), rtol=1e-5)


# ---- the paged cache -------------------------------------------------------
def _written(dev, dtype, fmt, rows, starts, heads, dh, size, seed, cu=True, edit=None):
    rng = np.random.default_rng(seed)
    gen = torch.Generator().manual_seed(seed)
    n = int(sum(rows))
    tab, pages = table_for([s + r for s, r in zip(starts, rows)], size, 2, rng)
    t = pool(fmt, pages, heads, size, dh, dev, gen)
    before = [None if x is None else x.clone() for x in t]
    x = torch.randn((n, 2 * heads, dh), generator=gen) * torch.exp(torch.randn((n, 2 * heads, 1), generator=gen))
    if edit:
        edit(x)
    x = x.to(DTYPES[dtype]).to(dev)
    k, v = x[:, :heads], x[:, heads:]
    cu_rows = i32(np.concatenate([[0], np.cumsum(rows)]), dev) if cu else None
    cache = evo.KVCache(*t)
    at = (i32(tab, dev), i32(starts, dev))
    evo.cache_write(cache, *at, k, v, cu_rows, max(rows) if cu else None)
    back = evo.cache_read(cache, *at, n, DTYPES[dtype], cu_rows, max(rows) if cu else None)
    return cache, before, tab, k, v, back


def _check_held(x, back, dtype, fmt, what):
    """A value read back is its code's: x / s to the nearest code, up to the
    rounding of s, of x / s and of the product (8 EPS32 of the row's largest
    code, which moves at most a tie), and of the value to dtype."""
    x, back = f64(x), f64(back)
    if fmt in ("fp32", "bf16"):
        assert np.array_equal(x, back, equal_nan=True), what
        return
    c, s = M.quantise(x, fmt)
    top = M.TOP[fmt]
    want = c * s[..., None]
    assert np.array_equal(np.isnan(back).all(-1), np.isnan(s)) and np.array_equal(np.isnan(back).any(-1), np.isnan(s)), what
    fine = np.isfinite(s)
    unit = s[fine][:, None]
    half = 0.5 * unit if fmt == "int8" else np.maximum(np.abs(x[fine]) * 2.0 ** -4, unit * 2.0 ** -10)
    read = np.abs(want[fine]) * (EPS16 * 1.01 if dtype == "bf16" else 4 * EPS32) + 1e-45
    assert np.all(np.abs(back[fine] - x[fine]) <= half + 8 * EPS32 * top * unit + read * 1.1), what
    # all but ties are the definition's codes
    off = np.abs(back[fine] - want[fine]) > read + 4 * EPS32 * np.abs(want[fine])
    y = np.divide(np.abs(x[fine]), unit, out=np.zeros_like(x[fine]), where=unit > 0)
    step = np.ones_like(y) if fmt == "int8" else 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3)
    tie = np.abs(y / step - np.floor(y / step) - 0.5) < 8 * EPS32 * top / step
    assert not np.any(off & ~tie & (unit > 1e-37)), what


PAIRS = [("fp32", "fp32"), ("bf16", "bf16"), ("fp32", "int8"), ("bf16", "int8"), ("fp32", "fp8"), ("bf16", "fp8")]


@pytest.mark.parametrize("dtype,fmt", PAIRS)
@pytest.mark.parametrize("dh,heads,size,rows,starts", [
    (64, 2, 64, [1], [0]), (64, 4, 64, [1, 1, 1], [63, 64, 200]), (128, 2, 128, [70, 1, 200, 64], [0, 127, 100, 64]),
    (32, 3, 256, [300, 5], [3, 250]), (64, 12, 64, [65, 0, 63, 2], [1, 10, 0, 62]), (128, 1, 1024, [513], [1020])])
def test_cache_holds_and_reads_back(dtype, fmt, dh, heads, size, rows, starts):
    dev = device()
    say(f"[gpu] cache {dtype} in {fmt} dh {dh} heads {heads} pages of {size} rows {rows} from {starts}")
    cache, before, tab, k, v, back = _written(dev, dtype, fmt, rows, starts, heads, dh, size, 5)
    _check_held(k, back[0], dtype, fmt, "keys")
    _check_held(v, back[1], dtype, fmt, "values")
    # nothing else was written
    touched = np.zeros((cache.n_pages, size), bool)
    for s, (r, b) in enumerate(zip(rows, starts)):
        for p in range(b, b + r):
            touched[M.place(tab, size, s, p)] = True
    free = torch.from_numpy(~touched).to(dev)
    for now, then, dim in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), before, (2, 3, 2, 2)):
        if now is None:
            continue
        a, b = (t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in (now, then))
        assert torch.equal(a.movedim(dim, 1)[free], b.movedim(dim, 1)[free])


@pytest.mark.parametrize("dtype,fmt", [p for p in PAIRS if p[1] in M.TOP])
def test_cache_of_extreme_rows(dtype, fmt):
    """Zeros, tiny and huge rows, ties, NaNs and infinities."""
    dev = device()

    def edit(x):
        x[0] = 0
        x[1] *= 1e-37
        x[2] *= 1e37
        x[3] = torch.arange(64) * 0.5                     # ties of int8 codes
        x[3, :, 63] = 127
        x[4, 0, 5], x[4, 3, 60] = NAN, NAN
        x[5, 1, 0], x[5, 2, 63] = INF, -INF
        x[6] = 3e-41
        x[7, :, :] = 448.0 / 64 * torch.arange(64)
    _, _, _, k, v, back = _written(dev, dtype, fmt, [9], [60], 2, 64, 64, 6, edit=edit)
    _check_held(k, back[0], dtype, fmt, "keys")
    _check_held(v, back[1], dtype, fmt, "values")
    assert not back[0][0].any()


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_rows_outside_the_table_are_not_written(fmt):
    dev = device()
    gen = torch.Generator().manual_seed(0)
    t = pool(fmt, 3, 2, 64, 64, dev, gen)
    raw = [x.clone() for x in t if x is not None]
    cache = evo.KVCache(*t)
    k = torch.randn(20, 2, 64, device=dev, dtype=torch.bfloat16)
    tab = i32([[0], [1]], dev)
    evo.cache_write(cache, tab, i32([60, -6], dev), k, k)       # 6 of each 10 rows lie outside
    got = evo.cache_read(cache, tab, i32([60, -6], dev), 20, torch.bfloat16)
    for y in got:
        assert not y[4:10].any() and not y[10:16].any() and y[:4].any() and y[16:].any()
    page2 = [x for x in t if x is not None]
    assert all(torch.equal(a[2], b[2]) for a, b in zip(page2, raw))
    # page numbers outside the cache are taken as its last page
    held = [x[:2].clone() for x in page2]
    evo.cache_write(cache, i32([[7], [-1]], dev), i32([0, 32], dev), k, k)
    assert all(torch.equal(a[:2], b) for a, b in zip(page2, held))
    got = evo.cache_read(cache, i32([[2], [2]], dev), i32([0, 32], dev), 20, torch.bfloat16)
    _check_held(k, got[0], "bf16", fmt, "keys")


@pytest.mark.parametrize("dtype,fmt", PAIRS)
@pytest.mark.parametrize("dh,hq,hk,rotary,pairs,rows,starts", [
    (64, 4, 4, 64, "halves", [1, 1], [5, 64]), (128, 8, 2, 64, "adjacent", [40, 3, 90], [0, 61, 100]),
    (32, 2, 2, 32, "adjacent", [129], [0])])
def test_qkv_write_is_norm_rope_and_write(dtype, fmt, dh, hq, hk, rotary, pairs, rows, starts):
    dev, n = device(), sum(rows)
    gen = torch.Generator().manual_seed(9)
    tab, pages = table_for([a + b for a, b in zip(rows, starts)], 64, 1, np.random.default_rng(9))
    t = pool(fmt, pages, hk, 64, dh, dev, gen)
    x = torch.randn((n, hq + 2 * hk, dh), generator=gen).to(DTYPES[dtype]).to(dev)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    table = evo.rope_table(300, rotary, device=dev)
    gains = [(1 + torch.randn(dh, generator=gen) * 0.3).to(dev) for _ in range(2)]
    cu = i32(np.concatenate([[0], np.cumsum(rows)]), dev)
    pos = i32(np.concatenate([np.arange(b, b + r) for r, b in zip(rows, starts)]), dev)
    cache = evo.KVCache(*t)
    at = (i32(tab, dev), i32(starts, dev))
    qo = evo.qkv_write(cache, *at, q, k, v, table, *gains, 1e-6, pairs, cu, max(rows))
    back = evo.cache_read(cache, *at, n, DTYPES[dtype], cu, max(rows))
    q2, k2 = evo.qk_norm_rope(q, k, pos, table, *gains, 1e-6, pairs)
    assert torch.equal(qo, q2)
    if fmt in ("fp32", "bf16"):
        assert torch.equal(back[0], k2) and torch.equal(back[1], v)
        return
    # keys are coded from the 32-bit result
    k32 = evo.qk_norm_rope(q.float(), k.float(), pos, table, *gains, 1e-6, pairs)[1]
    ref = M.norm_rope(f64(k), f64(gains[1]), f64(table), pos.cpu().numpy(), pairs, 1e-6)
    assert np.max(np.abs(f64(k32) - ref)) <= 1e-4
    _check_held(k32, back[0], dtype, fmt, "keys")
    _check_held(v, back[1], dtype, fmt, "values")


# ---- attention -------------------------------------------------------------
ATT_PAIRS = PAIRS
SHAPES = [
    # rows, lengths, heads, kv_heads, dh, page, options
    ([1], [1], 4, 4, 64, 64, {}),
    ([1, 1, 1], [64, 65, 0], 2, 2, 32, 64, {}),
    ([16], [1000], 4, 4, 64, 64, {}),
    ([16, 16], [63, 130], 4, 4, 64, 128, dict(causal=True)),
    ([5, 0, 17, 1], [5, 9, 400, 257], 8, 2, 64, 64, dict(causal=True, window=33)),
    ([33, 20], [300, 20], 6, 2, 128, 256, dict(causal=True, cap=20.0)),
    ([32, 7], [290, 64], 12, 12, 64, 64, dict(causal=True, prefix=[100, 3], window=20)),
    ([7, 9], [200, 129], 4, 1, 128, 64, dict(bias=True)),
    ([40], [513], 4, 2, 32, 1024, dict(causal=True, bias=True, cap=5.0, scale=0.5)),
    ([100, 3], [130, 700], 4, 4, 64, 64, dict(causal=True, bias=True)),
    ([12, 12], [200, 0], 3, 3, 128, 64, dict(window=50, starts=[-30, 4])),
    ([9, 30], [100, 70], 2, 1, 64, 64, dict(causal=True, starts=[-4, 60])),
    ([260], [500], 2, 2, 128, 64, dict(causal=True)),
    ([300, 150], [300, 470], 4, 2, 64, 64, dict(causal=True, prefix=[290, 5], cap=30.0)),
    ([1, 1], [5000, 4097], 16, 2, 64, 64, dict(causal=True)),
    ([2], [9001], 7, 1, 128, 256, dict(bias=True, window=4000)),
]


@pytest.mark.parametrize("dtype,fmt", ATT_PAIRS)
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_attention(dtype, fmt, i):
    rows, lengths, heads, kv_heads, dh, size, kw = SHAPES[i]
    say(f"[gpu] attention {dtype} over {fmt}: rows {rows} lengths {lengths} heads {heads}/{kv_heads} dh {dh} page {size} {kw}")
    c = Call(device(), dtype, fmt, rows, lengths, heads, kv_heads, dh, size, seed=i, **kw)
    c.check("attention")


@pytest.mark.parametrize("dtype,fmt", [("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp8")])
@pytest.mark.parametrize("rows,lengths", [([2], [20000]), ([1] * 3, [0, 3000, 1]), ([64], [2500])])
def test_parts_of_the_keys_join(dtype, fmt, rows, lengths):
    """Long keys and few rows are split over workgroups; the result is the same
    at every call, whatever the bound of the lengths says."""
    c = Call(device(), dtype, fmt, rows, lengths, 2, 2, 64, seed=3, causal=True)
    a = c.run()
    c.check("split", got=a)
    for more in ({}, dict(max_length=max(lengths))):
        b = c.run(**more)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c.check("one part", got=c.run(max_length=1))


@pytest.mark.parametrize("dtype,fmt", ATT_PAIRS)
@pytest.mark.parametrize("rows", [[6, 20], [150, 140]])
def test_what_is_not_seen_does_not_matter(dtype, fmt, rows):
    """NaNs and infinities in unwritten slots, in the future, outside the window:
    rows that do not see them keep their bits."""
    dev = device()
    c = Call(dev, dtype, fmt, rows, [200, 161], 4, 2, 64, seed=4, causal=True, window=90)
    clean = c.run()
    clean = [t.clone() for t in clean]
    c.check("clean", got=clean)
    k, v, ks, vs = c.tensors
    used = np.zeros((k.shape[0], 64), bool)
    for s, n in enumerate(c.lengths):
        for p in range(n):
            used[M.place(c.tab, 64, s, p)] = True
    junk = torch.from_numpy(~used).to(dev)
    bad = torch.tensor([NAN, INF, -INF], device=dev)
    kv, vv = k.permute(0, 2, 1, 3), v.permute(0, 3, 1, 2)           # [page][slot][head][dh]

    def spoil(mask):
        n = int(mask.sum())
        fill = bad[torch.arange(n * 2 * 64, device=dev) % 3].view(n, 2, 64)
        if ks is None:
            kv[mask], vv[mask] = fill.to(k.dtype), fill.flip(0).to(k.dtype)
        else:
            if fmt == "fp8":
                kv.view(torch.uint8)[mask] = 0x7f
                vv.view(torch.uint8)[mask] = 0xff
            ks.permute(0, 2, 1)[mask] = fill[:, :, 0]
            vs.permute(0, 2, 1)[mask] = fill[:, :, 1]
    spoil(junk)
    got = c.run()
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    # the last position of sequence 0 (seen by its last row alone) and position
    # 40 of sequence 1 (outside every window if its chunk begins at 131 or later)
    pg, sl = M.place(c.tab, 64, 0, 199)
    mask = torch.zeros_like(junk)
    mask[pg, sl] = True
    spoil(mask)
    if rows[1] == 20:
        pg, sl = M.place(c.tab, 64, 1, 40)
        mask = torch.zeros_like(junk)
        mask[pg, sl] = True
        spoil(mask)
    got = c.run()
    last = rows[0] - 1
    keep = [i for i in range(sum(rows)) if i != last]
    assert torch.equal(got[0][keep], clean[0][keep]) and torch.equal(got[1][keep], clean[1][keep])
    assert not torch.isfinite(got[0][last]).any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [[4], [200]])
def test_infinite_values_reach_the_rows_that_see_them(dtype, rows):
    dev = device()
    c = Call(dev, dtype, dtype, rows, [rows[0] + 3], 2, 2, 64, seed=5, causal=True)
    v = c.tensors[1]
    for pos, ch, x in ((rows[0] + 2, 3, INF), (rows[0] + 2, 4, -INF), (rows[0] + 1, 4, INF), (rows[0], 9, NAN), (1, 20, -INF)):
        pg, sl = M.place(c.tab, 64, 0, pos)
        v[pg, :, ch, sl] = x
    c.check("infinite values")


def test_empty_rows_and_sequences():
    dev = device()
    c = Call(dev, "bf16", "bf16", [3, 2, 4], [0, 5, 3], 2, 2, 64, seed=6, causal=True, starts=[0, -2, 0])
    out, lse = c.run(out=torch.full((9, 2, 64), 7.0, dtype=torch.bfloat16, device=dev))
    assert not out[:5].any() and torch.isneginf(lse[:5]).all() and out[5:].any()
    c.check("empty", got=(out, lse))
    cache = evo.KVCache(*c.tensors)
    o, e = evo.chunk_attention(c.q[:0], cache, i32(c.tab, dev), i32([0, 5, 3], dev), i32([0, 0, 0, 0], dev), 0)
    assert o.shape == (0, 2, 64) and e.shape == (0, 2)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "bf16"), ("fp32", "int8")])
@pytest.mark.parametrize("rows", [[20, 7], [170, 60]])
def test_strides_and_alignment(dtype, fmt, rows):
    """q and out as views whose rows are strided, unaligned, heads first."""
    dev = device()
    c = Call(dev, dtype, fmt, rows, [190, 100], 4, 2, 64, seed=7, causal=True)
    ref = c.run()
    c.check("plain", got=ref)
    n = sum(rows)
    odd = torch.zeros(n * (4 * 64 + 3) + 1, dtype=c.q.dtype, device=dev)[1:].view(n, 259)[:, :256].unflatten(1, (4, 64))
    odd.copy_(c.q)
    first = c.q.transpose(0, 1).contiguous().transpose(0, 1)
    for q in (odd, first, torch.cat([c.q, c.q], 2)[..., :64]):
        for out in (torch.zeros_like(c.q), torch.zeros(4, n, 64, dtype=c.q.dtype, device=dev).transpose(0, 1),
                    torch.zeros(n, 4 * 64 + 1, dtype=c.q.dtype, device=dev)[:, 1:].unflatten(1, (4, 64))):
            got = c.run(q=q, out=out)
            assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    # one query for all rows (stride 0)
    one = c.q[:1].expand(n, 4, 64)
    a, b = c.run(q=one), c.run(q=one.contiguous())
    assert torch.equal(a[0], b[0])


def test_shared_and_reordered_pages():
    """Two sequences over the same pages give what two copies give."""
    dev = device()
    c = Call(dev, "bf16", "bf16", [8, 8], [130, 130], 4, 4, 64, seed=8)
    c.tab[1] = c.tab[0]
    c.q[8:] = c.q[:8]
    out, lse = c.run()
    assert torch.equal(out[:8], out[8:]) and torch.equal(lse[:8], lse[8:])
    c.check("shared", got=(out, lse))


def test_another_stream_and_graph_replays():
    """On a stream of its own; and captured once, replayed with new contents."""
    dev = device()
    c = Call(dev, "bf16", "int8", [3, 2], [3000, 2000], 4, 2, 64, seed=9, causal=True)
    ref = c.run()
    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    got = c.run(stream=side)
    torch.cuda.current_stream(dev).wait_stream(side)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])

    cache = evo.KVCache(*c.tensors)
    tab, cu = i32(c.tab, dev), i32(c.cu, dev)
    starts, lengths = i32([2997, 1998], dev), i32([3000, 2000], dev)
    table = evo.rope_table(4096, 64, device=dev)
    x = torch.randn(5, 8, 64, device=dev, dtype=torch.bfloat16)

    def step():
        q = evo.qkv_write(cache, tab, starts, x[:, :4], x[:, 4:6], x[:, 6:], table, cu_rows=cu, max_rows=3)
        return evo.chunk_attention(q, cache, tab, lengths, cu, 3, causal=True)
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        held = step()
    for r in range(4):
        x.copy_(torch.randn(5, 8, 64, device=dev, dtype=torch.bfloat16))
        starts.copy_(i32([2997 - 500 * r, 1998 - 3 * r], dev))
        lengths.copy_(starts + i32([3, 2], dev))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = step()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), r


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes of keys, its last pages in use."""
    dev = device()
    pages, heads, dh = 270000, 4, 64                   # 8.8 GB of bf16 keys, as much of values
    k = torch.empty((pages, heads, 64, dh), dtype=torch.bfloat16, device=dev)
    v = torch.empty((pages, heads, dh, 64), dtype=torch.bfloat16, device=dev)
    cache = evo.KVCache(k, v)
    gen = torch.Generator().manual_seed(1)
    tab = np.array([[pages - 1, 5, pages - 3], [pages // 2, pages - 2, 0]], np.int32)
    x = torch.randn((300, 2 * heads, dh), generator=gen).to(torch.bfloat16).to(dev)
    at = (i32(tab, dev), i32([0, 0], dev))
    evo.cache_write(cache, *at, x[:, :heads], x[:, heads:])
    back = evo.cache_read(cache, *at, 300, torch.bfloat16)
    assert torch.equal(back[0], x[:, :heads]) and torch.equal(back[1], x[:, heads:])
    q = torch.randn((300, heads, dh), generator=gen).to(torch.bfloat16).to(dev)
    for rows in (4, 150):
        qq = torch.cat([q[:rows], q[150:150 + rows]])
        out, _ = evo.chunk_attention(qq, cache, at[0], i32([150, 150], dev))
        for s in range(2):
            kk, vv = f64(x[150 * s:150 * s + 150, :heads]), f64(x[150 * s:150 * s + 150, heads:])
            want, _ = M.attend(f64(qq[rows * s:rows * s + rows]), kk, vv, 0, dh ** -0.5)
            assert np.max(np.abs(f64(out[rows * s:rows * s + rows]) - want)) <= 1.1 * EPS16 * np.max(np.abs(vv))


def test_tables_and_lengths_that_lie_outside():
    """Whatever the device arrays hold, every access stays in the caller's
    arrays: the calls end, and in-range sequences are right."""
    dev = device()
    c = Call(dev, "bf16", "bf16", [4, 4], [100, 90], 2, 2, 64, seed=10, causal=True)
    want = c.run()
    tab = c.tab.copy()
    tab[1] = [1 << 30, -5][:tab.shape[1]] if tab.shape[1] == 2 else 1 << 30
    cache = evo.KVCache(*c.tensors)
    got = evo.chunk_attention(c.q, cache, i32(tab, dev), i32([100, 1 << 30], dev), i32([0, 4, 8], dev), 4, causal=True)
    assert torch.equal(got[0][:4], want[0][:4])
    got = evo.chunk_attention(c.q, cache, i32(c.tab, dev), i32([100, -7], dev), i32([0, 4, 1 << 30], dev), 5, causal=True)
    torch.cuda.synchronize()
    assert torch.equal(got[0][:4], want[0][:4])


@pytest.mark.parametrize("rows", [15, 150])
def test_row_numbers_that_lie_outside(rows):
    """cu_rows whose entries are any 32-bit numbers: no access leaves the call's
    rows, and rows that they still name are right."""
    dev = device()
    c = Call(dev, "bf16", "bf16", [rows, 4], [170, 90], 4, 2, 64, seed=11, causal=True)
    want = c.run()
    cache = evo.KVCache(*c.tensors)
    n = rows + 4
    for cu in ([-2 ** 31, rows, n], [0, rows, 2 ** 31 - 1], [0, rows, -2 ** 31], [2 ** 31 - 1, -2 ** 31, n]):
        got = evo.chunk_attention(c.q, cache, i32(c.tab, dev), i32([170, 90], dev), i32(cu, dev), n, causal=True)
        torch.cuda.synchronize()
        if cu[:2] == [0, rows]:
            assert torch.equal(got[0][:rows], want[0][:rows]), cu


@pytest.mark.parametrize("rows,lengths,heads", [([1], [9000], 4), ([16] * 24, [2500] * 24, 4), ([1] * 6, [20000] * 6, 8)])
def test_joined_parts_at_every_call(rows, lengths, heads):
    """Parts of the keys that workgroups of one launch join: the same bits at
    each of many calls, alone and recorded, in memory that other work used."""
    dev = device()
    c = Call(dev, "bf16", "bf16", rows, lengths, heads, 4, 64, seed=12, causal=True)
    cache, tab, lens, cu = evo.KVCache(*c.tensors), i32(c.tab, dev), i32(c.lengths, dev), i32(c.cu, dev)

    def call():
        return evo.chunk_attention(c.q, cache, tab, lens, cu, max(rows), causal=True)
    one = evo.chunk_attention(c.q, cache, tab, lens, cu, max(rows), causal=True, max_length=1)    # not in parts
    want = [t.clone() for t in call()]
    top = float(c.tensors[1].float().abs().max())
    assert float((want[0].float() - one[0].float()).abs().max()) <= 2.2 * EPS16 * top
    side = torch.cuda.Stream(dev)
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        held = call()
    wrong = torch.zeros((), dtype=torch.int64, device=dev)
    for r in range(200):
        got = call()
        wrong += (got[0] != want[0]).sum() + (got[1] != want[1]).sum()
        del got
        if r % 3 == 0:
            torch.empty(1 << (14 + r % 8), device=dev).normal_()
        held[0].zero_()
        graph.replay()
        wrong += (held[0] != want[0]).sum() + (held[1] != want[1]).sum()
    assert int(wrong) == 0


@pytest.mark.parametrize("dtype,fmt,rows,lengths,dh,kw", [
    ("bf16", "int8", [2060, 3], [2100, 700], 64, dict(causal=True, window=900)),
    ("bf16", "bf16", [1030, 2], [1100, 65], 32, dict(causal=True)),
    ("bf16", "int8", [100, 97], [300, 130], 128, dict(causal=True, cap=20.0)),
    ("bf16", "fp8", [130, 20], [190, 500], 128, dict(causal=True, prefix=[170, 0], window=50)),
    ("bf16", "fp8", [700], [800], 64, dict(causal=True, window=300)),
    ("bf16", "int8", [500], [520], 32, {})])
def test_attention_of_long_chunks(dtype, fmt, rows, lengths, dh, kw):
    """Both sides of the numbers of rows from which keys pass through LDS."""
    say(f"[gpu] long chunks {dtype} over {fmt}: rows {rows} lengths {lengths} dh {dh} {kw}")
    Call(device(), dtype, fmt, rows, lengths, 1, 1, dh, seed=13, **kw).check("long chunks")


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_unwritten_scales_do_not_matter_to_long_chunks(fmt):
    dev = device()
    c = Call(dev, "bf16", fmt, [150, 140], [200, 161], 2, 2, 128, seed=14, causal=True)
    clean = [t.clone() for t in c.run()]
    c.check("clean", got=clean)
    k, v, ks, vs = c.tensors
    unused = torch.ones((k.shape[0], 64), dtype=torch.bool)
    for s, n in enumerate(c.lengths):
        for p in range(n):
            unused[M.place(c.tab, 64, s, p)] = False
    unused = unused.to(dev)
    for x, bad in ((ks, NAN), (vs, INF)):
        x.permute(0, 2, 1)[unused] = bad
    if fmt == "fp8":
        k.permute(0, 2, 1, 3).view(torch.uint8)[unused] = 0x7f
        v.permute(0, 3, 1, 2).view(torch.uint8)[unused] = 0xff
    got = c.run()
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])


@pytest.mark.parametrize("dtype,fmt,rows", [("bf16", "int8", 64), ("bf16", "fp8", 60), ("fp32", "fp32", 120), ("bf16", "bf16", 60)])
def test_many_rows_over_few_keys(dtype, fmt, rows):
    """As many row tiles as the device has SIMDs and more: a wave takes a tile."""
    n = 34 if rows == 64 else 70
    lengths = [(37 * s) % 140 for s in range(n)]
    Call(device(), dtype, fmt, [rows - s % 3 for s in range(n)], lengths, 8, 8, 64, seed=15, causal=True).check("few keys")
