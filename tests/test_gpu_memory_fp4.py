"""The paged cache of 4-bit floats and the attention over it, on the GPU, against
the definition in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import evo_memory as M
from paper_2607_20293_amd import evo
from tests.gpu_util import device, say
from tests.memory_util import DTYPES, EPS16, Call, f64, i32, table_for

pytestmark = pytest.mark.gpu

FP4 = torch.float4_e2m1fn_x2
NAN, INF = float("nan"), float("inf")


def pool4(pages, heads, size, dh, dev, gen):
    """Codes of every kind everywhere, and scales."""
    k = torch.randint(0, 256, (pages, heads, size, dh // 2), generator=gen, dtype=torch.uint8)
    v = torch.randint(0, 256, (pages, heads, dh // 2, size), generator=gen, dtype=torch.uint8)
    scales = [(torch.rand((pages, heads, size), generator=gen) + 0.5).div_(3).to(dev) for _ in range(2)]
    return [k.to(dev), v.to(dev)] + scales


def handle(t):
    return evo.KVCache(t[0].view(FP4), t[1].view(FP4), t[2], t[3])


def values_of(t):
    """The codes' values as arrays k [pages][heads][slots][dh], v [pages][heads][dh][slots]."""
    return M.e2m1_of_bytes(t[0].cpu().numpy(), 3), M.e2m1_of_bytes(t[1].cpu().numpy(), 2)


class Call4(Call):
    """An attention call over a 4-bit cache and its reference."""

    def __init__(self, dev, dtype, rows, lengths, heads, kv_heads, dh, size=64, seed=0, **kw):
        super().__init__(dev, dtype, "int8", rows, lengths, heads, kv_heads, dh, size, seed, **kw)
        pages = self.tensors[0].shape[0]
        self.raw = pool4(pages, kv_heads, size, dh, dev, torch.Generator().manual_seed(seed + 1000))
        self.renew()

    def renew(self):
        self.tensors = [self.raw[0].view(FP4), self.raw[1].view(FP4), self.raw[2], self.raw[3]]

    def reference(self):
        held = self.tensors
        k, v = (torch.from_numpy(x) for x in values_of(self.raw))
        self.tensors = [k, v, self.raw[2], self.raw[3]]
        try:
            return super().reference()
        finally:
            self.tensors = held


# ---- the cache -------------------------------------------------------------
def coded(x):
    """(codes' values, scales) of rows x [...][dh] by the definition: the scale
    and the quotients are floats of 32 bits (a quotient of two of them, computed in
    64 bits and rounded, is correctly rounded)."""
    x = np.asarray(x, np.float64)
    bad = ~np.isfinite(x).all(-1)
    fine = np.where(bad[..., None], 0.0, x)
    s = (np.max(np.abs(fine), -1) / 6.0).astype(np.float32).astype(np.float64)
    y = np.where((s > 0)[..., None], fine, 0.0) / np.where(s > 0, s, 1.0)[..., None]
    y = np.clip(y.astype(np.float32).astype(np.float64), -6.0, 6.0)
    return M.e2m1(y), np.where(bad, NAN, s)


def _write_and_read(dev, dtype, rows, starts, heads, dh, size, seed=5, edit=None):
    gen = torch.Generator().manual_seed(seed)
    tab, pages = table_for([s + r for s, r in zip(starts, rows)], size, 2, np.random.default_rng(seed))
    t = pool4(pages, heads, size, dh, dev, gen)
    before = [x.clone() for x in t]
    n = int(sum(rows))
    x = torch.randn((n, 2 * heads, dh), generator=gen) * torch.exp(torch.randn((n, 2 * heads, 1), generator=gen))
    if edit:
        edit(x)
    x = x.to(DTYPES[dtype]).to(dev)
    k, v = x[:, :heads], x[:, heads:]
    cu = i32(np.concatenate([[0], np.cumsum(rows)]), dev)
    cache, at = handle(t), (i32(tab, dev), i32(starts, dev))
    evo.cache_write(cache, *at, k, v, cu, max(rows))
    back = evo.cache_read(cache, *at, n, DTYPES[dtype], cu, max(rows))
    # what lies in the cache, by the place of every row
    place = [M.place(tab, size, s, p) for s, (r, b) in enumerate(zip(rows, starts)) for p in range(b, b + r)]
    pg, sl = (torch.tensor(c, dtype=torch.long, device=dev) for c in zip(*place))
    held = [t[0][pg, :, sl], t[1][pg, :, :, sl], t[2][pg, :, sl], t[3][pg, :, sl]]
    free = torch.ones((pages, size), dtype=torch.bool, device=dev)
    free[pg, sl] = False
    for now, then, dim in zip(t, before, (2, 3, 2, 2)):
        assert torch.equal(now.movedim(dim, 1)[free], then.movedim(dim, 1)[free]), "other slots were written"
    return k, v, held, back


def _check_codes(x, codes, scale, back, dtype):
    """Codes, scales and what is read back are the definition's, bit by bit:
    nothing but roundings that it names.  (A row whose scale is below the normal
    floats is held to half a step of its largest code.)"""
    want, s = coded(f64(x))
    got = M.e2m1_of_bytes(codes.cpu().numpy(), codes.dim() - 1)
    got_s, fine = f64(scale), np.isfinite(s)
    assert np.array_equal(np.isnan(got_s), ~fine) and np.array_equal(np.isnan(f64(back)).all(-1), ~fine)
    normal = fine & (s > 2.0 ** -126)
    assert np.array_equal(got[normal], want[normal]) and np.array_equal(got_s[normal], s[normal])
    read = torch.from_numpy(want[normal] * s[normal][:, None]).float().to(DTYPES[dtype])
    assert np.array_equal(f64(back)[normal], f64(read))
    small = fine & ~normal
    assert np.all(np.abs(f64(back)[small] - f64(x)[small]) <= np.max(np.abs(f64(x)[small]), -1, initial=0)[:, None] / 6 + 3e-45)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dh,heads,size,rows,starts", [
    (64, 2, 64, [1], [0]), (64, 4, 64, [1, 1, 1], [63, 64, 200]), (128, 2, 128, [70, 1, 200, 64], [0, 127, 100, 64]),
    (32, 3, 256, [300, 5], [3, 250]), (64, 12, 64, [65, 0, 63, 2], [1, 10, 0, 62]), (128, 1, 1024, [513], [1020]),
    (32, 8, 64, [8200, 777], [5, 0]), (128, 8, 64, [4100, 4096], [1, 64])])
def test_cache_holds_the_nearest_codes(dtype, dh, heads, size, rows, starts):
    dev = device()
    say(f"[gpu] 4-bit cache {dtype} dh {dh} heads {heads} pages of {size} rows {rows} from {starts}")
    k, v, held, back = _write_and_read(dev, dtype, rows, starts, heads, dh, size)
    _check_codes(k, held[0], held[2], back[0], dtype)
    _check_codes(v, held[1], held[3], back[1], dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_of_every_size(dtype):
    """Zeros, tiny and huge rows, values on the borders between codes, NaNs and
    infinities."""
    def edit(x):
        x[0] = 0
        x[1] *= 1e-37
        x[2] *= 1e37
        x[3] = torch.arange(64) * 0.25 - 8
        x[3, :, :8] = torch.tensor([12.0, 0.5, 1.5, 2.5, 3.5, 5.0, 7.0, 10.0])      # 12: every other one is a border
        x[4, 0, 5], x[4, 3, 60] = NAN, NAN
        x[5, 1, 0], x[5, 2, 63] = INF, -INF
        x[6] = 3e-41
        x[7] = -x[3]
        x[8, :, 1:] = 0
        x[9] = 1.0
    k, v, held, back = _write_and_read(device(), dtype, [10], [60], 2, 64, 64, 6, edit)
    _check_codes(k, held[0], held[2], back[0], dtype)
    _check_codes(v, held[1], held[3], back[1], dtype)
    assert not back[0][0].any()


def test_neighbouring_tokens_share_no_byte():
    """Sequences that write neighbouring slots of one page in one call, and calls
    on two streams at once."""
    dev = device()
    gen = torch.Generator().manual_seed(2)
    t = pool4(1, 2, 64, 64, dev, gen)
    cache = handle(t)
    x = torch.randn((64, 4, 64), generator=gen).to(torch.bfloat16).to(dev)
    tab = torch.zeros((64, 1), dtype=torch.int32, device=dev)
    order = torch.randperm(64, generator=gen).int().to(dev)
    evo.cache_write(cache, tab, order, x[:, :2], x[:, 2:])
    back = evo.cache_read(cache, tab, order, 64, torch.bfloat16)
    keep = [b.clone() for b in back]
    _check_codes(x[:, :2], t[0][0].transpose(0, 1)[order.long()], t[2][0].t()[order.long()], back[0], "bf16")
    _check_codes(x[:, 2:], t[1][0].permute(2, 0, 1)[order.long()], t[3][0].t()[order.long()], back[1], "bf16")
    t[0].zero_(), t[1].zero_()
    torch.cuda.synchronize()
    for half in (0, 1):
        side = torch.cuda.Stream(dev)
        evo.cache_write(cache, tab[:32], order[half::2].contiguous(), x[half::2, :2], x[half::2, 2:], stream=side)
    torch.cuda.synchronize()
    back = evo.cache_read(cache, tab, order, 64, torch.bfloat16)
    assert torch.equal(back[0], keep[0]) and torch.equal(back[1], keep[1])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dh,hq,hk,rotary,pairs,rows,starts", [
    (64, 4, 4, 64, "halves", [1, 1], [5, 64]), (128, 8, 2, 64, "adjacent", [40, 3, 90], [0, 61, 100]),
    (32, 2, 2, 32, "adjacent", [129], [0])])
def test_qkv_write_into_four_bits(dtype, dh, hq, hk, rotary, pairs, rows, starts):
    """The queries of qk_norm_rope, and the cache that cache_write makes of the
    keys in 32 bits."""
    dev, n = device(), sum(rows)
    gen = torch.Generator().manual_seed(9)
    tab, pages = table_for([a + b for a, b in zip(rows, starts)], 64, 1, np.random.default_rng(9))
    t = pool4(pages, hk, 64, dh, dev, gen)
    u = [a.clone() for a in t]
    x = torch.randn((n, hq + 2 * hk, dh), generator=gen).to(DTYPES[dtype]).to(dev)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    table = evo.rope_table(300, rotary, device=dev)
    gains = [(1 + torch.randn(dh, generator=gen) * 0.3).to(dev) for _ in range(2)]
    cu = i32(np.concatenate([[0], np.cumsum(rows)]), dev)
    pos = i32(np.concatenate([np.arange(b, b + r) for r, b in zip(rows, starts)]), dev)
    at = (i32(tab, dev), i32(starts, dev))
    qo = evo.qkv_write(handle(t), *at, q, k, v, table, *gains, 1e-6, pairs, cu, max(rows))
    assert torch.equal(qo, evo.qk_norm_rope(q, k, pos, table, *gains, 1e-6, pairs)[0])
    k32 = evo.qk_norm_rope(q.float(), k.float(), pos, table, *gains, 1e-6, pairs)[1]
    evo.cache_write(handle(u), *at, k32, v.float(), cu, max(rows))
    assert all(torch.equal(a, b) for a, b in zip(t, u))


def test_slots_outside_the_table():
    dev = device()
    gen = torch.Generator().manual_seed(0)
    t = pool4(3, 2, 64, 64, dev, gen)
    raw = [x.clone() for x in t]
    cache = handle(t)
    k = torch.randn(20, 2, 64, device=dev, dtype=torch.bfloat16)
    tab = i32([[0], [1]], dev)
    evo.cache_write(cache, tab, i32([60, -6], dev), k, k)       # 6 of each 10 rows lie outside
    for y in evo.cache_read(cache, tab, i32([60, -6], dev), 20, torch.bfloat16):
        assert not y[4:10].any() and not y[10:16].any() and y[:4].any() and y[16:].any()
    assert all(torch.equal(a[2], b[2]) for a, b in zip(t, raw))


# ---- attention -------------------------------------------------------------
SHAPES = [
    # rows, lengths, heads, kv_heads, dh, page, options
    ([1], [1], 4, 4, 64, 64, {}),
    ([1, 1, 1], [64, 65, 0], 2, 2, 32, 64, {}),
    ([16], [1000], 4, 4, 64, 64, {}),
    ([16, 16], [63, 130], 4, 4, 64, 128, dict(causal=True)),
    ([5, 0, 17, 1], [5, 9, 400, 257], 8, 2, 64, 64, dict(causal=True, window=33)),
    ([33, 20], [300, 20], 6, 2, 128, 256, dict(causal=True, cap=20.0)),
    ([33, 20], [300, 20], 6, 2, 128, 256, dict(cap=100.0)),
    ([32, 7], [290, 64], 12, 12, 64, 64, dict(causal=True, prefix=[100, 3], window=20)),
    ([7, 9], [200, 129], 4, 1, 128, 64, dict(bias=True)),
    ([40], [513], 4, 2, 32, 1024, dict(causal=True, bias=True, cap=5.0, scale=0.5)),
    ([100, 3], [130, 700], 4, 4, 64, 64, dict(causal=True, bias=True)),
    ([12, 12], [200, 0], 3, 3, 128, 64, dict(window=50, starts=[-30, 4])),
    ([9, 30], [100, 70], 2, 1, 64, 64, dict(causal=True, starts=[-4, 60], scale=-0.2)),
    ([260], [500], 2, 2, 128, 64, dict(causal=True)),
    ([300, 150], [300, 470], 4, 2, 64, 64, dict(causal=True, prefix=[290, 5], cap=30.0)),
    ([1, 1], [5000, 4097], 16, 2, 64, 64, dict(causal=True)),
    ([2], [9001], 7, 1, 128, 256, dict(bias=True, window=4000)),
    ([100, 97], [300, 130], 1, 1, 128, 64, dict(causal=True, cap=100.0)),
    ([130, 20], [190, 500], 1, 1, 128, 512, dict(causal=True, prefix=[170, 0], window=50)),
    ([70, 66], [400, 66], 2, 2, 64, 64, dict(causal=True, bias=True)),
    ([2060, 3], [2100, 700], 1, 1, 64, 64, dict(causal=True, window=900)),
    ([1030, 2], [1100, 65], 1, 1, 32, 64, dict(causal=True)),
    ([64 - s % 3 for s in range(34)], [37 * s % 140 for s in range(34)], 8, 8, 64, 64, dict(causal=True)),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_attention_over_four_bits(dtype, i):
    rows, lengths, heads, kv_heads, dh, size, kw = SHAPES[i]
    say(f"[gpu] attention {dtype} over fp4: rows {rows} lengths {lengths} heads {heads}/{kv_heads} dh {dh} page {size} {kw}")
    Call4(device(), dtype, rows, lengths, heads, kv_heads, dh, size, seed=i, **kw).check("attention")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,lengths", [([2], [20000]), ([1] * 3, [0, 3000, 1]), ([64], [2500])])
def test_parts_of_the_keys_join(dtype, rows, lengths):
    c = Call4(device(), dtype, rows, lengths, 2, 2, 64, seed=3, causal=True)
    a = c.run()
    reference = c.reference()
    c.check("split", got=a, reference=reference)
    for more in ({}, dict(max_length=max(lengths))):
        b = c.run(**more)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c.check("one part", got=c.run(max_length=1), reference=reference)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,dh", [([6, 20], 64), ([150, 140], 64), ([150, 140], 128)])
def test_what_is_not_seen_does_not_matter(dtype, rows, dh):
    """Any codes, and NaNs and infinities as scales, in unwritten slots and in the
    future: rows that do not see them keep their bits; a row that sees such a slot
    does not stay finite."""
    dev = device()
    c = Call4(dev, dtype, rows, [200, 161], 4, 2, dh, seed=4, causal=True, window=90)
    clean = [t.clone() for t in c.run()]
    c.check("clean", got=clean)
    k, v, ks, vs = c.raw
    unused = torch.ones((k.shape[0], 64), dtype=torch.bool)
    for s, n in enumerate(c.lengths):
        for p in range(n):
            unused[M.place(c.tab, 64, s, p)] = False
    unused = unused.to(dev)

    def spoil(mask):
        n = int(mask.sum())
        k.permute(0, 2, 1, 3)[mask] = torch.randint(0, 256, (n, 2, dh // 2), dtype=torch.uint8, device=dev)
        v.permute(0, 3, 1, 2)[mask] = torch.randint(0, 256, (n, 2, dh // 2), dtype=torch.uint8, device=dev)
        ks.permute(0, 2, 1)[mask] = torch.tensor([NAN, INF], device=dev)
        vs.permute(0, 2, 1)[mask] = torch.tensor([-INF, NAN], device=dev)
    spoil(unused)
    got = c.run()
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    last = torch.zeros_like(unused)
    last[M.place(c.tab, 64, 0, 199)] = True
    spoil(last)
    got = c.run()
    keep = [i for i in range(sum(rows)) if i != rows[0] - 1]
    assert torch.equal(got[0][keep], clean[0][keep]) and torch.equal(got[1][keep], clean[1][keep])
    assert not torch.isfinite(got[0][rows[0] - 1]).any()


@pytest.mark.parametrize("rows", [[20, 7], [170, 60]])
def test_strides_and_alignment(rows):
    dev = device()
    c = Call4(dev, "bf16", rows, [190, 100], 4, 2, 64, seed=7, causal=True)
    ref = c.run()
    c.check("plain", got=ref)
    n = sum(rows)
    odd = torch.zeros(n * (4 * 64 + 3) + 1, dtype=c.q.dtype, device=dev)[1:].view(n, 259)[:, :256].unflatten(1, (4, 64))
    odd.copy_(c.q)
    first = c.q.transpose(0, 1).contiguous().transpose(0, 1)
    for q in (odd, first):
        for out in (torch.zeros_like(c.q), torch.zeros(4, n, 64, dtype=c.q.dtype, device=dev).transpose(0, 1),
                    torch.zeros(n, 4 * 64 + 1, dtype=c.q.dtype, device=dev)[:, 1:].unflatten(1, (4, 64))):
            got = c.run(q=q, out=out)
            assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


def test_written_attended_and_replayed():
    """Projection to cache to attention as a layer calls them, recorded once and
    replayed with other contents; and on a stream of its own."""
    dev = device()
    gen = torch.Generator().manual_seed(3)
    tab, pages = table_for([3000, 2000], 64, 1, np.random.default_rng(3))
    t = pool4(pages, 2, 64, 64, dev, gen)
    cache, tab, cu = handle(t), i32(tab, dev), i32([0, 3, 5], dev)
    starts, lengths = i32([2997, 1998], dev), i32([3000, 2000], dev)
    table = evo.rope_table(4096, 64, device=dev)
    x = torch.randn(5, 8, 64, device=dev, dtype=torch.bfloat16)

    def step(stream=None):
        q = evo.qkv_write(cache, tab, starts, x[:, :4], x[:, 4:6], x[:, 6:], table, cu_rows=cu, max_rows=3, stream=stream)
        return evo.chunk_attention(q, cache, tab, lengths, cu, 3, causal=True, stream=stream)
    want = step()
    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    got = step(side)
    torch.cuda.current_stream(dev).wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
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
        got = [y.clone() for y in held]
        want = step()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), r


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes of keys, its last pages in use."""
    dev = device()
    pages, heads, dh = 270000, 8, 64
    cache = evo.KVCache.empty(pages, heads, dh, 64, FP4, dev)
    assert cache.k.numel() > 2 ** 32
    gen = torch.Generator().manual_seed(1)
    tab = i32([[pages - 1, 5, pages - 3], [pages // 2, pages - 2, 0]], dev)
    x = torch.randn((300, 2 * heads, dh), generator=gen).to(torch.bfloat16).to(dev)
    evo.cache_write(cache, tab, i32([0, 0], dev), x[:, :heads], x[:, heads:])
    back = evo.cache_read(cache, tab, i32([0, 0], dev), 300, torch.bfloat16)
    held = []
    for y, part in zip(back, (x[:, :heads], x[:, heads:])):
        c, s = coded(f64(part))
        held.append(c * s[..., None])
        assert torch.equal(y, torch.from_numpy(held[-1]).float().to(torch.bfloat16).to(dev))
    q = torch.randn((300, heads, dh), generator=gen).to(torch.bfloat16).to(dev)
    for rows in (4, 150):
        qq = torch.cat([q[:rows], q[150:150 + rows]])
        out, _ = evo.chunk_attention(qq, cache, tab, i32([150, 150], dev))
        for s in range(2):
            part = slice(150 * s, 150 * s + 150)
            want, _ = M.attend(f64(qq[rows * s:rows * s + rows]), held[0][part], held[1][part], 0, dh ** -0.5)
            assert np.max(np.abs(f64(out[rows * s:rows * s + rows]) - want)) <= 1.1 * EPS16 * np.max(np.abs(held[1][part]))


def test_tables_and_lengths_that_lie_outside():
    dev = device()
    c = Call4(dev, "bf16", [4, 4], [100, 90], 2, 2, 64, seed=10, causal=True)
    want = c.run()
    tab = c.tab.copy()
    tab[1] = [1 << 30, -5]
    cache = evo.KVCache(*c.tensors)
    got = evo.chunk_attention(c.q, cache, i32(tab, dev), i32([100, 1 << 30], dev), i32([0, 4, 8], dev), 4, causal=True)
    assert torch.equal(got[0][:4], want[0][:4])
    got = evo.chunk_attention(c.q, cache, i32(c.tab, dev), i32([100, -7], dev), i32([0, 4, 1 << 30], dev), 5, causal=True)
    torch.cuda.synchronize()
    assert torch.equal(got[0][:4], want[0][:4])
