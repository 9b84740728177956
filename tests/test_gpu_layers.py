"""GPU parity of the layers around the attention with the definition in 64 bits:
products with 4-bit weights, norms around a block; and where they can go wrong."""
import numpy as np
import pytest
import torch

from oracle import evo_layers as E
from paper_2607_20293_amd import evo
from tests.gpu_util import device, say
from tests.layers_util import NormCall, check, linear_reference, random_weights
from tests.memory_util import f64, i32

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")


# ---- products with 4-bit weights -------------------------------------------
LINEAR = [  # rows, n_in, n_out
    (1, 1, 1), (1, 128, 16), (1, 8192, 33), (2, 31, 15), (16, 256, 1024), (17, 33, 17), (15, 127, 130), (3, 129, 700), (31, 500, 5),
    (32, 1024, 256), (33, 384, 64), (64, 640, 96), (65, 257, 129), (100, 96, 40), (128, 128, 128), (129, 1000, 257), (300, 4096, 130),
    (513, 160, 1000), (1, 640, 20011), (2100, 72, 8), (260, 2048, 520)]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,n_in,n_out", LINEAR)
def test_linear(dtype, rows, n_in, n_out):
    dev, gen = device(), torch.Generator().manual_seed(rows + n_in)
    say(f"[gpu] linear4 {dtype} rows {rows} {n_in} -> {n_out}")
    w = random_weights(n_out, n_in, gen, dev)
    x = torch.randn((rows, n_in), generator=gen).to(dtype).to(dev)
    bias = torch.randn(n_out, generator=gen).to(dev)
    for b, act in ((None, None), (bias, "silu"), (bias, "gelu")):
        check(evo.linear4(x, w, b, act), *linear_reference(x, w, b, act, dtype), f"{act}")


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,n_in,n_out", [(5, 200, 50), (40, 136, 33), (150, 264, 140), (300, 256, 256)])
def test_linear_strides(dtype, rows, n_in, n_out):
    """x and out as views, aligned and not; what lies around out keeps its value."""
    dev, gen = device(), torch.Generator().manual_seed(1)
    w = random_weights(n_out, n_in, gen, dev)
    x = torch.randn((rows, n_in), generator=gen).to(dtype).to(dev)
    want, bound = linear_reference(x, w, None, None, dtype)
    for pad, at in ((8, 0), (8, 8), (3, 1), (1, 0)):
        xv = torch.full((rows, n_in + pad), NAN, dtype=dtype, device=dev)[:, at:at + n_in] if at + n_in <= n_in + pad else None
        xv.copy_(x)
        for out_pad, out_at in ((0, 0), (5, 2), (8, 8)):
            base = torch.full((rows + 1, n_out + out_pad), 7.0, dtype=dtype, device=dev)
            out = base[:rows, out_at:out_at + n_out]
            assert evo.linear4(xv, w, out=out) is out
            check(out, want, bound, f"strides {pad} {at} {out_pad} {out_at}")
            assert bool((base[rows] == 7).all()) and bool((base[:, :out_at] == 7).all()) and bool((base[:, out_at + n_out:] == 7).all())
    one = x[:1].expand(rows, n_in)
    assert torch.equal(evo.linear4(one, w), evo.linear4(one.contiguous(), w))


@pytest.mark.parametrize("rows", [1, 20, 70, 300])
def test_linear_rows_do_not_meet(rows):
    """A NaN or an infinity in a row stays there, and a row's bits do not depend
    on the rows beside it or on its place among them."""
    dev, gen = device(), torch.Generator().manual_seed(2)
    w = random_weights(150, 300, gen, dev)
    x = torch.randn((rows, 300), generator=gen).to(BF16).to(dev)
    clean = evo.linear4(x, w)
    dirty = x.clone()
    dirty[rows // 2, 7], dirty[rows // 2, 299] = NAN, INF
    got = evo.linear4(dirty, w)
    keep = torch.arange(rows, device=dev) != rows // 2
    assert torch.equal(got[keep], clean[keep]) and bool(torch.isnan(got[rows // 2]).all())
    order = torch.randperm(rows, generator=gen).to(dev)
    assert torch.equal(evo.linear4(x[order], w), clean[order])


@pytest.mark.parametrize("rows", [3, 200])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_linear_extreme_scales(rows, dtype):
    """Groups of the least and the largest scales, and of the one that is a NaN."""
    dev, gen = device(), torch.Generator().manual_seed(3)
    w = random_weights(48, 256, gen, dev)
    w.scales[0] = 127 - 100
    w.scales[1] = 127 + 100
    w.scales[2, 3] = 255
    w.scales[3] = 0
    x = torch.randn((rows, 256), generator=gen).to(dtype).to(dev)
    got = evo.linear4(x, w)
    want, bound = linear_reference(x, w, None, None, dtype)
    keep = [i for i in range(48) if i != 3]
    check(got[:, keep], want[:, keep], bound[:, keep], "scales")
    assert bool(torch.isnan(got[:, 2]).all()) and not bool(torch.isnan(got[:, keep[:2] + keep[3:]]).any())
    # products of 2^-127 and values of some ones lie below the normal floats
    assert float(got[:, 3].float().abs().max()) < 1e-34


def test_linear_of_quantised_weights():
    """Weights of a layer: coded, used, read back, moved between types."""
    dev, gen = device(), torch.Generator().manual_seed(4)
    for n_out, n_in in ((64, 256), (33, 100), (5, 31)):
        m = torch.randn((n_out, n_in), generator=gen) * torch.exp(torch.randn((n_out, 1), generator=gen))
        want, e = E.quantise(m.numpy())
        for t in (m.to(dev), m.to(dev).double()):
            w = evo.Weights4.of(t)
            assert np.array_equal(f64(w.values()), want) and np.array_equal(w.scales.cpu().numpy(), e)
            other = evo.Weights4(w.codes.view(torch.float4_e2m1fn_x2), w.scales.view(torch.float8_e8m0fnu), n_in)
            x = torch.randn((7, n_in), generator=gen).to(dev)
            check(evo.linear4(x, other), *linear_reference(x, w, None, None, FP32), "quantised")


def test_linear_replayed_and_on_another_stream():
    dev, gen = device(), torch.Generator().manual_seed(5)
    w = random_weights(1000, 520, gen, dev)
    for rows in (4, 90, 400):
        x = torch.randn((rows, 520), generator=gen).to(BF16).to(dev)
        side = torch.cuda.Stream(dev)
        side.wait_stream(torch.cuda.current_stream(dev))
        got = evo.linear4(x, w, activation="silu", stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, evo.linear4(x, w, activation="silu"))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = evo.linear4(x, w, activation="silu")
        for r in range(3):
            x.copy_(torch.randn((rows, 520), generator=gen))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(held, evo.linear4(x, w, activation="silu"))


def test_linear_offsets_beyond_32_bits():
    """More than 2^32 values of x and of out."""
    dev, gen = device(), torch.Generator().manual_seed(6)
    rows, n_in, n_out = 70000, 128, 40
    w = random_weights(n_out, n_in, gen, dev)
    base = torch.empty((rows, 65536), dtype=BF16, device=dev)          # 9.2 GB
    x, out = base[:, :n_in], base[:, 32768:32768 + n_out]
    some = torch.tensor([0, 1, 40000, 65535, 65536, 69999], device=dev)
    x.zero_()
    x[some] = torch.randn((len(some), n_in), generator=gen).to(BF16).to(dev)
    evo.linear4(x, w, out=out)
    check(out[some], *linear_reference(x[some], w, None, None, BF16), "far rows")
    assert not bool(out[2:40000].any())


# ---- norms around a block --------------------------------------------------
TYPES = [(BF16, BF16), (FP32, BF16), (FP32, FP32)]


@pytest.mark.parametrize("stream,block", TYPES)
@pytest.mark.parametrize("rows,d,kw", [
    (1, 1, dict(pre="rms")), (16, 256, dict(pre="rms", post="rms", mods=1, even=True)),
    (5, 32, dict(pre="layer", post="layer", mods=3)), (33, 100, dict(pre="layer", post=None, mods=2)),
    (130, 128, dict(pre=None, post="rms", mods=4)), (7, 129, dict(pre="rms", post="layer", affine=False, alpha=0.5)),
    (64, 320, dict(pre="layer", has_y=False, mods=8, even=True, alpha=2.0)), (9, 500, dict(pre="rms", post="rms")),
    (6, 777, dict(pre="layer", post="rms", mods=6, even=True)), (11, 1024, dict(pre="rms", has_y=False, affine=False)),
    (4, 1500, dict(pre="layer", post="layer", eps=1e-3)), (3, 2048, dict(pre="rms", post="rms", mods=2)),
    (5, 2051, dict(pre="layer", post="rms", mods=1)), (2, 5120, dict(pre="rms", post="rms")), (3, 8192, dict(pre="layer", post="layer")),
    (2, 16384, dict(pre="layer", post="rms", mods=2)), (3, 16383, dict(pre="rms", post="layer")), (2000, 64, dict(pre="rms", mods=17)),
    (1, 4096, dict(pre="rms", post="rms", mods=1, even=True)), (700, 1000, dict(pre="layer", post=None, mods=5))])
def test_block_norm(stream, block, rows, d, kw):
    say(f"[gpu] block_norm {stream} {block} rows {rows} d {d} {kw}")
    NormCall(device(), stream, block, rows, d, seed=d + rows, **kw).check("norm")


@pytest.mark.parametrize("stream,block", TYPES)
@pytest.mark.parametrize("d", [64, 200, 1024, 3000])
def test_block_norm_strides_and_in_place(stream, block, d):
    dev = device()
    c = NormCall(dev, stream, block, 37, d, "rms", "layer", mods=5, seed=1)
    want = c.run()
    c.check("plain", got=want)

    def odd(t, pad, at):
        v = torch.full((t.shape[0], t.shape[1] + pad), NAN, dtype=t.dtype, device=dev)[:, at:at + t.shape[1]]
        return v.copy_(t)
    for pad, at in ((16, 8), (3, 1)):
        mods = {n: odd(c.kw[n], pad, at) for n in ("gate", "scale", "shift")}
        base = [torch.full((38, d + pad), 7.0, dtype=t, device=dev) for t in (stream, block)]
        outs = [b[:37, at:at + d] for b in base]
        got = c.run(x=odd(c.x, pad, at), y=odd(c.y, pad, at), x_out=outs[0], h_out=outs[1], **mods)
        assert got[0] is outs[0] and got[1] is outs[1]
        if pad == 16:
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        c.check("strided", got=got)
        for b in base:
            assert bool((b[37] == 7).all()) and bool((b[:, :at] == 7).all()) and bool((b[:, at + d:] == 7).all())
    x, y = c.x.clone(), c.y.clone()
    got = c.run(x=x, y=y, x_out=x, h_out=y)
    assert got[0] is x and got[1] is y and torch.equal(x, want[0]) and torch.equal(y, want[1])
    # a modulation that is the same for all (stride 0), and one row for all rows (stride 0)
    one = {n: c.kw[n][:1] for n in ("gate", "scale", "shift")}
    a = c.run(mod_rows=torch.zeros(37, dtype=torch.int32, device=dev), **one)
    b = c.run(**{n: t.expand(5, d) for n, t in one.items()})
    e = c.run(mod_rows=None, **one)
    assert all(torch.equal(a[i], b[i]) and torch.equal(a[i], e[i]) for i in (0, 1))
    a, b = c.run(x=c.x[:1].expand(37, d)), c.run(x=c.x[:1].expand(37, d).contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_block_norm_marks_rows_without_a_modulation():
    dev = device()
    c = NormCall(dev, BF16, BF16, 8, 256, "rms", "rms", mods=3, seed=2)
    rows = c.kw["mod_rows"].clone()
    want = c.run()
    for bad in (-1, 3, 2 ** 31 - 1, -2 ** 31):
        rows[5] = bad
        got = c.run(mod_rows=rows)
        for g, w in zip(got, want):
            assert bool(torch.isnan(g[5]).all()) and torch.equal(g[:5], w[:5]) and torch.equal(g[6:], w[6:])


@pytest.mark.parametrize("d", [48, 1024, 4096])
def test_block_norm_rows_do_not_meet(d):
    """NaNs and infinities stay in their row; rows of zeros and of one value, tiny
    and large ones."""
    dev = device()
    c = NormCall(dev, FP32, FP32, 21, d, "layer", "rms", seed=3)
    want = c.run()
    x, y = c.x.clone(), c.y.clone()
    x[4, d - 1], y[9, 0], y[20, 5] = NAN, INF, -INF
    got = c.run(x=x, y=y)
    keep = [i for i in range(21) if i not in (4, 9, 20)]
    for g, w in zip(got, want):
        assert torch.equal(g[keep], w[keep])
    assert bool(torch.isnan(got[1][[4, 9, 20]]).all())
    for spread in (1e-8, 1e4, 1e15):
        NormCall(dev, FP32, FP32, 5, d, "rms", "rms", spread=spread, seed=4).check(f"spread {spread}")
    c = NormCall(dev, FP32, FP32, 5, d, "layer", "layer", seed=5, offset=100.0)
    c.check("far from zero")
    zero = torch.zeros(3, d, device=dev)
    got = evo.block_norm(zero, zero, pre="layer", post="rms")
    assert not got[0].any() and not got[1].any()
    got = evo.block_norm(zero + 2.5, pre="layer", eps=1e-5)
    assert float(got[1].abs().max()) < 1e-2


def test_block_norm_without_residual_keeps_x():
    dev = device()
    x = torch.randn(5, 96, device=dev)
    got = evo.block_norm(x)
    assert got[0] is x
    x2, h = evo.block_norm(x, alpha=2.0)
    assert torch.equal(x2, 2 * x) and h.shape == x.shape
    copy = torch.empty_like(x)
    assert torch.equal(evo.block_norm(x, x_out=copy)[1], got[1]) and torch.equal(copy, x)
    assert evo.block_norm(x, dtype=BF16)[1].dtype == BF16
    x3, none = evo.block_norm(x, x, pre=None)
    assert none is None and torch.equal(x3, x + x)
    empty = evo.block_norm(x[:0], x[:0])
    assert empty[0].shape == (0, 96) and empty[1].shape == (0, 96)


def test_block_norm_replayed_and_on_another_stream():
    dev, gen = device(), torch.Generator().manual_seed(6)
    c = NormCall(dev, FP32, BF16, 100, 768, "layer", "rms", mods=4, seed=6)
    want = c.run()
    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    got = c.run(stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = c.run(pre=None, pre_gain=None, pre_bias=None, scale=None, shift=None, stream=side)
    torch.cuda.synchronize()
    assert got[1] is None and torch.equal(got[0], want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        held = c.run()
    for r in range(3):
        c.x.copy_(torch.randn((100, 768), generator=gen))
        c.kw["gate"].copy_(torch.randn((4, 768), generator=gen))
        c.kw["mod_rows"].copy_(torch.randint(0, 4, (100,), generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        want = c.run()
        assert torch.equal(held[0], want[0]) and torch.equal(held[1], want[1])


def test_block_norm_offsets_beyond_32_bits():
    dev, gen = device(), torch.Generator().manual_seed(7)
    rows, d = 70000, 64
    base = torch.empty((rows, 65536), dtype=BF16, device=dev)
    x, y, out, h = (base[:, a:a + d] for a in (0, 16384, 32768, 49152))
    x.zero_(), y.zero_()
    some = torch.tensor([0, 1, 40000, 65535, 65536, 69999], device=dev)
    c = NormCall(dev, BF16, BF16, len(some), d, "rms", "rms", seed=7)
    x[some], y[some] = c.x, c.y
    want = c.run()
    c.run(x=x, y=y, x_out=out, h_out=h)
    assert torch.equal(out[some], want[0]) and torch.equal(h[some], want[1])


def test_layer_of_four_bits():
    """The operators in a row as a layer calls them, against the layer in 64 bits:
    norm, projection, attention over a 4-bit cache, projection, norm, feed-forward."""
    from oracle import evo_memory as M
    dev, gen = device(), torch.Generator().manual_seed(8)
    heads, dh, n, past = 4, 64, 16, 200
    d = heads * dh
    x = torch.randn((n, d), generator=gen).to(dev)
    mods = torch.randn((1, 3 * d), generator=gen).mul_(0.2).to(dev)
    ws = {k: evo.Weights4.of((torch.randn(s, generator=gen) * s[1] ** -0.5).to(dev))
          for k, s in (("qkv", (3 * d, d)), ("out", (d, d)), ("up", (4 * d, d)), ("down", (d, 4 * d)))}
    cache = evo.KVCache.empty(5, heads, dh, 64, torch.float4_e2m1fn_x2, dev)
    tab = i32([[3, 1, 0, 4]], dev)
    old = torch.randn((past, 2 * heads, dh), generator=gen).to(dev)
    evo.cache_write(cache, tab, i32([0], dev), old[:, :heads], old[:, heads:])
    table = evo.rope_table(512, dh, device=dev)
    h = evo.block_norm(x)[1]
    qkv = evo.linear4(h, ws["qkv"]).unflatten(1, (3 * heads, dh))
    q = evo.qkv_write(cache, tab, i32([past], dev), qkv[:, :heads], qkv[:, heads:2 * heads], qkv[:, 2 * heads:], table)
    a, _ = evo.chunk_attention(q, cache, tab, i32([past + n], dev), causal=True)
    x1, h1 = evo.block_norm(x, evo.linear4(a.flatten(1), ws["out"]), post="rms", gate=mods[:, :d], scale=mods[:, d:2 * d],
                            shift=mods[:, 2 * d:])
    x2, none = evo.block_norm(x1, evo.linear4(evo.linear4(h1, ws["up"], activation="gelu"), ws["down"]), pre=None)
    assert none is None
    # the same from the definitions; keys and values as the cache holds them
    k, v = (f64(t) for t in evo.cache_read(cache, tab, i32([0], dev), past + n, FP32))
    w = {key: f64(t.values()) for key, t in ws.items()}
    g = [f64(t) for t in mods.split(d, 1)]
    x64 = f64(x)
    y = (E.norm(x64, "rms", None, None, 1e-6) @ w["qkv"].T).reshape(n, 3 * heads, dh)
    q64 = M.norm_rope(y[:, :heads], None, M.rope_table(512, dh), np.arange(past, past + n), "halves", 1e-6)
    o = M.attend(q64, k, v, past, dh ** -0.5, causal=True)[0].reshape(n, d)
    a1, b1 = E.block_norm(x64, o @ w["out"].T, "rms", "rms", None, None, None, None, *g, 1.0, 1e-6)
    want = a1 + E.linear(E.linear(b1, w["up"], None, "gelu"), w["down"])
    # fp32 throughout: each of some 10 operations is off by less than n EPS32 of the
    # row, n up to 1024 summands; the bound leaves 10 of them their worst case
    assert np.max(np.abs(f64(x2) - want)) <= 10 * 1024 * 2.0 ** -24 * np.max(np.abs(want))
