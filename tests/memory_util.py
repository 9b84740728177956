"""Inputs of the long-memory tests and the error bounds that their results are
held to."""
import numpy as np
import torch

from oracle import evo_memory as M
from paper_2607_20293_amd import evo

FORMATS = {"fp32": torch.float32, "bf16": torch.bfloat16, "int8": torch.int8, "fp8": torch.float8_e4m3fn}
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS32, EPS16 = 2.0 ** -24, 2.0 ** -8      # half a unit in the last place, relative (bf16 has 8 significant bits)


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def i32(v, dev):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=dev)


def pool(fmt, pages, heads, size, dh, dev, gen, spread=1.0):
    """Tensors of a cache that holds random values everywhere."""
    def normal(*shape):
        return torch.randn(shape, generator=gen).mul_(spread)
    k, v = normal(pages, heads, size, dh), normal(pages, heads, dh, size)
    if fmt in ("fp32", "bf16"):
        return [k.to(FORMATS[fmt]).to(dev), v.to(FORMATS[fmt]).to(dev), None, None]
    codes = [(x * 30).clamp(-127, 127) for x in (k, v)]
    codes = [(x.round() if fmt == "int8" else x).to(FORMATS[fmt]).to(dev) for x in codes]
    scales = [(torch.rand((pages, heads, size), generator=gen) + 0.5).div_(30).to(dev) for _ in range(2)]
    return codes + scales


def table_for(lengths, size, extra, rng):
    """A page table whose pages lie in random order, and the number of pages."""
    need = [max(1, -(-int(n) // size)) for n in lengths]
    pages = sum(need) + extra
    order = rng.permutation(pages)
    wide = max(need)
    tab, at = np.zeros((len(need), wide), np.int32), 0
    for s, n in enumerate(need):
        tab[s, :n] = order[at:at + n]
        at += n
    return tab, pages


class Call:
    """One attention call on the GPU and its reference."""

    def __init__(self, dev, dtype, fmt, rows, lengths, heads, kv_heads, dh, size=64, seed=0, **kw):
        self.rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        self.dev, self.dtype, self.fmt, self.kw = dev, dtype, fmt, dict(kw)
        self.rows, self.lengths, self.dh = list(rows), list(lengths), dh
        self.tab, pages = table_for(lengths, size, 2, self.rng)
        self.tensors = pool(fmt, pages, kv_heads, size, dh, dev, gen)
        self.q = torch.randn((sum(rows), heads, dh), generator=gen).mul_(1.5).to(DTYPES[dtype]).to(dev)
        self.cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.slopes = None
        if self.kw.pop("bias", False):
            self.slopes = torch.tensor([2.0 ** (-4.0 * (h + 1) / heads) for h in range(heads)])

    def run(self, q=None, **more):
        cache = evo.KVCache(*self.tensors)
        kw = {k: v for k, v in self.kw.items() if k not in ("prefix", "starts")}
        for name in ("prefix", "starts"):
            if self.kw.get(name) is not None:
                kw[name] = i32(self.kw[name], self.dev)
        if self.slopes is not None:
            kw["slopes"] = self.slopes.to(self.dev)
        return evo.chunk_attention(self.q if q is None else q, cache, i32(self.tab, self.dev), i32(self.lengths, self.dev),
                                   i32(self.cu, self.dev), max(self.rows), **{**kw, **more})

    def reference(self):
        """(out, lse, bound of out's error, bound of lse's error).

        z's error: dh products summed in fp32, each within EPS32 of its part of
        sum |q k|, doubled; scaling, cap and bias round a few times relative to
        their own size.  A term exp(z) is then off by the factor 1 + 2 dz, sums
        over n keys by n EPS32.  With bf16 products each term is rounded once
        more and a bf16 output once, each by at most EPS16 and by half of it
        in the mean: held to EPS16 of the largest value in all."""
        k, v, ks, vs = self.tensors
        arr = [f64(k), f64(v)] + [None if s is None else f64(s) for s in (ks, vs)]
        q, dh = f64(self.q), self.dh
        scale = self.kw.get("scale") or dh ** -0.5
        cap, window = self.kw.get("cap", 0.0), self.kw.get("window", 0)
        slopes = None if self.slopes is None else self.slopes.double().numpy()
        outs, lses, bo, bl = [], [], [], []
        for s, (n, length) in enumerate(zip(self.rows, self.lengths)):
            kk, vv = M.gather(*arr, self.tab, s, length)
            start = length - n if self.kw.get("starts") is None else self.kw["starts"][s]
            prefix = 0 if self.kw.get("prefix") is None else self.kw["prefix"][s]
            x = q[self.cu[s]:self.cu[s + 1]]
            o, e = M.attend(x, kk, vv, start, scale, self.kw.get("causal", False), window, cap, slopes, prefix)
            fine_k, fine_v = np.where(np.isfinite(kk), kk, 0), np.where(np.isfinite(vv), vv, 0)
            products = np.max(np.abs(x), initial=0) * np.max(np.sum(np.abs(fine_k), -1), initial=0) * abs(scale)
            far = 0 if slopes is None else np.max(slopes) * (abs(start) + n + length)
            dz = 2 * EPS32 * (dh * products + 8 * (min(products, cap) if cap else products) + 8 * cap + 4 * far)
            top = np.max(np.abs(fine_v), initial=0)
            out_bound = top * (2 * (2 * dz + 2 * (length + 64) * EPS32) + (EPS16 * 1.01 if self.dtype == "bf16" else 0))
            outs.append(o)
            lses.append(e)
            bo.append(np.full(o.shape, out_bound))
            bl.append(np.full(e.shape, 2 * dz + (length + 64) * EPS32 + 1e-6 + 4 * EPS32 * products))
        return tuple(np.concatenate(t) for t in (outs, lses, bo, bl))

    def check(self, what, got=None, reference=None):
        out, lse = self.run() if got is None else got
        want, want_lse, bo, bl = self.reference() if reference is None else reference
        out, lse = f64(out), f64(lse)
        assert np.array_equal(np.isnan(out), np.isnan(want)), f"{what}: NaNs differ"
        assert np.array_equal(np.isneginf(lse), np.isneginf(want_lse)), f"{what}: empty rows differ"
        fine, fine_l = np.isfinite(want), np.isfinite(want_lse)
        assert np.array_equal(out[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
        err, err_l = np.abs(out - np.where(fine, want, 0))[fine], np.abs(lse - np.where(fine_l, want_lse, 0))[fine_l]
        bo, bl = bo[fine], bl[fine_l]

        def share(e, b):
            return np.max(e[b > 0] / b[b > 0], initial=0)
        print(f"  {what}: out {share(err, bo):.3f}, lse {share(err_l, bl):.3f} of their bounds", flush=True)
        assert np.all(err <= bo) and np.all(err_l <= bl), what
