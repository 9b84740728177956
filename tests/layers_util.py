"""Inputs of the tests of the layers around the attention, and the error bounds
that their results are held to."""
import numpy as np
import torch

from oracle import evo_layers as E
from paper_2607_20293_amd import evo
from tests.memory_util import EPS16, EPS32, f64


def random_weights(n_out, n_in, gen, dev, spread=3):
    """4-bit weights of any codes, groups of different sizes, zeros behind n_in."""
    c = -(-n_in // 128)
    codes = torch.randint(0, 256, (n_out, 64 * c), generator=gen, dtype=torch.uint8)
    scales = torch.randint(127 - spread, 128 + spread, (n_out, 4 * c), generator=gen, dtype=torch.uint8)
    k = torch.arange(128 * c)
    codes &= torch.where(k[0::2] < n_in, 15, 0).to(torch.uint8) | torch.where(k[1::2] < n_in, 240, 0).to(torch.uint8)
    scales[:, -(-n_in // 32):] = 0
    return evo.Weights4(codes.to(dev), scales.to(dev), n_in)


def linear_reference(x, weights, bias, act, dtype):
    """(result, bound of the error): n_in products, exact in 32 bits or rounded once
    (fp32 rows), summed in some order: each sum and product within 2 EPS32 of the
    sum of magnitudes; the bias and the activation (whose slope is below 1.2) a few
    more roundings; an output in bf16 one of EPS16."""
    w = E.weights4(weights.codes.view(torch.uint8).cpu().numpy(), weights.scales.view(torch.uint8).cpu().numpy(), weights.n_in)
    x, b = f64(x), None if bias is None else f64(bias)
    want = E.linear(x, w, b, act)
    size = np.abs(x) @ np.abs(w).T + (0 if b is None else np.abs(b))
    bound = 1.2 * 2 * (weights.n_in + 8) * EPS32 * size + 16 * EPS32 * np.abs(want) + 1e-37
    return want, bound + (EPS16 * 1.01 * np.abs(want) if dtype == torch.bfloat16 else 0)


def check(got, want, bound, what):
    got = f64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaNs differ"
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), what
    err = np.abs(got[fine] - want[fine])
    share = np.max(err / np.maximum(bound[fine], 1e-300), initial=0)
    print(f"  {what}: {share:.3f} of its bound", flush=True)
    assert share <= 1, what


class NormCall:
    """A call of block_norm and its reference."""

    def __init__(self, dev, stream, block, rows, d, pre="rms", post=None, affine=True, mods=0, even=False, has_y=True,
                 alpha=1.0, eps=1e-6, seed=0, spread=1.0, offset=0.0):
        gen = torch.Generator().manual_seed(seed)

        def normal(*shape, scale=1.0):
            return torch.randn(shape, generator=gen).mul_(scale)
        self.x = (normal(rows, d, scale=3 * spread) + offset).to(stream).to(dev)
        self.y = (normal(rows, d, scale=spread) + offset).to(block).to(dev) if has_y else None
        self.kw = dict(pre=pre, post=post, alpha=alpha, eps=eps)
        for name, kind in (("pre", pre), ("post", post)):
            for what in ("gain", "bias"):
                if affine and kind:
                    self.kw[f"{name}_{what}"] = (normal(d, scale=0.3) + (what == "gain")).to(dev)
        self.of_row = None
        if mods:
            for name in ("gate", "scale", "shift") if pre else ("gate",):
                if name != "gate" or has_y:
                    self.kw[name] = normal(mods, d, scale=0.4).to(block).to(dev)
            self.of_row = torch.arange(rows) // (rows // mods) if even else torch.randint(0, mods, (rows,), generator=gen)
            if not even:
                self.kw["mod_rows"] = self.of_row.int().to(dev)
        self.block = block

    def run(self, **kw):
        return evo.block_norm(kw.pop("x", self.x), kw.pop("y", self.y), dtype=self.block, **{**self.kw, **kw})

    def reference(self):
        """[(x', bound), (h, bound)].  A norm of a row u: n products and sums, each
        within EPS32 of its part of mean(u^2), halved by the root, a few roundings of
        the result; layer norm takes the mean off first, which is within (n + 4) EPS32
        of mean(|u|), and so is the difference, the error of which is divided by the
        deviation.  An error of u reaches the norm divided by its denominator, once
        directly and once through the denominator."""
        k = {n: (f64(v) if isinstance(v, torch.Tensor) else v) for n, v in self.kw.items() if n != "mod_rows"}
        x, y = f64(self.x), None if self.y is None else f64(self.y)
        d = x.shape[1]
        mod = {n: (k[n][self.of_row.numpy()] if n in k else None) for n in ("gate", "scale", "shift")}
        out, h = E.block_norm(x, y, k["pre"], k["post"], k.get("pre_gain"), k.get("pre_bias"), k.get("post_gain"),
                              k.get("post_bias"), mod["gate"], mod["scale"], mod["shift"], k["alpha"], k["eps"])

        def norm_error(u, du, name):
            """The error of a norm of u that is du off, each row's largest."""
            kind = k[name]
            if kind is None:
                return du
            gain = np.max(np.abs(k.get(name + "_gain", np.ones(1))))
            bias = np.max(np.abs(k.get(name + "_bias", np.zeros(1))))
            v = u - np.mean(u, -1, keepdims=True) if kind == "layer" else u
            den = np.sqrt(np.mean(v * v, -1, keepdims=True) + k["eps"])
            if kind == "layer":
                du = 2 * du + ((d + 4) * np.mean(np.abs(u), -1, keepdims=True) + np.max(np.abs(u), -1, keepdims=True)) * EPS32
            top = np.max(np.abs(v), -1, keepdims=True) / den
            return gain * (du / den * (1 + top) + (d / 2 + 16) * EPS32 * top) + 2 * EPS32 * (bias + gain * top)
        size = np.max(np.abs(k["alpha"] * x), -1, keepdims=True)
        dx = 0
        if y is not None:
            u = E.norm(y, k["post"], k.get("post_gain"), k.get("post_bias"), k["eps"])
            g = 1 if mod["gate"] is None else np.max(np.abs(mod["gate"]), -1, keepdims=True)
            dx = g * norm_error(y, 0, "post")
            size = size + g * np.max(np.abs(u), -1, keepdims=True)
        dx = dx + 4 * EPS32 * size
        half = [EPS16 * 1.01 if t == torch.bfloat16 else EPS32 for t in (self.x.dtype, self.block)]
        found = [(out, dx + half[0] * np.abs(out))]
        if h is not None:
            m = 1 if mod["scale"] is None else 1 + np.max(np.abs(mod["scale"]), -1, keepdims=True)
            t = 0 if mod["shift"] is None else np.max(np.abs(mod["shift"]), -1, keepdims=True)
            top = np.max(np.abs(h), -1, keepdims=True)
            found.append((h, m * norm_error(out, dx, "pre") + 4 * EPS32 * (m * top + t) + half[1] * np.abs(h)))
        return found

    def check(self, what, got=None):
        got = self.run() if got is None else got
        want = self.reference()
        assert (got[1] is None) == (len(want) == 1)
        for name, y, (w, b) in zip(("x", "h"), got, want):
            check(y, w, np.broadcast_to(b, w.shape), f"{what}, {name}")
