"""fp64 NumPy reference of the layers around the attention: products with 4-bit
weights and norms around a block.  Shares no code with the library."""
from __future__ import annotations

import numpy as np
from scipy.special import erf

from oracle import evo_memory as M


def weights4(codes, scales, n_in):
    """W [n_out][n_in] of bytes of two codes and exponents of groups of 32."""
    v = M.e2m1_of_bytes(codes, 1)
    unit = np.exp2(np.asarray(scales, np.float64) - 127)
    unit[np.asarray(scales) == 255] = np.nan
    return (v * np.repeat(unit, 32, axis=1))[:, :n_in]


def quantise(w):
    """(values, exponents) of weights: the least power of two that brings a
    group's largest magnitude to 6 or below, between 2^-126 and 2^125."""
    w = np.asarray(w, np.float64)
    n_out, n_in = w.shape
    full = np.zeros((n_out, -(-n_in // 128) * 128))
    full[:, :n_in] = w
    groups = full.reshape(n_out, -1, 32)
    e = np.full(groups.shape[:2], -127)
    for i in range(n_out):
        for g in range(groups.shape[1]):
            top = np.max(np.abs(groups[i, g]))
            if top > 0:
                x = -126
                while x < 125 and top > 6 * 2.0 ** x:
                    x += 1
                e[i, g] = x
    y = np.clip(groups / 2.0 ** e[..., None], -6, 6)
    return (M.e2m1(y) * 2.0 ** e[..., None]).reshape(n_out, -1)[:, :n_in], e + 127


def activate(y, act):
    if act == "silu":
        with np.errstate(over="ignore"):
            return y / (1 + np.exp(-y))
    if act == "gelu":
        return 0.5 * y * (1 + erf(y / np.sqrt(2)))
    return y


def linear(x, w, bias=None, act=None):
    y = np.asarray(x, np.float64) @ w.T
    return activate(y if bias is None else y + np.asarray(bias, np.float64), act)


def norm(u, kind, gain, bias, eps):
    if kind is None:
        return u
    if kind == "layer":
        u = u - np.mean(u, -1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        u = u / np.sqrt(np.mean(u * u, -1, keepdims=True) + eps)
    u = u if gain is None else u * gain
    return u if bias is None else u + bias


def block_norm(x, y, pre, post, pre_gain, pre_bias, post_gain, post_bias, gate, scale, shift, alpha, eps):
    """All float64; gate, scale and shift [rows][d] or None.  (x', h)."""
    out = alpha * x
    if y is not None:
        u = norm(y, post, post_gain, post_bias, eps)
        out = out + (u if gate is None else gate * u)
    if pre is None:
        return out, None
    h = norm(out, pre, pre_gain, pre_bias, eps)
    h = h if scale is None else h * (1 + scale)
    return out, h if shift is None else h + shift
