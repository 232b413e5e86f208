"""Plain 64-bit forms of what a decoder does between its projections: the key-value cache, attention of one token over it, and
the norms around a block.  Test infrastructure: numpy only, slow, sharing no code with the library."""
from __future__ import annotations

import numpy as np


def bf16(x):
    """Nearest bf16 (ties to even) of fp64 or fp32 values, as fp64; NaN and infinities stay."""
    f = np.asarray(x, np.float64)
    u = f.astype(np.float32)
    # fp64 -> fp32 -> bf16 would round twice: make the fp32 step sticky (odd last bit where it was inexact)
    b = u.view(np.uint32).astype(np.uint64)
    with np.errstate(invalid="ignore"):
        over = np.abs(u.astype(np.float64)) > np.abs(f)
        inexact = (u.astype(np.float64) != f) & np.isfinite(f) & np.isfinite(u)
    b = np.where(over & inexact, b - 1, b)          # truncated towards zero
    b = np.where(inexact, b | 1, b)
    r = (b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000
    out = r.astype(np.uint32).view(np.float32).astype(np.float64)
    return np.where(np.isfinite(u), out, u)


def rope(x, cos, sin):
    """x [tokens, heads, dim], cos, sin [tokens, dim / 2] fp32: the pinned arithmetic, every product and sum rounded to fp32, one
    rounding to bf16."""
    h = x.shape[-1] // 2
    a, b = x[..., :h].astype(np.float32), x[..., h:].astype(np.float32)
    c, s = cos[:, None].astype(np.float32), sin[:, None].astype(np.float32)
    return bf16(np.concatenate([a * c - b * s, b * c + a * s], -1))


def quantise(x):
    """Codes and gamma of rows x [..., dim] (Eq. 7-9 per row)."""
    x32 = np.asarray(x, np.float32)
    amax = np.maximum(np.abs(x32).max(-1), np.float32(1e-5))
    gamma = (np.float32(128) / amax).astype(np.float32)
    codes = np.clip(np.rint(x32 * gamma[..., None]), -128, 127)
    bad = ~np.isfinite(x32).all(-1)
    gamma = np.where(bad, np.float32(np.nan), gamma)
    codes = np.where(bad[..., None], 0, codes)
    return codes.astype(np.int8), gamma


def attend(q, k, v, scale):
    """q [heads, dim] over k, v [positions, kv heads, dim]: output, log of the weights' sum, sum |p v| / sum p (the size that errors of
    the weights scale with) and max over positions of scale sum |q k|."""
    heads, dim = q.shape
    n, kv, _ = k.shape
    out, lse, spread = np.zeros((heads, dim)), np.full(heads, -np.inf), np.zeros((heads, dim))
    big = np.zeros(heads)
    if n == 0:
        return out, lse, spread, big
    for h in range(heads):
        kh, vh = k[:, h * kv // heads], v[:, h * kv // heads]
        s = scale * (kh @ q[h])
        m = s.max()
        if m == -np.inf:
            continue
        p = np.exp(s - m)
        out[h], spread[h] = p @ vh / p.sum(), p @ np.abs(vh) / p.sum()
        lse[h], big[h] = m + np.log(p.sum()), (abs(scale) * (np.abs(kh) @ np.abs(q[h]))).max()
    return out, lse, spread, big


def rms(z, eps):
    return z / np.sqrt((z * z).mean(-1, keepdims=True) + eps)


def block_norm(x, y, post, gate, pre, res_scale, eps):
    """s and h (None without pre), unrounded."""
    s = res_scale * x
    if y is not None:
        u = rms(y, eps) * post if post is not None else y
        s = s + (gate if gate is not None else 1.0) * u
    return s, None if pre is None else rms(s, eps) * pre


def rms_backward(g, z, eps):
    """Gradient of rms(z) . g with respect to z, row by row."""
    n = z.shape[-1]
    r = 1 / np.sqrt((z * z).mean(-1, keepdims=True) + eps)
    return r * g - z * (g * z).sum(-1, keepdims=True) * r ** 3 / n


def block_norm_backward(ds, dh, s, y, post, gate, pre, res_scale, eps):
    """dict of dx, dy, dpost, dgate (per feature), dpre; absent inputs None."""
    out = {}
    g = np.zeros_like(ds if ds is not None else dh) if ds is None else ds.copy()
    if dh is not None:
        g = g + rms_backward(dh * pre, s, eps)
        out["dpre"] = (dh * rms(s, eps)).sum(0)
    out["dx"] = res_scale * g
    e = g if gate is None else g * gate
    if gate is not None:
        out["dgate"] = (g * (rms(y, eps) * post if post is not None else y)).sum(0)
    if post is not None:
        out["dpost"] = (e * rms(y, eps)).sum(0)
        e = rms_backward(e * post, y, eps)
    out["dy"] = e
    return out
