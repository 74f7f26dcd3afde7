"""64-bit reference of the 8-bit integer rows, their product, the norms on both sides of a branch, the 8-bit
cache and its attention: test infrastructure only (numpy, float64), written from the definitions in the ABI header."""
from __future__ import annotations

import numpy as np

from oracle import scaled


def int_rows(x: np.ndarray):
    """(int8 [r][c], fp32 scale [r]) of fp32 values x: each quotient and product rounded to fp32, as defined."""
    x = np.asarray(x, np.float32)
    top = np.max(np.abs(x), axis=1)
    bad, zero = ~np.isfinite(top), top < 2.0 ** -100
    t = np.where(bad | zero, np.float32(1), top)
    up = np.where(bad | zero, np.float32(0), np.float32(127) / t)
    with np.errstate(invalid="ignore"):
        q = np.where(up[:, None] == 0, np.float32(0), np.rint(x * up[:, None]))
    return q.astype(np.int8), np.where(bad, np.float32(np.nan), np.where(zero, np.float32(0), t / np.float32(127)))


def linear(a, sa, w, sw, bias):
    """The layer before its activation, and the size of the product's part of it."""
    p = (a.astype(np.float64) @ w.astype(np.float64).T) * (sa.astype(np.float64)[:, None] * sw.astype(np.float64))
    return p + (0.0 if bias is None else bias.astype(np.float64)), np.abs(p)


def norm(x, eps):
    x = np.asarray(x, np.float64)
    return x / np.sqrt(np.mean(x * x, axis=1, keepdims=True) + eps)


def norm_residual(h, y, post, gate, residual, weight, shift, scale, eps):
    """(h, what was added to it, its modulated norm): rows already matched with their request's gate, shift, scale."""
    h, add = np.asarray(h, np.float64), 0.0
    if y is not None:
        add = norm(y, eps) * (1.0 if post is None else post) * (1.0 if gate is None else gate)
        h = residual * h + add
    a = norm(h, eps)
    if weight is not None:
        a = a * weight
    if scale is not None:
        a = a * (1.0 + scale)
    return h, add, a if shift is None else a + shift


def head_codes(x: np.ndarray):
    """(codes [r][heads][dh], scale bytes [r][heads]) of x [r][heads][dh]."""
    s = scaled.scale_bytes(np.max(np.abs(x), axis=2, initial=0.0))
    with np.errstate(invalid="ignore"):
        v = np.where((s == 255)[..., None], np.nan, x / scaled.powers(s)[..., None])
    return scaled.encode(v), s


def cache_values(codes: np.ndarray, scale: np.ndarray) -> np.ndarray:
    """codes [tokens][heads][dh] with scale bytes [heads][tokens] as values."""
    return scaled.CODES[codes] * scaled.powers(scale).T[..., None]


def attention(q, k, v, cu_q, tok_off, scale):
    """q [rows][heads][dh], k and v [tokens][kv_heads][dh]: (o, sum of |weight * value|, the largest sum of
    |query * key| of the row); rows outside the requests are NaN."""
    rows, heads, dh = q.shape
    group = heads // k.shape[1]
    o, size, score = np.full((rows, heads, dh), np.nan), np.zeros((rows, heads, dh)), np.zeros((rows, heads, 1))
    for b in range(len(cu_q) - 1):
        r, t = slice(cu_q[b], cu_q[b + 1]), slice(tok_off[b], tok_off[b + 1])
        if tok_off[b] == tok_off[b + 1]:
            o[r] = 0
            continue
        for h in range(heads if cu_q[b] < cu_q[b + 1] else 0):
            kh, vh = k[t, h // group], v[t, h // group]
            s = (q[r, h] @ kh.T) * scale
            w = np.exp(s - np.max(s, axis=1, keepdims=True))
            w /= np.sum(w, axis=1, keepdims=True)
            o[r, h], size[r, h] = w @ vh, w @ np.abs(vh)
            score[r, h] = np.max(np.abs(q[r, h]) @ np.abs(kh).T, axis=1, keepdims=True) * scale
    return o, size, score
