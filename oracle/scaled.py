"""64-bit reference of the 8-bit rows with block scales, the norm that feeds them, rotary positions and
the product: test infrastructure only (numpy, float64), written from the definitions in the ABI header."""
from __future__ import annotations

import numpy as np


def _decode_table() -> np.ndarray:
    """The value of every e4m3 byte: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b & 128, -v, v)


CODES = _decode_table()


def encode(v: np.ndarray) -> np.ndarray:
    """Nearest e4m3 byte of |v| <= 448, ties to the even code; NaN to 0x7f."""
    v = np.asarray(v, np.float64)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6))) - 3)
    r = np.rint(v / step) * step                       # rint: ties to even, as the mantissa's last bit
    mag = np.abs(np.where(np.isnan(r), 0.0, r))
    b = np.searchsorted(CODES[:127], mag)
    assert np.array_equal(CODES[b], mag)
    return np.where(np.isnan(v), 0x7f, b + 128 * np.signbit(v)).astype(np.uint8)


def stride(cols: int) -> int:
    return (-(-cols // 128) + 3) // 4 * 4


def scale_bytes(top: np.ndarray) -> np.ndarray:
    """Scale byte of blocks of largest magnitude `top` (NaN or inf where a block holds one)."""
    top = np.asarray(top, np.float64)
    bad = ~np.isfinite(top)
    t = np.where(bad | (top == 0), 1.0, top)
    e = np.ceil(np.log2(t / 448.0))
    e = np.where(t > 448.0 * 2.0 ** e, e + 1, e)
    e = np.where(t <= 448.0 * 2.0 ** (e - 1), e - 1, e)
    s = np.clip(np.where(top == 0, -126, e), -126, 127) + 127
    return np.where(bad, 255, s).astype(np.uint8)


def block_tops(x: np.ndarray, block_rows: int) -> np.ndarray:
    r, c = x.shape
    p = np.zeros((-(-r // block_rows) * block_rows, -(-c // 128) * 128))
    p[:r, :c] = np.abs(x)
    p = p.reshape(p.shape[0] // block_rows, block_rows, p.shape[1] // 128, 128)
    return np.max(p, axis=(1, 3))                      # NaN propagates


def spread(per_block: np.ndarray, r: int, c: int, block_rows: int) -> np.ndarray:
    return np.repeat(np.repeat(per_block, block_rows, 0)[:r], 128, 1)[:, :c]


def powers(s: np.ndarray) -> np.ndarray:
    return np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127))


def quant(x: np.ndarray, block_rows: int = 1):
    """(codes [r][c], scale bytes [blocks][ceil(c / 128)]) of x."""
    x = np.asarray(x, np.float64)
    s = scale_bytes(block_tops(x, block_rows))
    with np.errstate(invalid="ignore"):
        v = np.where(spread(s == 255, *x.shape, block_rows), np.nan, x / spread(powers(s), *x.shape, block_rows))
    return encode(v), s


def values(q: np.ndarray, s: np.ndarray, block_rows: int = 1) -> np.ndarray:
    """What codes and their scale bytes (padding allowed) stand for."""
    nk = -(-q.shape[1] // 128)
    return CODES[q] * spread(powers(s[:, :nk]), *q.shape, block_rows)


def rms(h, y, gate, weight, shift, scale, eps):
    """(h + gate y, its modulated norm): rows already matched with their request's gate, shift, scale."""
    h = np.asarray(h, np.float64) + (0.0 if y is None else np.asarray(y, np.float64) * (1.0 if gate is None else gate))
    a = h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    if weight is not None:
        a = a * weight
    if scale is not None:
        a = a * (1.0 + scale)
    return h, a if shift is None else a + shift


def rope(x, pos, dims, theta, step, halves):
    """x [rows][heads][dh] turned by pos [rows][axes]."""
    x = np.asarray(x, np.float64)
    out = x.copy()
    at = 0
    for a, d in enumerate(dims):
        for j in range(d // 2):
            ang = pos[:, a].astype(np.float64) * (step[a] * theta[a] ** (-2.0 * j / d))
            c, n = np.cos(ang)[:, None], np.sin(ang)[:, None]
            u, v = (at + j, at + j + d // 2) if halves else (at + 2 * j, at + 2 * j + 1)
            out[..., u], out[..., v] = x[..., u] * c - x[..., v] * n, x[..., u] * n + x[..., v] * c
        at += d
    return out


def gelu(z):
    return 0.5 * z * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (z + 0.044715 * z ** 3)))

