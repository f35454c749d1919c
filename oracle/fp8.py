"""fp64 reference of 8-bit rows, the product over them and the row operators between two
projections (residual addition with the RMS norm, the gated activation).

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): nothing in the product path may
import this module.  Written from the formulas and the layouts in ``include/subspec.h``.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128


def _table():
    """The value of each e4m3 code (sign, 4 exponent bits of bias 7, 3 fraction bits; all ones is NaN)."""
    out = np.empty(256)
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        v = np.nan if c & 127 == 127 else (f / 8.0 * 2.0 ** -6 if e == 0 else (1 + f / 8.0) * 2.0 ** (e - 7))
        out[c] = -v if c & 128 else v
    return out


E4M3 = _table()


def e4m3_code(v):
    """Codes of |v| <= 448, to nearest, of two equally near the even one; NaN for what is not finite."""
    v = np.asarray(v, np.float64)
    mags = E4M3[:127]
    a = np.where(np.isfinite(v), np.abs(v), 0.0)
    hi = np.clip(np.searchsorted(mags, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - mags[lo], mags[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(np.isfinite(v), code, 127)
    return (code | np.where(np.signbit(v) & np.isfinite(v), 128, 0)).astype(np.uint8)


def fp8_rows(x):
    """(codes uint8 [R][K], scale bytes uint8 [R][K / 128]) of float64 rows."""
    R, K = x.shape
    b = x.reshape(R, K // BLOCK, BLOCK)
    top = np.where(np.isfinite(b), np.abs(b), 0.0).max(-1)
    e = np.full(top.shape, -126)
    for _ in range(256):
        e = np.where(top > 448.0 * np.exp2(e.astype(np.float64)), e + 1, e)
    codes = e4m3_code(b / np.exp2(e.astype(np.float64))[..., None])
    return codes.reshape(R, K), (e + 127).astype(np.uint8)


def fp8_values(codes, scale_bytes):
    """float64 rows that 8-bit rows stand for."""
    R, K = codes.shape
    v = E4M3[codes].reshape(R, K // BLOCK, BLOCK) * np.exp2(scale_bytes.astype(np.float64) - 127.0)[..., None]
    return v.reshape(R, K)


def scale_words(scale_bytes, fill=127):
    """uint32 [ceil(K / 512)][R] from bytes [R][K / 128]; bytes past the last block hold `fill`."""
    R, B = scale_bytes.shape
    out = np.full((R, (B + 3) // 4 * 4), fill, np.uint32)
    out[:, :B] = scale_bytes
    w = out.reshape(R, -1, 4)
    return np.ascontiguousarray((w[..., 0] | w[..., 1] << 8 | w[..., 2] << 16 | w[..., 3] << 24).T)


def scale_bytes(words, K):
    """bytes [R][K / 128] from words [ceil(K / 512)][R]."""
    w = np.asarray(words).view(np.uint32).T[..., None] >> np.array([0, 8, 16, 24], np.uint32) & 255
    return w.reshape(w.shape[0], -1)[:, : K // BLOCK].astype(np.uint8)


def weight_tiles(codes):
    """Codes [N][K] in the order of weight tiles, code by code."""
    N, K = codes.shape
    out = np.empty(N * K, np.uint8)
    n, k = np.arange(N)[:, None], np.arange(K)[None, :]
    at = 2048 * (n // 16 * (K // 128) + k // 128) + 1024 * (k % 128 // 64) + 256 * (k % 64 // 16) + 16 * (n % 16) + k % 16
    out[at] = codes
    return out


def add_norm(x, residual, weight, eps: float):
    """(s, y) of float64 rows."""
    s = x if residual is None else x + residual
    return s, s / np.sqrt(np.mean(s * s, -1, keepdims=True) + eps) * weight


def silu_mul(g, u):
    with np.errstate(over="ignore"):
        return np.where(g >= 0, g / (1.0 + np.exp(-np.abs(g))), g * np.exp(-np.abs(g)) / (1.0 + np.exp(-np.abs(g)))) * u
