"""Reference of the key/value cache held in 4 bits and of the tree attention over it.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): nothing in the product path may
import this module.

Per group of a row: m = fp16(min x), s = fp16((max x - min x) / 15), codes
clamp(rint((x - m) / s), 0, 15), each step in fp32 as the interface states it; a code stands for
m + s c, formed here in float64.  The byte layout is the one of ``include/subspec.h``.
Attention is the softmax-weighted sum over each query's visible positions in float64.
"""
from __future__ import annotations

import numpy as np

from .qlinear import bf16_bits_to_f64
from .tree_attn import visible_positions


def kv4_quantize(x, group: int):
    """Codes (uint8 [..., 128]), scales and minima (float16 [..., 128 / group]) of rows x."""
    x = np.nan_to_num(np.asarray(x, dtype=np.float32), nan=0.0, posinf=65504.0, neginf=-65504.0)
    x = np.clip(x, np.float32(-65504), np.float32(65504)).reshape(*x.shape[:-1], 128 // group, group)
    lo, hi = x.min(-1), x.max(-1)
    lo = np.where((lo == 0) & ((x == 0) & np.signbit(x)).any(-1), np.float32(-0.0), lo)  # -0 lies below 0
    m = lo.astype(np.float16)
    s = ((hi - lo) / np.float32(15)).astype(np.float16)
    d = x - m.astype(np.float32)[..., None]
    s32 = s.astype(np.float32)[..., None]
    q = np.divide(d, s32, out=np.zeros_like(d), where=s32 > 0)
    codes = np.clip(np.rint(q), 0, 15).astype(np.uint8)
    return codes.reshape(*x.shape[:-2], 128), s, m


def kv4_value(codes, s, m):
    """m + s c in float64."""
    G = s.shape[-1]
    c = codes.reshape(*codes.shape[:-1], G, 128 // G).astype(np.float64)
    return (m.astype(np.float64)[..., None] + s.astype(np.float64)[..., None] * c).reshape(codes.shape)


def kv4_places(S: int, group: int, value: bool):
    """For every position < S and dimension: the byte and bit of its code within a head's
    buffer, and the byte of its scale (the minimum is 16 bytes on)."""
    G = 128 // group
    p = np.arange(S)[:, None]
    d = np.arange(128)[None, :]
    w = p % 32
    if value:
        byte = 1024 * (d // 64) + 16 * (16 * (w % 16 // 4) + d % 16) + 4 * (d % 64 // 16)
        e = w % 4 + 4 * (w // 16)
    else:
        byte = 1024 * (w // 16) + 16 * (16 * (d % 32 // 8) + w % 16) + 4 * (d // 32)
        e = d % 8
    bit = 16 * (e % 2) + 4 * (e // 2)
    tile = p // 32 * (2048 + 128 * G)
    scale = tile + 2048 + 32 * (G * (w % 16 // 4) + d // group) + 2 * (w % 4 + 4 * (w // 16))
    return np.broadcast_arrays(tile + byte + bit // 8, bit % 8, scale)


def kv4_bytes(Hkv: int, S: int, group: int) -> int:
    return Hkv * (S // 32) * (2048 + 128 * (128 // group))


def kv4_write(cache, positions, codes, s, m, group: int, value: bool):
    """Writes rows (codes [n][Hkv][128], s, m [n][Hkv][G]) at `positions` of a cache's bytes
    [Hkv][bytes of a head], in place."""
    Hkv, size = cache.shape
    S = size // (2048 + 128 * (128 // group)) * 32
    byte, bit, scale = kv4_places(S, group, value)
    for i, pos in enumerate(positions):
        for h in range(Hkv):
            for d in range(128):
                b = byte[pos, d]
                cache[h, b] = (int(cache[h, b]) & ~(0xF << int(bit[pos, d]))) | (int(codes[i, h, d]) << int(bit[pos, d]))
            for g in range(128 // group):
                at = scale[pos, g * group]
                cache[h, at:at + 2] = np.frombuffer(s[i, h, g].tobytes(), np.uint8)
                cache[h, at + 16:at + 18] = np.frombuffer(m[i, h, g].tobytes(), np.uint8)


def kv4_read(cache, group: int, value: bool):
    """(codes [S][Hkv][128], s, m [S][Hkv][G]) of a cache's bytes [Hkv][bytes of a head]."""
    Hkv, size = cache.shape
    G = 128 // group
    S = size // (2048 + 128 * G) * 32
    byte, bit, scale = kv4_places(S, group, value)
    codes = np.empty((S, Hkv, 128), np.uint8)
    s, m = np.empty((S, Hkv, G), np.float16), np.empty((S, Hkv, G), np.float16)
    for h in range(Hkv):
        codes[:, h] = (cache[h][byte] >> bit) & 15
        half = np.ascontiguousarray(cache[h]).view(np.float16)
        s[:, h] = half[scale[:, ::group] // 2]
        m[:, h] = half[scale[:, ::group] // 2 + 8]
    return codes, s, m


def tree_attention_values(q_bits, K, V, P: int, T: int, mask_bits, scale: float):
    """Output [M][Hq][128] (float64) over keys and values [positions][Hkv][128] (float64), and
    sum_j p_j |v_j| of the same shape."""
    M, Hq, _ = q_bits.shape
    Hkv = K.shape[1]
    q = bf16_bits_to_f64(q_bits)
    out, wabs = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(M):
        pos = visible_positions(mask_bits, i, P, T, M)
        if pos.size == 0:
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            sc = (K[pos, g] @ q[i, h]) * scale
            p = np.exp(sc - sc.max())
            p /= p.sum()
            out[i, h] = p @ V[pos, g]
            wabs[i, h] = p @ np.abs(V[pos, g])
    return out, wabs
