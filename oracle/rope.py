"""fp64 reference of the preparation of queries, keys and values from the fused q|k|v
projection: bias, RMS norm per head and position rotation.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): nothing in the product path may
import this module.

Per token and head: add the bias; for query and key heads divide by the root of the mean
square plus eps and multiply by the weight (where there is one); then rotate each pair (a, b) of
the first `rot` dimensions by position * inv_freq[pair].  Pairs are (p, p + rot / 2), or
(2 p, 2 p + 1) where interleaved.
"""
from __future__ import annotations

import numpy as np

from .qlinear import bf16_bits_to_f64


def rotated_pairs(rot: int, interleaved: bool):
    """Index pairs of the rotation, in the order of inv_freq."""
    return [(2 * p, 2 * p + 1) if interleaved else (p, p + rot // 2) for p in range(rot // 2)]


def rope_head(x, weight, eps: float, position: int, inv_freq, rot: int, interleaved: bool):
    """One head row (float64 [128]) normed and rotated."""
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y / np.sqrt(np.mean(y * y) + eps) * weight
    out = y.copy()
    for p, (a, b) in enumerate(rotated_pairs(rot, interleaved)):
        t = float(position) * float(inv_freq[p])
        out[a] = y[a] * np.cos(t) - y[b] * np.sin(t)
        out[b] = y[b] * np.cos(t) + y[a] * np.sin(t)
    return out


def qkv_rope(qkv_bits, bias_bits, q_weight_bits, k_weight_bits, eps: float, positions, inv_freq, rot: int,
             interleaved: bool, Hq: int, Hkv: int):
    """(q [M][Hq][128], k [M][Hkv][128], v [M][Hkv][128]) in float64 from bf16 bit patterns
    (qkv [M][>= (Hq + 2 Hkv) * 128])."""
    M, heads = qkv_bits.shape[0], Hq + 2 * Hkv
    x = bf16_bits_to_f64(qkv_bits[:, : heads * 128]).reshape(M, heads, 128)
    if bias_bits is not None:
        x = x + bf16_bits_to_f64(bias_bits).reshape(1, heads, 128)
    qw = None if q_weight_bits is None else bf16_bits_to_f64(q_weight_bits)
    kw = None if k_weight_bits is None else bf16_bits_to_f64(k_weight_bits)
    out = x.copy()
    for i in range(M):
        for h in range(Hq + Hkv):
            out[i, h] = rope_head(x[i, h], qw if h < Hq else kw, eps, int(positions[i]), inv_freq, rot, interleaved)
    return out[:, :Hq], out[:, Hq:Hq + Hkv], out[:, Hq + Hkv:]
