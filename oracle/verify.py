"""fp64 reference of the verification of a drafted tree with given uniform numbers.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): nothing in the product path may
import this module.

From row 0 on: the row's distribution p = softmax(l / T); its drafted continuations hold the
first part of [0, 1) in index order (a repeated token only at its first index), the other
tokens the rest in token order; the uniform number picks one.  A drafted token continues the
path, any other is the next token.  At T = 0 the largest logit (lowest token) is picked.
"""
from __future__ import annotations

import numpy as np

from .qlinear import bf16_bits_to_f64


def tree_children(parent, token, V: int):
    """Children of every row in index order: entries with a parent that does not come before
    them or a token outside the vocabulary do not count, nor does a sibling's repeat."""
    N = len(parent)
    kids = [[] for _ in range(N + 1)]
    for j in range(N):
        p, t = int(parent[j]), int(token[j])
        if -1 <= p < j and 0 <= t < V and all(int(token[i]) != t for i in kids[p + 1]):
            kids[p + 1].append(j)
    return kids


def tree_verify(logits_bits, parent, token, uniform, temperature: float):
    """(accepted indices, next token, margin): margin is the smallest distance of a uniform
    number to a border of a drafted token's interval that was met on the way (inf: none)."""
    V = logits_bits.shape[1]
    kids = tree_children(parent, token, V)
    row, path, margin = 0, [], float("inf")
    while True:
        l = bf16_bits_to_f64(logits_bits[row])
        if np.isnan(l).any() or np.isposinf(l).any() or np.isneginf(l).all():
            return path, -1, margin
        if temperature == 0.0:
            best = int(np.argmax(l))
            hit = [j for j in kids[row] if int(token[j]) == best]
            if not hit:
                return path, best, margin
        else:
            with np.errstate(over="ignore"):
                p = np.exp((l - l.max()) / temperature)
            p /= p.sum()
            u, f, hit = float(uniform[row]), 0.0, []
            for j in kids[row]:
                f2 = f + p[int(token[j])]
                if f2 > f:
                    margin = min(margin, abs(u - f2), abs(u - f) if f > 0 else np.inf)
                if u < f2:
                    hit = [j]
                    break
                f = f2
            if not hit:
                rest = p.copy()
                rest[[int(token[j]) for j in kids[row]]] = 0.0
                if rest.sum() <= 0.0:
                    return path, max(int(token[j]) for j in kids[row] if p[int(token[j])] > 0), margin
                over = np.nonzero((np.cumsum(rest) > u - f) & (rest > 0))[0]
                return path, int(over[0]) if over.size else int(np.nonzero(rest)[0][-1]), margin
        path.append(hit[0])
        row = hit[0] + 1
