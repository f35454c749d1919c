"""The tree attention over the 4-bit cache where its arithmetic is at its ends: scores far apart or
very large, values that are small beside one, weights far below the heaviest.  Against the fp64 oracle on the
values that the cache holds, with bounds that follow from the arithmetic and not from the
values' absolute size."""
import math

import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss
from test_gpu_kv4_attn import _bf16, _fill, _held, _run

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
D = 128
SCALE = 1.0 / math.sqrt(D)


def _wide(a, group):
    return np.repeat(a.astype(np.float64), group, axis=-1)


def _score_error(q, kh, group, scale=SCALE):
    """How far a score may be off [M][Hq]: fp32 sums of exact products of codes, four chained matrix
    products of terms up to 15 s |q| and the minima's share, rounded at most 16 times in all, as 2^-20
    of the sum of the terms' sizes."""
    qa = np.abs(oracle.bf16_bits_to_f64(q))
    size = 15 * _wide(kh[1], group) + np.abs(_wide(kh[2], group))  # [n][Hkv][128]
    G = q.shape[1] // size.shape[1]
    return np.stack([2.0 ** -20 * abs(scale) * (qa[:, h] @ size[:, h // G].T).max(1) for h in range(q.shape[1])], 1)



# --- small values ------------------------------------------------------------------------------------

@pytest.mark.parametrize("size", [0, -6, -9, -12, -16])
@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("M,Hq,Hkv,P", [(1, 128, 128, 20000), (6, 384, 128, 9000), (6, 28, 4, 20000), (8, 16, 2, 200)])
def test_kv4_attention_keeps_small_values_beside_heavy_positions(M, Hq, Hkv, P, group, size):
    """Every wavefront meets a position 2^20 times as heavy as the others, whose value is 0: the output is
    the others' share alone.  Its error is bounded relative to the values, whatever their size: 2^-11 for
    each of three roundings of a weight (with its scale and without), nothing absolute."""
    n, S = P + M, (P + M + 31) // 32 * 32
    rng = np.random.default_rng([M, Hkv, P, -size])
    splits, tiles = ss.subspec_tree_attention_kv4_plan(M, Hq, Hkv, P, 0)
    heavy = np.array([32 * (s * tiles + t) + 7 for s in range(splits) for t in range(min(8, tiles)) if 32 * (s * tiles + t) + 7 < P])
    k, v = rng.standard_normal((n, 1, D)) * 0.05, (rng.standard_normal((n, 1, D)) + 0.5) * 2.0 ** size
    k[heavy] = 20 * math.log(2.0) / math.sqrt(D)  # against a query of ones
    v[heavy] = 0.0
    q = np.ones((M, Hq, D))
    q, k, v = _bf16(q), _bf16(k), _bf16(v)
    mask = np.array([[(1 << M) - 1]] * M, np.uint32)
    all_heads = np.zeros(Hkv, int)
    got = _run(q, *_fill(k[:, all_heads], v[:, all_heads], S, group), mask, M, Hq, Hkv, S, P, 0, group, SCALE)
    kh, vh = _held(k, group), _held(v, group)
    K, V = oracle.kv4_value(*kh), oracle.kv4_value(*vh)
    ref, wabs = oracle.tree_attention_values(q[:, :1], K, V, P, 0, mask, SCALE)
    _, wmin = oracle.tree_attention_values(q[:, :1], K, _wide(vh[2], group), P, 0, mask, SCALE)
    assert 0 < wabs.max() < 2.0 ** size
    err = 2 * _score_error(q[:, :1], kh, group)[..., None]
    tol = 2.0 ** -8 * np.abs(ref) + (err + 2.0 ** -11) * (3 * wabs + wmin)
    assert np.all(np.abs(got - ref) <= tol), float((np.abs(got - ref) / tol).max())
