"""The tree attention over the 4-bit cache where its arithmetic is at its ends: scores far apart or
very large, values that are small beside one, weights far below the heaviest.  Against the fp64 oracle on the
values that the cache holds, with bounds that follow from the arithmetic and not from the
values' absolute size."""
import math

import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss
from paper_2509_18344_amd import synth
from oracle.tree_attn import visible_positions
from test_gpu_kv4_attn import _bf16, _check, _fill, _held, _run

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


def _half_step(x):
    """Half the distance of bf16 numbers (8 bits) at |x|."""
    return np.ldexp(1.0, np.frexp(np.maximum(np.abs(x), 2.0 ** -126))[1] - 9)


# --- very large scores -----------------------------------------------------------------------------

LARGE = [
    (6, 28, 4, 100, 42),    # a workgroup takes a head whole
    (6, 28, 4, 2048, 60),   # ranges, tiles in registers
    (8, 16, 2, 3000, 90),   # 64 rows a head
    (1, 128, 128, 2500, 0),   # five tiles a wavefront
    (1, 128, 128, 5000, 0),   # ten, in a ring
    (6, 64, 32, 5000, 20),
]


@pytest.mark.parametrize("q_size,k_size", [(1e3, 1e2), (1e5, 1e3), (1e6, 3e3), (1e8, 1e4), (1e30, 1e4), (1e36, 1e4)])
@pytest.mark.parametrize("M,Hq,Hkv,P,T", LARGE)
def test_kv4_attention_of_very_large_scores_is_the_largest_ones_value(M, Hq, Hkv, P, T, q_size, k_size):
    """Scores of 2^17 and more, where fp32 holds no fraction of them: a row whose largest score
    lies further above the second than both may be off gets that position's value."""
    group = 64 if P % 3 else 128
    n, S = P + T + M, (P + T + M + 31) // 32 * 32
    rng = np.random.default_rng([M, Hq, P, int(math.log10(q_size))])
    q = _bf16(rng.standard_normal((M, Hq, D)) * q_size)
    own = min(Hkv, 2)
    k, v = rng.standard_normal((n, own, D)) * k_size, rng.standard_normal((n, own, D)) + 0.5
    if q_size in (1e5, 1e30):
        v *= 2.0 ** 11  # value scales far above 1
    k, v = (_bf16(a)[:, np.arange(Hkv) % own] for a in (k, v))
    mask = synth.tree_levels_mask(T, 6, M, 5)
    got = _run(q, *_fill(k, v, S, group), mask, M, Hq, Hkv, S, P, T, group, SCALE)
    assert np.isfinite(got).all()
    some = sorted({0, Hkv // 2, Hkv - 1})
    G = Hq // Hkv
    heads = [g * G + i for g in some for i in range(G)]
    q, got, k, v = q[:, heads], got[:, heads], k[:, some], v[:, some]
    kh, vh = _held(k, group), _held(v, group)
    K, V = oracle.kv4_value(*kh), oracle.kv4_value(*vh)
    err = _score_error(q, kh, group)
    apart = 0
    for i in range(M):
        pos = visible_positions(mask, i, P, T, M)
        for h in range(len(heads)):
            sc = K[pos, h // G] @ oracle.bf16_bits_to_f64(q)[i, h] * SCALE
            first, second = np.argsort(sc)[-1:-3:-1]
            if sc[first] - sc[second] < 2 * err[i, h] + 30:  # e^-30: the others' share is nothing
                continue
            apart += 1
            ref = V[pos[first], h // G]
            tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * np.abs(V).max()
            assert np.all(np.abs(got[i, h] - ref) <= tol), (i, h, np.abs(got[i, h] - ref).max())
    assert apart > 0.8 * M * len(heads)


@pytest.mark.parametrize("q_size", [1e3, 1e5, 1e7, 1e9])
@pytest.mark.parametrize("M,Hq,Hkv,P,T", LARGE)
def test_kv4_attention_of_equal_large_scores_is_their_values_mean(M, Hq, Hkv, P, T, q_size):
    """Positions with the same key have the same score to the bit, however large, and weigh the
    same wherever they lie: in other tiles, wavefronts and ranges."""
    group, n = 64, P + T + M
    S = (n + 31) // 32 * 32
    rng = np.random.default_rng([M, Hq, P])
    q = _bf16(np.abs(rng.standard_normal((M, Hq, D)) + 2.0) * q_size)
    k = -np.abs(rng.standard_normal((n, 1, D))) * 1e3
    alike = np.unique(np.concatenate([[3, P - 1], rng.choice(P, 5, replace=False)]))
    k[alike] = np.abs(rng.standard_normal((1, 1, D))) * 1e3  # scores above every other
    v = rng.standard_normal((n, 1, D))
    k, v = (_bf16(a)[:, np.zeros(Hkv, int)] for a in (k, v))
    mask = synth.tree_levels_mask(T, 6, M, 5)
    got = _run(q, *_fill(k, v, S, group), mask, M, Hq, Hkv, S, P, T, group, SCALE)
    ref = oracle.kv4_value(*_held(v[:, :1], group))[alike, 0]
    # the weights are equal, but each rounds with its value's scale: 2^-11 of the parts of a value
    tol = 2.0 ** -8 * np.abs(ref.mean(0)) + 2.0 ** -10 * (np.abs(ref).mean(0) + 4.0)
    assert np.all(np.abs(got - ref.mean(0)) <= tol), np.abs(got - ref.mean(0)).max()


# --- small values ------------------------------------------------------------------------------------

@pytest.mark.parametrize("size", [0, -6, -9, -12, -16])
@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("M,Hq,Hkv,P,each", [(1, 128, 128, 20000, True), (6, 384, 128, 9000, True), (6, 28, 4, 20000, True),
                                             (8, 16, 2, 200, True), (6, 40, 8, 40000, True), (6, 40, 8, 40000, False),
                                             (1, 8, 8, 90000, False)])
def test_kv4_attention_keeps_small_values_beside_heavy_positions(M, Hq, Hkv, P, each, group, size):
    """Every wavefront (or one) meets a position 2^20 times as heavy as the others, whose value is 0: the
    output is the others' share alone.  Its error is bounded relative to the values, whatever their size: 2^-11 for
    each of three roundings of a weight (with its scale and without), nothing absolute."""
    n, S = P + M, (P + M + 31) // 32 * 32
    rng = np.random.default_rng([M, Hkv, P, -size])
    splits, tiles = ss.subspec_tree_attention_kv4_plan(M, Hq, Hkv, P, 0)
    heavy = np.array([32 * (s * tiles + t) + 7 for s in range(splits) for t in range(min(8, tiles)) if 32 * (s * tiles + t) + 7 < P])
    heavy = heavy if each else heavy[len(heavy) // 2:][:1]
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


# --- the weights' bits -------------------------------------------------------------------------------

@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("M,Hq,Hkv,P,T", [(6, 28, 4, 0, 26), (1, 8, 8, 40, 0), (8, 16, 2, 3, 90), (4, 128, 128, 11, 8),
                                          (6, 28, 4, 2048, 60), (1, 128, 128, 2500, 0)])
def test_kv4_attention_rounds_once(M, Hq, Hkv, P, T, group):
    """Values of either sign, so that outputs are small beside the terms they are sums of: an output
    is the bf16 number next to the exact one but for the scores' error and 2^-17 of the terms' sizes
    (a weight carries 21 bits, its product with the scale 20, sums are in fp32)."""
    n, S = P + T + M, (P + T + M + 31) // 32 * 32
    rng = np.random.default_rng([M, Hq, P, T])
    q, k = rng.standard_normal((M, Hq, D)) * 0.2, rng.standard_normal((n, 1, D)) * 0.2
    v = np.where(rng.random((n, 1, D)) < 0.5, -1.0, 1.0) * 2.0 ** rng.integers(-2, 3, (n, 1, 1))
    q, k, v = _bf16(q), _bf16(k), _bf16(v)
    mask = rng.integers(0, 2 ** 32, (M, (T + M + 31) // 32), dtype=np.uint64).astype(np.uint32)
    mask[:, 0] |= 1
    heads = np.zeros(Hkv, int)
    got = _run(q, *_fill(k[:, heads], v[:, heads], S, group), mask, M, Hq, Hkv, S, P, T, group, SCALE)
    q, got = q[:, :28], got[:, :28]
    kh, vh = _held(k, group), _held(v, group)
    ref, wabs = oracle.tree_attention_values(q, oracle.kv4_value(*kh), oracle.kv4_value(*vh), P, T, mask, SCALE)
    # the sums run over the minimum's and the codes' parts of a value: up to three times its size
    err = (2 * _score_error(q, kh, group)[..., None] + 2.0 ** -17) * 3 * wabs
    tol = _half_step(np.abs(ref) + err) + err
    off = np.abs(got - ref) > tol
    assert not off.any(), (int(off.sum()), off.size, float((np.abs(got - ref) / tol).max()))


# --- products of very different sizes beside each other --------------------------------------------------

@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("heads", [1, 4, 30, 64])
def test_kv4_attention_keeps_light_weights_beside_a_heavy_one(heads, group):
    """One position of every eight that a matrix product takes together is 2^12 times as heavy as the
    others and 0 in most dimensions, though none of its codes is: what the others add there stands to
    2^-19 of what the products sum over."""
    M, P = 1, 31
    n, S = P + M, 32
    rng = np.random.default_rng([heads, group])
    heavy = np.array([1, 5, 9, 13])
    k, v = rng.standard_normal((n, 1, D)) * 0.05, rng.standard_normal((n, 1, D))
    k[heavy] = 12 * math.log(2.0) / math.sqrt(D)  # against a query of ones
    v[heavy] = 0.0
    v[heavy, :, ::64], v[heavy, :, 1::64] = -1.0, 0.875  # minimum -1, scale 1 / 8: a 0 is code 8
    q = _bf16(np.ones((M, heads, D)))
    k, v = _bf16(k), _bf16(v)
    mask = np.array([[1]], np.uint32)
    got = _run(q, *_fill(k, v, S, group), mask, M, heads, 1, S, P, 0, group, SCALE)
    kh, vh = _held(k, group), _held(v, group)
    K, V = oracle.kv4_value(*kh), oracle.kv4_value(*vh)
    zero = (V[heavy, 0] == 0).all(0)
    assert zero.sum() == 124 and (vh[0][heavy][:, 0, zero] == 8).all()
    ref, wabs = oracle.tree_attention_values(q, K, V, P, 0, mask, SCALE)
    _, parts = oracle.tree_attention_values(q, K, _wide(vh[1], group) * vh[0] + np.abs(_wide(vh[2], group)), P, 0, mask, SCALE)
    tol = _half_step(ref) + 2 * _score_error(q, kh, group)[..., None] * wabs + 2.0 ** -19 * parts
    off = (np.abs(got - ref) > tol)[..., zero]
    assert not off.any(), (int(off.sum()), off.size, float((np.abs(got - ref) / tol)[..., zero].max()))


@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("M,P", [(1, 11), (6, 700)])
def test_kv4_attention_keeps_small_dimensions_of_a_query_beside_a_large_one(M, P, group):
    """One dimension of a query is thousands of times the others, and the keys agree in it (code 1):
    scores differ by the others alone, and by the fp32 roundings of sums of that size."""
    heads, n, S = min(28, 64 // M), P + M, (P + M + 31) // 32 * 32
    rng = np.random.default_rng([M, P, group])
    q = rng.standard_normal((M, heads, D)) * 3.0
    q[..., 8::group] = 2.0 ** 13
    k = rng.uniform(-1.0, 1.0, (n, 1, D))
    k[..., 0::group], k[..., 1::group] = -1.0, 0.875  # minimum -1, scale 1 / 8
    k[..., 8::group] = -0.875                       # code 1
    v = rng.standard_normal((n, 1, D))
    q, k, v = _bf16(q), _bf16(np.clip(k, -1.0, 0.875)), _bf16(v)
    mask = rng.integers(0, 2 ** 32, (M, 1), dtype=np.uint64).astype(np.uint32)
    got = _run(q, *_fill(k, v, S, group), mask, M, heads, 1, S, P, 0, group, SCALE)
    kh, vh = _held(k, group), _held(v, group)
    assert (kh[0][..., 8::group] == 1).all() and (_wide(kh[1], group) == 0.125).all()
    ref, wabs = oracle.tree_attention_values(q, oracle.kv4_value(*kh), oracle.kv4_value(*vh), P, 0, mask, SCALE)
    # sums of 16 groups of eight products and what precedes them, rounded once each; the minima's share, three times
    qa = np.abs(oracle.bf16_bits_to_f64(q))
    err = SCALE * (16 * 2.0 ** -24 * (qa @ (0.125 * kh[0][:, 0]).T).max(-1) + 3 * 2.0 ** -24 * qa.sum(-1))[..., None]
    tol = _half_step(np.abs(ref) + 2 * err * wabs) + (2 * err + 2.0 ** -17) * 3 * wabs
    off = np.abs(got - ref) > tol
    assert not off.any(), (int(off.sum()), off.size, float((np.abs(got - ref) / tol).max()))


# --- one query tile in a ring -----------------------------------------------------------------------------

@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("M,Hq,Hkv,P,T,q_scale", [(1, 128, 128, 5000, 0, 1.0), (1, 64, 64, 9300, 40, 2.0), (5, 96, 48, 15000, 33, 1.0),
                                                  (16, 64, 64, 9500, 90, 1.5)])
def test_kv4_attention_of_few_rows_over_many_tiles(M, Hq, Hkv, P, T, q_scale, group):
    """Up to 16 rows a head and nine tiles a wavefront and more."""
    splits, tiles = ss.subspec_tree_attention_kv4_plan(M, Hq, Hkv, P, T)
    assert splits > 1 and -(-tiles // 8) >= 9
    _check(M, Hq, Hkv, P, T, group, P + T, q_scale=q_scale, what=f"M={M} Hkv={Hkv} P={P} group={group}")
