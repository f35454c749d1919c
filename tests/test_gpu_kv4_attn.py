"""GPU parity of the tree attention over the 4-bit cache against the fp64 oracle on the
values that the cache holds.

Tolerance, from the arithmetic.  A value is m + s c.  The kernel rounds a weight p to fp16 for
the sum of weights and for the minima, and the product of that and s once more for the
codes: 2^-11 relative each, so 2^-11 (sum_j p_j |v_j| + |o|) for the first and 2^-11 sum_j p_j
|v_j - m_j| for the second, together at most 2^-11 sum_j p_j (3 |v_j| + |m_j|).  Below fp16's normal
range a rounding is 2^-25 absolute, where the heaviest weight of the row is at least 2^(8 - E), 2^E
(E >= 0) above the largest scale of a value.  Half of the positions' weights are scaled by 2^-4 before the
product with s (their codes are 16 times as large), so there three roundings add up: of p for the
minima, of p / 16, and of its product with s: L 2^(E - 33) (max |v| + 16 * 15 (max s + 1)).
Scores: fp32 sums of exact products of codes, 4 chained matrix products of terms up to 15 s |q|, at
most four roundings each, and the minima's share: 2^-20 scale sum_d (15 s + |m|) |q_d| absolute, plus 2^-21 of the largest
score for the exponent's argument; either changes a weight by as much relatively, and the
output by twice that times sum_j p_j |v_j|.  Second products sum in fp32: 2^-18 of sum_j p_j (15 s_j + |m_j|).  The output
is rounded to bf16: 2^-8."""
import math

import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss
from paper_2509_18344_amd import synth

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"
D = 128


def _dev(bits):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(DEV)


def _bf16(x):
    return synth.bf16_bits(torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16))


def _fill(k, v, S, group, junk=0):
    """Caches with rows k, v [n][Hkv][128] (bf16 bits) at positions 0 .. n - 1; what is not
    written holds `junk` bytes."""
    n, Hkv = k.shape[:2]
    dk = torch.full((ss.subspec_kv4_bytes(Hkv, S, group),), junk, dtype=torch.uint8, device=DEV)
    dv = torch.full_like(dk, junk)
    ss.subspec_kv4_append(_dev(k), _dev(v), n, None, None, n, Hkv, S, 0, group, dk, dv)
    return dk, dv


def _held(bits, group):
    return oracle.kv4_quantize(oracle.bf16_bits_to_f64(bits), group)


def _run(q, dk, dv, mask, M, Hq, Hkv, S, P, T, group, scale, stream=None):
    out = torch.full((M + 1, Hq, D), -7, dtype=torch.int16, device=DEV)
    torch.cuda.synchronize()  # the call may run on another stream
    ss.subspec_tree_attention_kv4(_dev(q), dk, dv, torch.from_numpy(mask.view(np.int32)).to(DEV), M, Hq, Hkv, S, P, T,
                                  group, scale, out, stream)
    torch.cuda.synchronize()
    assert bool((out[M] == -7).all())
    return oracle.bf16_bits_to_f64(out[:M].cpu().numpy().view(np.uint16))


def _check(M, Hq, Hkv, P, T, group, seed, q_scale=1.0, mask=None, S=None, scale=1.0 / math.sqrt(D), junk=0, v_scale=None,
           what=""):
    n = P + T + M
    S = S or (n + 31) // 32 * 32 + 32
    rng = np.random.default_rng([M, Hq, Hkv, P, T, seed])
    q = _bf16(rng.standard_normal((M, Hq, D)) * q_scale)
    own = min(Hkv, 8)  # many heads share the rows of eight
    k = rng.standard_normal((n, own, D))
    k[:, :, ::16] *= 3.0
    v = rng.standard_normal((n, own, D)) + 0.5
    if v_scale is not None:
        v *= v_scale(rng, n)[:, None, None]
    k, v = (_bf16(a)[:, np.arange(Hkv) % own] for a in (k, v))
    if mask is None:
        mask = synth.tree_levels_mask(T, 6, M, seed)
    dk, dv = _fill(k, v, S, group, junk)
    got = _run(q, dk, dv, mask, M, Hq, Hkv, S, P, T, group, scale)
    if Hkv > own:  # and three of them are compared
        some = np.array([0, Hkv // 2, Hkv - 1])
        G, Hkv = Hq // Hkv, 3
        heads = (some[:, None] * G + np.arange(G)).ravel()
        q, got, k, v, Hq = q[:, heads], got[:, heads], k[:, some], v[:, some], 3 * G
    kh, vh = _held(k, group), _held(v, group)
    K, V = oracle.kv4_value(*kh), oracle.kv4_value(*vh)
    ref, wabs = oracle.tree_attention_values(q, K, V, P, T, mask, scale)
    wide = lambda a: np.repeat(a.astype(np.float64), group, axis=-1)  # noqa: E731
    _, wmin = oracle.tree_attention_values(q, K, wide(vh[2]), P, T, mask, scale)
    _, wstep = oracle.tree_attention_values(q, K, wide(vh[1]), P, T, mask, scale)
    qa = np.abs(oracle.bf16_bits_to_f64(q))
    G = Hq // Hkv
    delta = np.empty((M, Hq, 1))
    for h in range(Hq):
        size = 15 * wide(kh[1]) + np.abs(wide(kh[2]))
        delta[:, h, 0] = (2.0 ** -20 * abs(scale) * (qa[:, h] @ size[:, h // G].T).max(1) +
                          2.0 ** -21 * np.abs(oracle.bf16_bits_to_f64(q)[:, h] @ K[:, h // G].T * scale).max(1))
    E = max(0, math.frexp(float(vh[1].max()))[1])
    tol = (2.0 ** -8 * np.abs(ref) + 2.0 ** -11 * (3 * wabs + wmin) + n * 2.0 ** (E - 33) * (np.abs(V).max() + 240 * (1 + float(vh[1].max()))) +
           2 * delta * wabs + 2.0 ** -18 * (15 * wstep + wmin))
    err = np.abs(got - ref)
    assert np.all(err <= tol), (what, float(err.max()), float((err / np.maximum(tol, 1e-300)).max()))
    return got


SHAPES = [
    (6, 28, 4, 2048, 282, 1.0),   # Qwen2.5-7B, last pass of a depth-48 tree
    (6, 28, 4, 2048, 282, 4.0),   # peaked scores
    (6, 40, 8, 1000, 60, 1.0),    # Qwen2.5-32B: 30 query rows
    (1, 28, 4, 1, 0, 1.0),        # two positions
    (1, 1, 1, 0, 0, 1.0),         # one position
    (6, 28, 4, 100, 0, 2.0),
    (6, 28, 4, 0, 36, 1.0),       # no committed context
    (8, 16, 2, 33, 7, 1.0),       # 64 query rows a head, ragged tails
    (12, 12, 3, 500, 21, 1.0),    # 48 query rows: three tiles
    (3, 4, 4, 77, 13, 1.5),       # no grouping
    (1, 40, 8, 4096, 0, 1.0),     # a single token over full tiles and one more position
    (5, 10, 2, 5000, 95, 1.0),
    (1, 16, 16, 9000, 0, 2.0),    # several rounds of tiles per wavefront
    (10, 12, 2, 6001, 200, 1.0),  # 60 rows, long
    # many heads, so that a wavefront has five tiles and more: 1, 17, 64, 20 and 40 rows a head
    (1, 128, 128, 2500, 0, 1.0),
    (17, 34, 34, 5000, 20, 1.0),
    (16, 64, 16, 4900, 90, 2.0),
    (20, 64, 64, 5101, 13, 1.0),
    (40, 40, 40, 4000, 20, 1.0),
]


@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("M,Hq,Hkv,P,T,qs", SHAPES)
def test_kv4_attention_matches_oracle(M, Hq, Hkv, P, T, qs, group):
    _check(M, Hq, Hkv, P, T, group, 7 * P + T + M, q_scale=qs, what=f"M={M} Hq={Hq} Hkv={Hkv} P={P} T={T} group={group}")


@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("M,Hq,Hkv,P,T", [(6, 28, 4, 700, 42), (8, 16, 2, 45, 90), (1, 8, 8, 2000, 3)])
def test_kv4_attention_counts_every_visible_position_once(M, Hq, Hkv, P, T, group):
    """With q = 0 all weights are equal; position j holds a 1 in dimension j % 128 alone, so an
    output is the share of the visible positions with that remainder: a whole number over
    the number of visible ones, which bf16's 2^-8 cannot blur below 128 of them."""
    n = P + T + M
    k = _bf16(np.random.default_rng(1).standard_normal((n, Hkv, D)))
    v = np.zeros((n, Hkv, D), np.float32)
    v[np.arange(n), :, np.arange(n) % D] = 1.0
    rng = np.random.default_rng(3)
    mask = rng.integers(0, 2 ** 32, (M, (T + M + 31) // 32), dtype=np.uint64).astype(np.uint32)  # bits past T + M too
    S = (n + 31) // 32 * 32
    dk, dv = _fill(k, _bf16(v), S, group)
    got = _run(np.zeros((M, Hq, D), np.uint16), dk, dv, mask, M, Hq, Hkv, S, P, T, group, 0.088)
    for i in range(M):
        seen = np.array([True] * P + [bool((int(mask[i, j // 32]) >> (j % 32)) & 1) for j in range(T + M)])
        at = np.nonzero(seen)[0]
        expect = np.bincount(at % D, minlength=D)
        assert np.array_equal(np.rint(got[i] * at.size), np.broadcast_to(expect, (Hq, D))), i


def test_kv4_attention_query_without_visible_positions_gets_zeros():
    M, Hq, Hkv, P, T = 2, 4, 2, 0, 3
    mask = np.zeros((M, 1), np.uint32)
    mask[1, 0] = 1 << (T + 1)
    got = _check(M, Hq, Hkv, P, T, 64, 5, mask=mask, what="empty row")
    assert not got[0].any()
    # every range of a longer tree without a visible position for some of the rows
    M, Hq, Hkv, T = 6, 28, 4, 282
    mask = synth.tree_levels_mask(T, 6, M, 3)
    mask[[0, 4]] = 0
    mask[2] = 0
    mask[2, 3] = 1 << 5  # one position of one tile
    got = _check(M, Hq, Hkv, 0, T, 128, 6, mask=mask, what="empty rows")
    assert not got[[0, 4]].any()


@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("junk", [0xFF, 0x7C])
def test_kv4_attention_positions_that_nothing_wrote(group, junk):
    """Positions past the last and tree positions that no row allows hold NaN and infinite
    scales; nothing of them reaches an output."""
    M, Hq, Hkv, P, T = 4, 8, 2, 37, 61
    n = P + T + M
    S = 160
    rng = np.random.default_rng([group, junk])
    q = _bf16(rng.standard_normal((M, Hq, D)))
    k, v = _bf16(rng.standard_normal((n, Hkv, D))), _bf16(rng.standard_normal((n, Hkv, D)))
    hidden = rng.choice(T, 20, replace=False)
    mask = rng.integers(0, 2 ** 32, (M, (T + M + 31) // 32), dtype=np.uint64).astype(np.uint32)
    for j in hidden:
        mask[:, j // 32] &= ~np.uint32(1 << (j % 32))
    dk = torch.full((ss.subspec_kv4_bytes(Hkv, S, group),), junk, dtype=torch.uint8, device=DEV)
    dv = torch.full_like(dk, junk)
    rows = np.arange(n, dtype=np.int32)
    rows[P + hidden] = -1
    ss.subspec_kv4_append(_dev(k), _dev(v), n, torch.from_numpy(rows).to(DEV), None, n, Hkv, S, 0, group, dk, dv)
    got = _run(q, dk, dv, mask, M, Hq, Hkv, S, P, T, group, 0.1)
    clean = _fill(k, v, S, group)
    same = _run(q, *clean, mask, M, Hq, Hkv, S, P, T, group, 0.1)
    assert np.isfinite(got).all() and np.array_equal(got, same)


@pytest.mark.parametrize("group", [64, 128])
@pytest.mark.parametrize("M,Hq,Hkv,P,T", [(4, 8, 2, 37, 61), (6, 28, 4, 2048, 282), (8, 16, 2, 70000, 90)])
def test_kv4_attention_large_scales_where_nothing_is_seen(M, Hq, Hkv, P, T, group):
    """The same bits whatever finite scales and minima lie past the last position and at tree
    positions that no row allows: 0x7777 is 30576, beside values of 2^-7 whose weights would
    lose their bits to it."""
    n = P + T + M
    S = (n + 31) // 32 * 32 + 64
    rng = np.random.default_rng([group, P])
    q = _bf16(rng.standard_normal((M, Hq, D)))
    k, v = _bf16(rng.standard_normal((n, Hkv, D))), _bf16(rng.standard_normal((n, Hkv, D)) * 2.0 ** -7)
    hidden = rng.choice(T, T // 3, replace=False)
    mask = rng.integers(0, 2 ** 32, (M, (T + M + 31) // 32), dtype=np.uint64).astype(np.uint32)
    for j in hidden:
        mask[:, j // 32] &= ~np.uint32(1 << (j % 32))
    rows = np.arange(n, dtype=np.int32)
    rows[P + hidden] = -1
    got = []
    for junk in (0, 0x77):
        dk = torch.full((ss.subspec_kv4_bytes(Hkv, S, group),), junk, dtype=torch.uint8, device=DEV)
        dv = torch.full_like(dk, junk)
        ss.subspec_kv4_append(_dev(k), _dev(v), n, torch.from_numpy(rows).to(DEV), None, n, Hkv, S, 0, group, dk, dv)
        got.append(_run(q, dk, dv, mask, M, Hq, Hkv, S, P, T, group, 0.1))
    assert np.array_equal(*got)


@pytest.mark.parametrize("q_scale", [1e-38, 5e37])
def test_kv4_attention_scale_zero_for_any_q(q_scale):
    _check(3, 8, 2, 200, 9, 64, 13, q_scale=q_scale, scale=0.0, what=f"q of {q_scale}, scale 0")


@pytest.mark.parametrize("scale", [-0.05, 0.0, 1.0])
def test_kv4_attention_scales_of_either_sign(scale):
    _check(3, 8, 2, 200, 9, 64, 11, scale=scale, what=f"scale={scale}")


@pytest.mark.parametrize("spread", ["tiny", "large", "mixed", "constant"])
def test_kv4_attention_value_scales_far_apart(spread):
    def scales(rng, n):
        if spread == "tiny":
            return np.full(n, 2.0 ** -9)
        if spread == "large":
            return np.full(n, 2.0 ** 11)
        if spread == "constant":
            return np.where(np.arange(n) % 3 == 0, 0.0, 1.0)
        return 2.0 ** rng.integers(-8, 9, n)
    for group in (64, 128):
        _check(4, 8, 2, 900, 30, group, 12, v_scale=scales, what=spread)


def test_kv4_attention_nan_stays_in_its_row():
    M, Hq, Hkv, P, T = 2, 8, 2, 300, 0
    rng = np.random.default_rng(9)
    q = rng.standard_normal((M, Hq, D))
    q[0, 3, 7] = np.nan
    k, v = _bf16(rng.standard_normal((P + M, Hkv, D))), _bf16(rng.standard_normal((P + M, Hkv, D)))
    mask = np.array([[1], [3]], np.uint32)
    dk, dv = _fill(k, v, 320, 64)
    got = _run(_bf16(q), dk, dv, mask, M, Hq, Hkv, 320, P, T, 64, 0.1)
    assert np.isnan(got[0, 3]).all()
    got[0, 3] = 0
    assert np.isfinite(got).all()


def test_kv4_attention_deterministic_and_on_another_stream():
    M, Hq, Hkv, P, T = 6, 28, 4, 700, 42
    n, S = P + T + M, 768
    rng = np.random.default_rng(77)
    q, k, v = _bf16(rng.standard_normal((M, Hq, D))), _bf16(rng.standard_normal((n, Hkv, D))), _bf16(rng.standard_normal((n, Hkv, D)))
    mask = synth.tree_levels_mask(T, 6, M, 77)
    dk, dv = _fill(k, v, S, 64)
    torch.cuda.synchronize()
    a = _run(q, dk, dv, mask, M, Hq, Hkv, S, P, T, 64, 0.125)
    st = torch.cuda.Stream()
    for s in (None, st):
        torch.cuda.synchronize()
        assert np.array_equal(a, _run(q, dk, dv, mask, M, Hq, Hkv, S, P, T, 64, 0.125, s))


def test_kv4_attention_heads_far_apart_in_a_long_cache():
    """Positions whose byte offsets pass 2^31 and 2^32: the last head of a cache of 32 heads of
    2^21 positions (4.8 GB each for keys and values), 2^11 of them used."""
    Hkv, S, group, M, P = 32, 1 << 21, 64, 2, 2046
    head = ss.subspec_kv4_bytes(1, S, group)
    assert head * (Hkv - 1) > 2 ** 32
    rng = np.random.default_rng(4)
    n = P + M
    k, v = _bf16(rng.standard_normal((n, Hkv, D))), _bf16(rng.standard_normal((n, Hkv, D)))
    q = _bf16(rng.standard_normal((M, Hkv, D)))
    mask = np.array([[1], [3]], np.uint32)
    dk = torch.zeros((Hkv * head,), dtype=torch.uint8, device=DEV)
    dv = torch.zeros_like(dk)
    ss.subspec_kv4_append(_dev(k), _dev(v), n, None, None, n, Hkv, S, 0, group, dk, dv)
    got = _run(q, dk, dv, mask, M, Hkv, Hkv, S, P, 0, group, 0.1)
    small = _fill(k, v, 2048, group)
    assert np.array_equal(got, _run(q, *small, mask, M, Hkv, Hkv, 2048, P, 0, group, 0.1))
    # rows at the far end, read back
    pos = S - 40
    ss.subspec_kv4_append(_dev(k), _dev(v), n, None, None, 40, Hkv, S, pos, group, dk, dv)
    out = [torch.empty((40, Hkv, D), dtype=torch.int16, device=DEV) for _ in range(4)]
    ss.subspec_kv4_read(dk, dv, Hkv, S, pos, 40, group, out[0], out[1])
    ss.subspec_kv4_read(*small, Hkv, 2048, 0, 40, group, out[2], out[3])
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])
