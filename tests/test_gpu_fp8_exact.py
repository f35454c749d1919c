"""GPU parity of the product in 8-bit floating point with exact products at any number of rows.

Tolerance: products are exact, sums in fp32: K / 128 + 32 roundings of 2^-23 W, W the sum of magnitudes
(as in test_gpu_fp8.py), and one to bf16, 2^-8; small whole numbers have no rounding."""
import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss

from test_gpu_fp8 import DEV, _random_rows, _tiled_weight, codes_to, weight
from test_gpu_fp8_kinds import _pick, _some
from test_gpu_rows import bf16, dev, rows8

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# every kind of launch above 64 rows: (kernel, rows, columns of a tile, K shared, more than one tile a workgroup or two
# workgroups a compute unit), as test_library_fp8_exact_cpu.py holds the plan to
KINDS = {
    (65, 16, 128): (1, 32, 64, False, False), (73, 5536, 256): (1, 32, 64, False, True), (66, 16, 640): (1, 32, 64, True, False),
    (68, 5600, 384): (1, 64, 64, False, False), (811, 2496, 512): (1, 64, 64, False, True), (113, 1952, 1152): (1, 64, 64, True, False),
    (65, 13424, 512): (1, 64, 128, False, False), (333, 10880, 640): (1, 64, 128, False, True), (108, 5232, 3840): (1, 64, 128, True, False),
    (66, 4848, 128): (2, 32, 256, False, False), (194, 16400, 384): (2, 32, 256, False, True), (65, 5984, 7296): (2, 32, 256, True, False),
    (261, 15056, 896): (2, 32, 256, True, True), (102, 16528, 512): (2, 64, 256, False, False), (199, 19152, 640): (2, 64, 256, False, True),
    (113, 10432, 5632): (2, 64, 256, True, False), (197, 18800, 1920): (2, 64, 256, True, True),
}


def linear(x, xs, w, ws, M, N, K, stream=None, pad=24):
    y = torch.full((M * N + pad,), 7.0, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    ss.subspec_fp8_linear_exact(x, xs, w, ws, M, N, K, y, stream)
    torch.cuda.synchronize()
    assert bool((y[M * N:] == 7).all())
    return y[: M * N].view(M, N)


def _check(y, x8, w8):
    xv, wv = oracle.fp8_values(*x8), oracle.fp8_values(*w8)
    ref, size = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    err, tol = np.abs(y - ref), 2.0 ** -8 * np.abs(ref) + (xv.shape[1] / 128 + 32) * 2.0 ** -23 * size
    assert np.all(err <= tol), (float((err / np.maximum(tol, 1e-300)).max()), np.argwhere(err > tol)[:4].tolist())


@pytest.mark.parametrize("M,N,K", KINDS)
def test_products_are_exact_at_any_number_of_rows(M, N, K):
    rng = np.random.default_rng([80, M, N, K])
    x8, w8 = _random_rows(rng, M, K), _tiled_weight(rng, N, K)
    x, (t, ws) = codes_to(*x8), weight(*w8)
    y = linear(*x, t, ws, M, N, K)
    m, n = _pick(M), _pick(N)
    _check(_some(y, m, n), tuple(a[m] for a in x8), tuple(a[n] for a in w8))
    for _ in range(2):  # and the counters are as they were
        assert torch.equal(linear(*x, t, ws, M, N, K).view(torch.int16), y.view(torch.int16))
    # products that the 8-bit units would cut away: 448 * 448 next to 2^-9 * 448 in every eight, their sums cancel
    xc, wc = np.zeros((M, K), np.uint8), np.zeros((N, K), np.uint8)
    xc[:, 0::8], xc[:, 1::8], xc[:, 2::8] = 0x7E, 0xFE, 0x01
    wc[:] = 0x7E
    one, onew = np.full((M, K // 128), 127), np.full((N, K // 128), 127)
    y = linear(*codes_to(xc, one), *weight(wc, onew), M, N, K)
    assert bool((y == K / 8 * 448 / 512).all())


@pytest.mark.parametrize("M,N,K", KINDS)
def test_whole_numbers_are_exact(M, N, K):
    rng = np.random.default_rng([81, M, N, K])
    p = rng.integers(-30, 31, K // 128)
    xv = rng.integers(1, 3, (M, K)) * rng.choice([-1, 1], (M, K)) * (rng.random((M, K)) < min(1.0, 200 / K))
    wv = (rng.integers(1, 3, (131, K)) * rng.choice([-1, 1], (131, K)))
    at = np.arange(N) * 37 % 131
    t, ws = weight(oracle.e4m3_code(wv)[at], np.broadcast_to(127 - p, (N, K // 128)))
    y = linear(*codes_to(oracle.e4m3_code(xv), np.broadcast_to(127 + p, (M, K // 128))), t, ws, M, N, K)
    m, n = _pick(M), _pick(N)
    ref = xv[m].astype(np.float64) @ wv[at[n]].T.astype(np.float64)
    small = np.abs(ref) <= 256
    assert small.mean() > 0.99
    assert np.array_equal(_some(y, m, n)[small], ref[small])


@pytest.mark.parametrize("M,N,K", KINDS)
def test_bf16_rows_give_the_bits_of_their_8_bit_rows(M, N, K):
    rng = np.random.default_rng([82, M, N, K])
    xd = dev(bf16(rng.standard_normal((M, K)) * np.repeat(np.exp2(rng.integers(-4, 5, (M, K // 128))), 128, 1)))
    t, ws = weight(*_tiled_weight(rng, N, K))
    c, s = rows8(M, K)
    ss.subspec_fp8_rows(xd, M, K, c, s)
    y8 = linear(c, s, t, ws, M, N, K).view(torch.int16)
    for _ in range(2):
        assert torch.equal(linear(xd, None, t, ws, M, N, K).view(torch.int16), y8)


@pytest.mark.parametrize("M,N,K", [k for k in KINDS if k[2] >= 384])
def test_all_scales_zeros_and_nan(M, N, K):
    rng = np.random.default_rng([83, M, N, K])
    x8, w8 = _random_rows(rng, M, K), _tiled_weight(rng, N, K)
    p = np.array([-126, 0, 120, -100, 7, 60, -60, 1, 100])[np.arange(K // 128) % 9]
    x8, w8 = (x8[0].copy(), np.broadcast_to(127 + p, x8[1].shape)), (w8[0].copy(), np.broadcast_to(127 - p, w8[1].shape))
    y = linear(*codes_to(*x8), *weight(*w8), M, N, K)
    m, n = _pick(M), _pick(N)
    _check(_some(y, m, n), tuple(a[m] for a in x8), tuple(a[n] for a in w8))
    x8[0][M // 2, K - 1], w8[0][N - 3, 0] = 0xFF, 0x7F
    z = linear(*codes_to(*x8), *weight(*w8), M, N, K)
    nan = torch.isnan(z)
    assert bool(nan[M // 2].all()) and bool(nan[:, N - 3].all()) and int(nan.sum()) == M + N - 1
    assert torch.equal(torch.where(nan, 0, z), torch.where(nan, 0, y))
    # rows of zeros beside others of ordinary scales
    x8, w8 = _random_rows(rng, M, K), _tiled_weight(rng, N, K)
    w, xz, empty = weight(*w8), tuple(a.copy() for a in x8), np.arange(M) % 3 == 1
    y = linear(*codes_to(*x8), *w, M, N, K)
    xz[0][empty], xz[1][empty] = 0, 1
    z = linear(*codes_to(*xz), *w, M, N, K)
    off = torch.from_numpy(empty).to(DEV)
    assert not bool(z[off].any()) and torch.equal(z[~off].view(torch.int16), y[~off].view(torch.int16))


@pytest.mark.parametrize("M,N,K", [(1, 272, 640), (16, 3584, 3584), (30, 512, 640), (49, 1024, 2176), (64, 5120, 1152)])
def test_up_to_64_rows_it_is_the_same_call(M, N, K):
    rng = np.random.default_rng([84, M, N, K])
    xd, w = dev(bf16(rng.standard_normal((M, K)))), weight(*_random_rows(rng, N, K))
    y = torch.empty((M, N), dtype=torch.bfloat16, device=DEV)
    ss.subspec_fp8_linear(xd, None, *w, M, N, K, y)
    assert torch.equal(linear(xd, None, *w, M, N, K).view(torch.int16), y.view(torch.int16))


def test_on_another_stream():
    M, N, K = 108, 5232, 3840
    rng = np.random.default_rng(85)
    xd, w = dev(bf16(rng.standard_normal((M, K)))), weight(*_tiled_weight(rng, N, K))
    y = linear(xd, None, *w, M, N, K)
    assert torch.equal(linear(xd, None, *w, M, N, K, torch.cuda.Stream()).view(torch.int16), y.view(torch.int16))


def test_a_layers_second_half_keeps_the_precision_of_its_last_rounding():
    # gate|up, activation into 8-bit rows, down, against 64 bits with gate|up rounded to bf16 between.  A rounding's
    # error is even over a step of 2^-7 of the binade's low end: in the 2-norm 2^-7 / sqrt(12) of a value there, less of
    # every other.  Sums that differ in fp32's last places (2^-20 at most) tip one in 2^12 of gate|up's roundings by
    # 2^-7, and those and their own difference one code in 2^12 or fewer by 2^-3: 2^-9 / 64 on top at most.
    from paper_2509_18344_amd import prepare
    M, K, I = 400, 768, 1536
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    x = rnd(M, K).to(torch.bfloat16)
    up, down = (rnd(2 * I, K) / K ** 0.5).to(torch.bfloat16), (rnd(K, I) / I ** 0.5).to(torch.bfloat16)
    pu, pd = prepare.fp8_weight(up), prepare.fp8_weight(down)
    gu, y = torch.empty((M, 2 * I), dtype=torch.bfloat16, device=DEV), torch.empty((M, K), dtype=torch.bfloat16, device=DEV)
    h, hs = rows8(M, I)

    def values(t):
        v = t.double().cpu().numpy()
        return oracle.fp8_values(*oracle.fp8_rows(v))

    ref = values(x) @ values(up).T
    ref = oracle.bf16_bits_to_f64(oracle.bf16_round_bits(ref.astype(np.float32)))
    ref = oracle.silu_mul(ref[:, :I], ref[:, I:])
    ref = oracle.fp8_values(*oracle.fp8_rows(ref)) @ values(down).T
    off = {}
    for name in ("subspec_fp8_linear_exact", "subspec_fp8_linear"):
        call = getattr(ss, name)
        call(x, None, pu["w"], pu["w_scales"], M, 2 * I, K, gu)
        ss.subspec_silu_mul(gu, M, I, None, h, hs)
        call(h, hs, pd["w"], pd["w_scales"], M, K, I, y)
        off[name] = float(np.linalg.norm(y.double().cpu().numpy() - ref) / np.linalg.norm(ref))
    print(off)
    assert off["subspec_fp8_linear_exact"] <= 2.0 ** -7 / 12 ** 0.5 + 2.0 ** -15
