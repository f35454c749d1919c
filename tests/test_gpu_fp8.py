"""GPU parity of the product in 8-bit floating point against the fp64 oracle.

Tolerance, from the arithmetic.  Up to EXACT rows the products are exact and their sums in fp32.  Above, the
matrix units sum the products of eight neighbouring k (8 i .. 8 i + 7)
on a grid: with E the largest sum of the two codes' exponents among the eight (a subnormal code's is -6),
each product is cut towards zero to a multiple of 2^(E - 13).  The largest itself, with at most 6 binary
places below its own exponent, lies on the grid or its cut is one of the grid's steps like the others', so
eight products lose less than 8 * 2^(E - 13), and 2^E is at most the product of the two sides' largest
powers among the eight.  The groups' sums, the blocks of 128 and the parts of K are added in fp32: K / 128
blocks one after the other (a few more where K is cut into parts) and at most 16 alignments within a
block, each counted as a whole unit of the last place of the sum of magnitudes W = sum |x w|, 2^-23 W.
Then one rounding to bf16, 2^-8 relative.  Small whole numbers have no rounding at all and must come out
equal.  test_sums_of_eight_products holds the grid itself to the units."""
import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss

from test_gpu_rows import bf16, dev, f64, host, rows8, values8

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"
EXACT = 64  # rows up to which products are not cut


def codes_to(codes, bytes_):
    """Codes [R][K] and scale bytes on the GPU; bytes past the last block hold the scale of NaN."""
    return (torch.from_numpy(np.ascontiguousarray(codes)).to(DEV),
            torch.from_numpy(oracle.scale_words(bytes_, fill=255).view(np.int32)).to(DEV))


def weight(codes, bytes_):
    c, s = codes_to(codes, bytes_)
    t = torch.empty(codes.size, dtype=torch.uint8, device=DEV)
    ss.subspec_fp8_pack(c, *codes.shape, t)
    return t, s


def linear(x, xs, w, ws, M, N, K, stream=None, pad=24):
    y = torch.full((M * N + pad,), 7.0, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    ss.subspec_fp8_linear(x, xs, w, ws, M, N, K, y, stream)
    torch.cuda.synchronize()
    assert bool((y[M * N:] == 7).all())
    return y[: M * N].view(M, N)


def _powers(codes, bytes_):
    """2^(exponent of a code and its scale), 0 for a zero: float64 [R][K]."""
    e = np.maximum((codes >> 3 & 15).astype(int), 1) - 7
    p = np.exp2(e + np.repeat(bytes_.astype(int) - 127, 128, 1).astype(float))
    return np.where(codes & 127, p, 0.0)


def check(y, x8, w8, what="", rows=None):
    """y (bf16 on the GPU) against the product of 8-bit rows, (codes, scale bytes) each."""
    xv, wv = oracle.fp8_values(*x8), oracle.fp8_values(*w8)
    K = xv.shape[1]
    exact = (rows or len(xv)) <= EXACT
    ref, wabs = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    px, pw = (_powers(*r).reshape(len(r[0]), K // 8, 8).max(-1) for r in (x8, w8))
    cut = 8 * 2.0 ** -13 * (px @ pw.T) * (not exact)
    err, tol = np.abs(f64(host(y)) - ref), 2.0 ** -8 * (np.abs(ref) + cut) + cut + (K / 128 + 32) * 2.0 ** -23 * wabs
    assert np.all(err <= tol), (what, float((err / np.maximum(tol, 1e-300)).max()), np.argwhere(err > tol)[:4].tolist())


def _random_rows(rng, R, K, spread=3):
    """Rows whose blocks have different scales, as 8-bit rows."""
    x = rng.standard_normal((R, K)) * np.repeat(np.exp2(rng.integers(-spread, spread + 1, (R, K // 128))), 128, 1)
    return oracle.fp8_rows(x)


# every way in: rows from one to past each tile, columns of one tile, of odd numbers of tiles and of many, short and long K
SHAPES = [(1, 16, 128), (1, 3584, 3584), (1, 48, 27648), (2, 16, 256), (3, 208, 640), (6, 5120, 1152), (7, 512, 18944), (8, 1040, 384),
          (13, 16, 18944), (16, 272, 512), (17, 272, 512), (31, 80, 1024), (33, 528, 1280), (48, 16, 4096), (49, 3584, 896), (64, 256, 2176), (65, 272, 640),
          (96, 144, 128), (127, 128, 1920), (128, 1024, 512), (129, 400, 768), (200, 16, 5120), (255, 256, 256), (257, 272, 384), (289, 1168, 1152),
          (300, 4112, 128), (512, 512, 1024), (600, 784, 640), (1000, 2064, 896), (1025, 528, 384), (2049, 272, 256)]


# every kind of launch: (kernel, rows, columns of a tile, K shared by workgroups, more than one tile a workgroup or two
# workgroups a compute unit), as tests/test_library_fp8_cpu.py holds the plan to
KINDS = {
    (18, 368, 5888): (1, 32, 64, True, False), (19, 6224, 384): (1, 32, 64, False, False), (20, 17008, 384): (1, 32, 64, False, True),
    (34, 2528, 1664): (1, 64, 64, True, False), (33, 8208, 384): (1, 64, 64, False, False), (35, 18976, 256): (1, 64, 128, False, False),
    (34, 9024, 3712): (1, 64, 128, True, False), (18, 16448, 4864): (2, 32, 256, True, False), (34, 19536, 7808): (2, 64, 256, True, False),
    (40, 70000, 384): (2, 64, 256, False, True), (66, 16, 384): (1, 64, 64, False, False), (67, 16, 896): (1, 64, 64, True, False),
    (65, 16, 256): (1, 64, 128, False, False), (66, 16, 640): (1, 64, 128, True, False), (69, 18272, 256): (1, 96, 128, False, False),
    (67, 8352, 6016): (1, 96, 128, True, False), (66, 16, 128): (1, 128, 128, False, False), (2267, 272, 6784): (1, 128, 128, True, False),
    (130, 17312, 256): (2, 128, 256, False, False), (275, 33024, 128): (2, 128, 256, False, True), (1233, 14800, 6016): (2, 128, 256, True, True),
    (400, 16512, 128): (2, 192, 256, False, False), (514, 27152, 128): (2, 192, 256, False, True), (144, 18000, 5248): (2, 192, 256, True, False),
    (516, 26448, 2560): (2, 192, 256, True, True), (579, 16480, 128): (2, 256, 256, False, False), (786, 26256, 128): (2, 256, 256, False, True),
    (1175, 15008, 6016): (2, 256, 256, True, True),
}


def check_some(y, x8, w8, what=""):
    """check() of about 200 rows and columns, the ends of every tile's among them."""
    M, N = y.shape
    pick = lambda n: np.unique(np.r_[np.arange(min(n, 35)), np.arange(max(0, n - 70), n), np.arange(31, n, max(32, n // 64 // 32 * 32)),  # noqa: E731
                                     np.arange(32, n, max(32, n // 64 // 32 * 32))])
    m, n = pick(M), pick(N)
    check(y[torch.from_numpy(m).to(DEV)][:, torch.from_numpy(n).to(DEV)], tuple(a[m] for a in x8), tuple(a[n] for a in w8), what, M)


def _tiled_weight(rng, N, K, spread=3):
    """Rows of a weight that repeat after an odd number of them, and its tiles and scales on the GPU."""
    c, b = _random_rows(rng, min(N, 131), K, spread)
    at = np.arange(N) * 37 % len(c)
    return c[at], b[at]


@pytest.mark.parametrize("M,N,K", KINDS)
def test_every_kind_of_launch(M, N, K):
    rng = np.random.default_rng([63, M, N, K])
    x8, w8 = _random_rows(rng, M, K), _tiled_weight(rng, N, K)
    t, ws = weight(*w8)
    x = codes_to(*x8)
    y = linear(*x, t, ws, M, N, K)
    check_some(y, x8, w8)
    for _ in range(2):  # and the counters are as they were
        assert torch.equal(linear(*x, t, ws, M, N, K).view(torch.int16), y.view(torch.int16))


@pytest.mark.parametrize("M,N,K", [k for k in KINDS if k[2] >= 384 and k[0] * k[1] < 2 ** 23])
def test_every_kind_over_all_scales_and_with_nan(M, N, K):
    rng = np.random.default_rng([64, M, N, K])
    x8, w8 = _random_rows(rng, M, K), _tiled_weight(rng, N, K)
    p = np.array([-126, 0, 120, -100, 7, 60, -60, 1, 100])[np.arange(K // 128) % 9]
    x8, w8 = (x8[0].copy(), np.broadcast_to(127 + p, x8[1].shape)), (w8[0].copy(), np.broadcast_to(127 - p, w8[1].shape))
    x, (t, ws) = codes_to(*x8), weight(*w8)
    y = linear(*x, t, ws, M, N, K)
    check_some(y, x8, w8)
    x8[0][M // 2, K - 1], w8[0][N - 3, 0] = 0xFF, 0x7F
    x, (t, ws) = codes_to(*x8), weight(*w8)
    z = linear(*x, t, ws, M, N, K)
    nan = torch.isnan(z)
    assert bool(nan[M // 2].all()) and bool(nan[:, N - 3].all()) and int(nan.sum()) == M + N - 1
    assert torch.equal(torch.where(nan, 0, z), torch.where(nan, 0, y))


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_fp8_linear_matches_oracle(M, N, K):
    rng = np.random.default_rng([50, M, N, K])
    xc, xb = _random_rows(rng, M, K)
    wc, wb = _random_rows(rng, N, K)
    t, ws = weight(wc, wb)
    y = linear(*codes_to(xc, xb), t, ws, M, N, K)
    check(y, (xc, xb), (wc, wb))


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_fp8_linear_of_whole_numbers_is_exact(M, N, K):
    rng = np.random.default_rng([51, M, N, K])
    # a few values of a row are not zero: -2, -1, 1, 2 under powers that differ from block to block and cancel
    def rows(R, keep, sign):
        v = rng.integers(1, 3, (R, K)) * rng.choice([-1, 1], (R, K)) * (rng.random((R, K)) < keep)
        return oracle.e4m3_code(v), v, sign
    keep = min(1.0, 30 / K)
    p = rng.integers(-30, 31, K // 128)
    xc, xv, _ = rows(M, keep, 1)
    wc, wv, _ = rows(N, 1.0, -1)
    t, ws = weight(wc, np.broadcast_to(127 - p, (N, K // 128)))
    y = linear(*codes_to(xc, np.broadcast_to(127 + p, (M, K // 128))), t, ws, M, N, K)
    ref = xv.astype(np.float64) @ wv.T
    small = np.abs(ref) <= 256
    assert small.mean() > 0.99
    assert np.array_equal(f64(host(y))[small], ref[small])


@pytest.mark.parametrize("M,N,K", [(1, 3584, 3584), (5, 272, 27648), (3, 5120, 16384), (16, 512, 640), (17, 512, 640), (31, 272, 5248), (49, 1024, 2176), (40, 272, 2176), (100, 272, 5120), (289, 528, 1152), (700, 1040, 512)])
def test_bf16_rows_give_the_bits_of_their_8_bit_rows(M, N, K):
    rng = np.random.default_rng([52, M, N, K])
    x = rng.standard_normal((M, K)) * np.repeat(np.exp2(rng.integers(-4, 5, (M, K // 128))), 128, 1)
    x[rng.random((M, K)) < 0.01] *= 500.0
    x[M // 2, :128] = 0.0
    x = bf16(x)
    wc, wb = _random_rows(rng, N, K)
    t, ws = weight(wc, wb)
    xd = dev(x)
    y = linear(xd, None, t, ws, M, N, K)
    c, s = rows8(M, K)
    ss.subspec_fp8_rows(xd, M, K, c, s)
    y8 = linear(c, s, t, ws, M, N, K)
    assert torch.equal(y.view(torch.int16), y8.view(torch.int16))
    check(y, oracle.fp8_rows(f64(x)), (wc, wb))
    bytes_ = ws.view(torch.uint8).view(-1, N, 4)  # scales as bytes
    assert torch.equal(linear(c.view(torch.float8_e4m3fn), s.view(torch.float8_e8m0fnu), t, bytes_, M, N, K).view(torch.int16), y.view(torch.int16))
    for _ in range(3):
        assert torch.equal(linear(xd, None, t, ws, M, N, K).view(torch.int16), y.view(torch.int16))


@pytest.mark.parametrize("M", [16, 32])
def test_bf16_rows_of_all_scales_give_the_bits_of_their_8_bit_rows(M):
    # one block a row, from bf16's smallest numbers to its largest, with zeros, infinities and NaN beside them
    N, K = 48, 128
    rng = np.random.default_rng([65, M])
    x = bf16(rng.standard_normal((M, K)) * np.exp2(np.linspace(-134.0, 126.0, M))[:, None])
    x[1, ::3] &= 0x8003  # the last bits of subnormal numbers
    x[M - 3, 5:] = 0x8000
    x[M - 2, 7], x[2, 100], x[2, 101] = 0x7F80, 0xFF80, 0x7FC3
    c, s = rows8(M, K)
    ss.subspec_fp8_rows(dev(x), M, K, c, s)
    for power in (100, 0, -100):
        t, ws = weight(oracle.e4m3_code(rng.uniform(-4, 4, (N, K))), np.full((N, 1), 127 + power))
        y, y8 = linear(dev(x), None, t, ws, M, N, K), linear(c, s, t, ws, M, N, K)
        a, b = (v.float().cpu().numpy() for v in (y, y8))
        assert np.array_equal(a, b, equal_nan=True), (power, np.argwhere(~((a == b) | (np.isnan(a) & np.isnan(b))))[:5])
        if power == 100:
            assert np.isfinite(a[0]).all() and (a[0] != 0).any() and np.isnan(a[2]).all()


@pytest.mark.parametrize("M", [1, 16, 33, 130, 270])
def test_sums_of_eight_products(M):
    # the grid that the units sum eight products on, product by product, on codes of all magnitudes
    N, K = 32, 256
    rng = np.random.default_rng([61, M])
    xc, wc = (((rng.integers(0, 127, (R, K)) | rng.integers(0, 2, (R, K)) * 128).astype(np.uint8)) for R in (M, N))
    xb, wb = np.full((M, 2), 127), np.full((N, 2), 127)
    t, ws = weight(wc, wb)
    y = f64(host(linear(*codes_to(xc, xb), t, ws, M, N, K)))
    ex, ew = (np.maximum((c >> 3 & 15).astype(int), 1) - 7 for c in (xc, wc))
    xv, wv = oracle.E4M3[xc], oracle.E4M3[wc]
    for m in range(M):
        p, e = (xv[m] * wv).reshape(N, K // 8, 8), (ex[m] + ew).reshape(N, K // 8, 8)
        grid = np.exp2(e.max(-1, keepdims=True) - 13.0)
        ref = (np.trunc(p / grid) * grid if M > EXACT else p).sum((1, 2))
        tol = 2.0 ** -8 * np.abs(ref) + (K / 128 + 32) * 2.0 ** -23 * np.abs(p).sum((1, 2))
        assert np.all(np.abs(y[m] - ref) <= tol), m


@pytest.mark.parametrize("M", [1, 9, 40, 130, 300])
def test_scales_over_their_whole_range(M):
    # a block of x and its block of w whose powers cancel, from 2^-126 to 2^126; one pair meets at each k block
    N, K = 64, 128 * 9
    rng = np.random.default_rng([53, M])
    xc, wc = (oracle.e4m3_code(rng.uniform(-4, 4, (R, K))) for R in (M, N))
    p = np.array([-126, -100, -60, -1, 0, 7, 60, 100, 120])
    xb, wb = np.broadcast_to(127 + p, (M, 9)), np.broadcast_to(127 - p, (N, 9))
    t, ws = weight(wc, wb)
    y = linear(*codes_to(xc, xb), t, ws, M, N, K)
    check(y, (xc, xb), (wc, wb))


@pytest.mark.parametrize("M", [1, 20, 70, 270])
def test_nan_stays_in_its_row_and_column(M):
    N, K = 80, 640
    rng = np.random.default_rng([54, M])
    xc, xb = _random_rows(rng, M, K)
    wc, wb = _random_rows(rng, N, K)
    t, ws = weight(wc, wb)
    clean = f64(host(linear(*codes_to(xc, xb), t, ws, M, N, K)))
    xc, wc = xc.copy(), wc.copy()
    xc[M // 2, 300], wc[17, 639] = 0x7F, 0xFF
    t, ws = weight(wc, wb)
    y = f64(host(linear(*codes_to(xc, xb), t, ws, M, N, K)))
    hit = np.zeros((M, N), bool)
    hit[M // 2], hit[:, 17] = True, True
    assert np.isnan(y[hit]).all() and np.array_equal(y[~hit], clean[~hit])
    x = bf16(rng.standard_normal((M, K)))
    x[0, 3], x[M - 1, 600] = 0x7F80, 0x7FC0
    y = f64(host(linear(dev(x), None, t, ws, M, N, K)))
    assert np.isnan(y[[0, M - 1]]).all() and np.isnan(y[:, 17]).all() and np.isfinite(np.delete(y[1: M - 1], 17, 1)).all()


@pytest.mark.parametrize("N,K", [(16, 128), (48, 640), (272, 1280)])
def test_pack_is_the_oracles_order(N, K):
    c = np.random.default_rng([55, N, K]).integers(0, 256, (N, K)).astype(np.uint8)
    t = torch.full((N * K + 32,), 0x5A, dtype=torch.uint8, device=DEV)
    ss.subspec_fp8_pack(torch.from_numpy(c).to(DEV).view(torch.float8_e4m3fn), N, K, t)
    assert np.array_equal(t[: N * K].cpu().numpy(), oracle.weight_tiles(c)) and bool((t[N * K:] == 0x5A).all())


@pytest.mark.parametrize("other", ["current", "stream", "handle"])
def test_prepared_weight(other):
    from paper_2509_18344_amd import prepare
    N, K, M = 272, 640, 5
    rng = np.random.default_rng(62)
    w, x = bf16(rng.standard_normal((N, K))), bf16(rng.standard_normal((M, K)))
    wd, xd = dev(w), dev(x)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    p = prepare.fp8_weight(wd, {"current": None, "stream": s, "handle": s.cuda_stream}[other])
    s.synchronize()
    wc, wb = oracle.fp8_rows(f64(w))
    assert np.array_equal(p["w"].cpu().numpy(), oracle.weight_tiles(wc))
    check(linear(xd, None, p["w"], p["w_scales"], M, p["N"], p["K"]), oracle.fp8_rows(f64(x)), (wc, wb))


def test_results_past_2_31_elements():
    M, N, K = 32800, 65552, 128  # 2.15e9 results
    rng = np.random.default_rng(56)
    xc, xb = _random_rows(rng, 64, K)
    wc, wb = _random_rows(rng, 48, K)
    xr, wr = np.arange(M) * 7 % 64, np.arange(N) * 5 % 48
    t, ws = weight(wc[wr], wb[wr])
    x, xs = codes_to(xc[xr], xb[xr])
    y = torch.empty((M, N), dtype=torch.bfloat16, device=DEV)
    ss.subspec_fp8_linear(x, xs, t, ws, M, N, K, y)
    rows = np.r_[0:3, M // 2, M - 40:M]
    for cols in (slice(-300, None), slice(300)):
        check(y[torch.from_numpy(rows).to(DEV)][:, cols], (xc[xr[rows]], xb[xr[rows]]), (wc[wr[cols]], wb[wr[cols]]), "", M)


def test_weights_past_2_32_bytes():
    M, N, K = 2, 262160, 16512  # 4.3e9 codes
    rng = np.random.default_rng(57)
    xc, xb = _random_rows(rng, M, K)
    wc, wb = _random_rows(rng, 16, K)
    tile = torch.from_numpy(oracle.weight_tiles(wc)).to(DEV)
    t = tile.repeat(N // 16)
    last = oracle.fp8_rows(rng.standard_normal((16, K)))
    t[-tile.numel():] = torch.from_numpy(oracle.weight_tiles(last[0])).to(DEV)
    bytes_ = np.concatenate([np.tile(wb, (N // 16 - 1, 1)), last[1]])
    ws = torch.from_numpy(oracle.scale_words(bytes_).view(np.int32)).to(DEV)
    y = linear(*codes_to(xc, xb), t, ws, M, N, K)
    check(y[:, :16], (xc, xb), (wc, wb))
    check(y[:, -16:], (xc, xb), last)
    assert torch.equal(y[:, 16:32], y[:, -32:-16])


def _layer(rng, K, I):
    up, down = _random_rows(rng, 2 * I, K, 0), _random_rows(rng, K, I, 0)
    return dict(up=up, down=down, K=K, I=I, dev=(*weight(*up), *weight(*down)), w=bf16(1 + 0.2 * rng.standard_normal(K)))


def _mlp(l, x, res, M, out, stream=None):
    """The calls of a layer's second half; x and res are on the GPU, res is updated in place."""
    K, I = l["K"], l["I"]
    up, ups, down, downs = l["dev"]
    ss.subspec_add_norm(x, res, out["w"], 1e-6, M, K, res, None, out["a"], out["as"], stream)
    ss.subspec_fp8_linear(out["a"], out["as"], up, ups, M, 2 * I, K, out["gu"], stream)
    ss.subspec_silu_mul(out["gu"], M, I, None, out["h"], out["hs"], stream)
    ss.subspec_fp8_linear(out["h"], out["hs"], down, downs, M, K, I, out["y"], stream)
    return out["y"]


def _mlp_buffers(l, M):
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    a, h = rows8(M, l["K"]), rows8(M, l["I"])
    return {"a": a[0], "as": a[1], "h": h[0], "hs": h[1], "gu": e(M, 2 * l["I"]), "y": e(M, l["K"]), "w": dev(l["w"])}


def _mlp_steps_check(l, M, out, x, res):
    """Every step against the oracle of what the step before handed it."""
    K, I = l["K"], l["I"]
    s, y = oracle.add_norm(f64(x), f64(res), f64(l["w"]), 1e-6)
    a8 = values8(out["a"], out["as"], M, K)
    a = a8[2]
    assert np.all(np.abs(a - y) <= 2.0 ** -4 * np.abs(y) * 1.001 + np.repeat(np.abs(y).reshape(M, -1, 128).max(-1), 128, 1) * 2.0 ** -17)
    check(out["gu"], a8[:2], l["up"], "up")
    gu = f64(host(out["gu"]))
    h = oracle.silu_mul(gu[:, :I], gu[:, I:])
    h8 = values8(out["h"], out["hs"], M, I)
    hv = h8[2]
    assert np.all(np.abs(hv - h) <= 2.0 ** -4 * np.abs(h) * 1.001 + np.repeat(np.abs(h).reshape(M, -1, 128).max(-1), 128, 1) * 2.0 ** -17)
    check(out["y"], h8[:2], l["down"], "down")
    return s


@pytest.mark.parametrize("M", [1, 7, 49, 289])
def test_two_layers_mlps_one_after_the_other(M):
    rng = np.random.default_rng([58, M])
    layers = [_layer(rng, 640, 896), _layer(rng, 640, 896)]
    x, res = bf16(rng.standard_normal((M, 640))), bf16(4 * rng.standard_normal((M, 640)))
    xd, rd = dev(x), dev(res)
    for l in layers:
        out = _mlp_buffers(l, M)
        y = _mlp(l, xd, rd, M, out)
        torch.cuda.synchronize()
        s = _mlp_steps_check(l, M, out, x, res)
        assert np.all(np.abs(f64(host(rd)) - s) <= 2.0 ** -8 * np.abs(s) * 1.001)
        xd, x, res = y.clone(), host(y), host(rd)
