"""GPU parity of the row operators (residual addition with the RMS norm, gated activation) and of 8-bit
rows against the fp64 oracle.

Tolerances, from the arithmetic.  A bf16 output is rounded once: 2^-8 relative, and 2^-134 absolute below
bf16's normal range.  Norm, before that, in fp32: s is one rounding (2^-24), the sum of squares has at most
64 roundings a thread and 20 in the tree, halved by the root, the root, quotient and products six more:
below 2^-17 of y.  Activation: the exponent |g| / 2 in base 2 carries two roundings, so p^2 is off by
|g| 2^-23 relative, and ten roundings or hardware functions of 1 ulp follow: |g| 2^-23 + 2^-20.  8-bit
rows of bf16 values are exact arithmetic with one rounding: codes and scales have to be equal.  8-bit rows
of fp32 results: half a step of e4m3 at the given scale, 2^-4 relative or 2^-10 of the scale's power, on top
of the above; the scale may be the neighbour's where the block's largest lies at its border."""
import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"


def bf16(a):
    return oracle.bf16_round_bits(np.ascontiguousarray(a, np.float32))


def f64(bits):
    return oracle.bf16_bits_to_f64(bits)


def dev(bits):
    return None if bits is None else torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(DEV).view(torch.bfloat16)


def host(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


def rows8(M, K, pad=0):
    """Buffers of 8-bit rows, `pad` elements behind them."""
    return (torch.full((M * K + pad,), 0x5A, dtype=torch.uint8, device=DEV),
            torch.full(((K + 511) // 512 * M + pad,), 0x5A5A5A5A, dtype=torch.int32, device=DEV))


def values8(codes, scales, M, K):
    c = codes[: M * K].cpu().numpy().reshape(M, K)
    s = oracle.scale_bytes(scales[: (K + 511) // 512 * M].cpu().numpy().reshape(-1, M), K)
    return c, s, oracle.fp8_values(c, s)


def check8(codes, scales, M, K, y, rel):
    """8-bit rows of fp32 results y that are off by `rel` relative."""
    c, s, v = values8(codes, scales, M, K)
    top = np.abs(y).reshape(M, K // 128, 128).max(-1)
    for sign in (-1, 1):  # the scale is that of a value within the results' error
        _, b = oracle.fp8_rows(np.repeat(top * (1 + sign * rel), 128, 1))
        assert np.all(s >= b if sign < 0 else s <= b), "scales"
    p = np.repeat(np.exp2(s.astype(np.float64) - 127), 128, 1)
    err = np.abs(v - y)
    tol = np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * p) * (1 + 2.0 ** -10) + rel * np.abs(y)
    assert np.all(err <= tol), ("codes", float((err / tol).max()))


NORM_REL = 2.0 ** -17


def _norm(x, res, w, eps, pad=24, stream=None, eight=True):
    M, K = x.shape
    s, y = (torch.full((M * K + pad,), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    c, e = rows8(M, K, pad) if eight else (None, None)
    xd, rd, wd = dev(x), dev(res), dev(w)
    torch.cuda.synchronize()  # the call may run on another stream
    ss.subspec_add_norm(xd, rd, wd, eps, M, K, s, y, c, e, stream)
    torch.cuda.synchronize()
    assert bool((s[M * K:] == 7).all()) and bool((y[M * K:] == 7).all())
    if eight:
        assert bool((c[M * K:] == 0x5A).all()) and bool((e[(K + 511) // 512 * M:] == 0x5A5A5A5A).all())
    return host(s[: M * K]).reshape(M, K), host(y[: M * K]).reshape(M, K), c, e


def _check_norm(x, res, w, eps, **kw):
    M, K = x.shape
    s, y, c, e = _norm(x, res, w, eps, eight=K % 128 == 0, **kw)
    rs, ry = oracle.add_norm(f64(x), None if res is None else f64(res), f64(w), eps)
    if res is None:
        assert np.array_equal(s, x)
    assert np.all(np.abs(f64(s) - rs) <= (2.0 ** -8 + 2.0 ** -23) * np.abs(rs) + 2.0 ** -134)
    err, tol = np.abs(f64(y) - ry), (2.0 ** -8 + NORM_REL) * np.abs(ry) + 2.0 ** -134
    assert np.all(err <= tol), float((err / tol).max())
    if c is not None:
        check8(c, e, M, K, ry, NORM_REL)
    return s, y


def _rand(seed, M, K, scale=1.0, mean=0.0):
    return bf16(np.random.default_rng([seed, M, K]).standard_normal((M, K)) * scale + mean)


@pytest.mark.parametrize("M,K", [
    (1, 3584), (1, 5120), (7, 8), (3, 128), (2, 136), (5, 512), (4, 520), (2, 1536), (3, 2048), (3, 2056), (2, 4096), (2, 4224),
    (2, 6144), (2, 6152), (2, 8192), (2, 8320), (2, 16384), (2, 16512), (2, 27648), (2, 32768), (1, 32896), (1, 65536), (49, 5120), (300, 640),
    (515, 8), (520, 1024), (512, 1032), (600, 2056), (513, 3584), (512, 4104), (530, 8192), (512, 8320),
])
@pytest.mark.parametrize("residual", [False, True])
def test_add_norm_matches_oracle(M, K, residual):
    x, w = _rand(1, M, K), _rand(2, 1, K, 0.2, 1.0)[0]
    _check_norm(x, _rand(3, M, K, 4.0) if residual else None, w, 1e-6)


def test_add_norm_ends_of_the_types():
    K = 256
    x = f64(_rand(4, 9, K))
    x[0] = 0.0           # nothing: eps keeps it finite
    x[1] *= 2.0 ** -70   # squares near fp32's smallest
    x[2] *= 2.0 ** -120  # and below it
    x[3] *= 2.0 ** 70    # squares past its range
    x[4] *= 2.0 ** 124
    x[5, 3:] = 0.0
    x[6] *= 2.0 ** -126  # numbers below bf16's normal ones
    x = bf16(x)
    w = _rand(5, 1, K, 0.2, 1.0)[0]
    for eps in (1e-6, 0.0 + 2.0 ** -140, 1e-20, 1.0):
        _, y = _check_norm(x, None, w, eps)
        assert not f64(y[0]).any()


def test_add_norm_infinities_and_nan_stay_in_their_rows():
    K = 384
    x, res, w = _rand(6, 5, K), _rand(7, 5, K), _rand(8, 1, K, 0.2, 1.0)[0]
    clean = _norm(x, res, w, 1e-6)
    x = x.copy()
    x[1, 5], x[3, 200] = 0x7F80, 0x7FC0
    s, y, c, e = _norm(x, res, w, 1e-6)
    keep = [0, 2, 4]
    assert np.array_equal(s[keep], clean[0][keep]) and np.array_equal(y[keep], clean[1][keep])
    assert np.isposinf(f64(s[1])[5]) and np.isnan(f64(y[1])[5]) and not f64(y[1])[np.arange(K) != 5].any()
    assert np.isnan(f64(y[3])).all() and np.isnan(f64(s[3])[200])
    v = values8(c, e, 5, K)[2]
    assert np.isnan(v[1, 5]) and np.isnan(v[3]).all()
    assert np.array_equal(v[keep], values8(clean[2], clean[3], 5, K)[2][keep])


def test_add_norm_in_place_and_outputs_left_out():
    M, K = 5, 1152
    x, res, w = _rand(9, M, K), _rand(10, M, K), _rand(11, 1, K, 0.2, 1.0)[0]
    s, y, c, e = _norm(x, res, w, 1e-6)
    xd, rd = dev(x), dev(res)
    ss.subspec_add_norm(xd, rd, dev(w), 1e-6, M, K, rd, xd, None, None)  # the stream and the rows in place
    assert np.array_equal(host(rd), s) and np.array_equal(host(xd), y)
    xd, rd = dev(x), dev(res)
    ss.subspec_add_norm(xd, rd, dev(w), 1e-6, M, K, xd, rd, None, None)
    assert np.array_equal(host(xd), s) and np.array_equal(host(rd), y)
    c2, e2 = rows8(M, K)
    ss.subspec_add_norm(dev(x), dev(res), dev(w), 1e-6, M, K, None, None, c2, e2)
    assert all(np.array_equal(a, b) for a, b in zip(values8(c, e, M, K), values8(c2, e2, M, K)))
    y2 = torch.empty((M, K), dtype=torch.bfloat16, device=DEV)
    ss.subspec_add_norm(dev(x), dev(res), dev(w), 1e-6, M, K, None, y2, None, None)
    assert np.array_equal(host(y2), y)


ACT = [(1, 18944), (6, 18944), (3, 8), (2, 128), (5, 264), (2, 2048), (3, 2056), (2, 27648), (65, 384), (1, 128 * 1025)]


def _act_ref(g, u):
    h = oracle.silu_mul(g, u)
    return h, np.abs(h) * (np.abs(g) * 2.0 ** -23 + 2.0 ** -20)


@pytest.mark.parametrize("M,I", ACT)
def test_silu_mul_matches_oracle(M, I):
    x = _rand(20, M, 2 * I, 3.0)
    eight = I % 128 == 0
    h = torch.full((M * I + 24,), 7.0, dtype=torch.bfloat16, device=DEV)
    c, e = rows8(M, I, 24) if eight else (None, None)
    ss.subspec_silu_mul(dev(x), M, I, h, c, e)
    torch.cuda.synchronize()
    assert bool((h[M * I:] == 7).all())
    ref, add = _act_ref(f64(x[:, :I]), f64(x[:, I:]))
    err, tol = np.abs(f64(host(h[: M * I])).reshape(M, I) - ref), 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -8) + add + 2.0 ** -133
    assert np.all(err <= tol), float((err / tol).max())
    if eight:
        assert bool((c[M * I:] == 0x5A).all()) and bool((e[(I + 511) // 512 * M:] == 0x5A5A5A5A).all())
        check8(c, e, M, I, ref, 2.0 ** -17)  # |g| < 32
        c2, e2 = rows8(M, I)
        ss.subspec_silu_mul(dev(x), M, I, None, c2, e2)
        assert all(np.array_equal(a, b) for a, b in zip(values8(c, e, M, I), values8(c2, e2, M, I)))


def test_silu_mul_far_gates():
    I = 64
    g = np.concatenate([np.linspace(-160, 160, I - 4), [-1e4, 1e4, 0.0, -0.0]])
    g = f64(bf16(g[None]))
    for u in (1.0, -3e30, 2.0 ** -100, 2.0 ** 100):
        x = bf16(np.concatenate([g, np.full((1, I), u)], 1))
        h = torch.empty((1, I), dtype=torch.bfloat16, device=DEV)
        ss.subspec_silu_mul(dev(x), 1, I, h, None, None)
        ref, add = _act_ref(g, f64(x[:, I:]))
        err = np.abs(f64(host(h)) - ref)
        # past |g| = 160 the second half of the exponential may leave fp32's normal numbers
        tol = 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -8) + add + 2.0 ** -133
        ok = (err <= tol) | (np.abs(ref) > 3.3895e38)
        assert ok.all(), (u, g[~ok], err[~ok], ref[~ok])


def test_silu_mul_of_infinities_and_nan():
    x = np.zeros((1, 256), np.float32)
    x[0, :8] = [np.inf, -np.inf, np.nan, 1, 1, 1, 2, 0]
    x[0, 128:136] = [1, 1, 1, np.inf, -np.inf, np.nan, 0, 5]
    h = torch.empty((1, 128), dtype=torch.bfloat16, device=DEV)
    c, e = rows8(1, 128)
    ss.subspec_silu_mul(dev(bf16(x)), 1, 128, h, c, e)
    got = f64(host(h))[0]
    assert np.isposinf(got[0]) and np.isnan(got[1:3]).all() and np.isposinf(got[3]) and np.isneginf(got[4]) and np.isnan(got[5])
    assert not got[6:].any()
    v = values8(c, e, 1, 128)[2][0]
    assert np.isnan(v[:6]).all() and not v[6:].any()


def _wild(seed, M, K):
    """bf16 rows over the whole range: blocks of all scales, zeros, borders, subnormal numbers."""
    rng = np.random.default_rng([seed, M, K])
    x = rng.standard_normal((M, K)).astype(np.float32)
    b = x.reshape(M, K // 128, 128)
    b *= np.exp2(rng.integers(-135, 126, (M, K // 128, 1)).astype(np.float64)).astype(np.float32)
    b[rng.random((M, K // 128)) < 0.1] = 0.0
    near = rng.random((M, K // 128)) < 0.3  # the largest at, above and below 448 times a power
    b[near, 0] = (np.array([1.75, 1.7578125, 1.7421875], np.float32)[rng.integers(0, 3, near.sum())] * np.exp2(rng.integers(-100, 120, near.sum()))).astype(np.float32)
    return bf16(x)


@pytest.mark.parametrize("M,K", [(1, 128), (1, 3584), (3, 640), (7, 2048), (5, 2176), (130, 512), (2, 27648)])
def test_fp8_rows_are_the_oracles_bits(M, K):
    x = _wild(30, M, K)
    if M > 2:
        x[1, 7], x[1, 9], x[2, 300] = 0x7F80, 0xFF80, 0x7FC1
    c, e = rows8(M, K, 24)
    ss.subspec_fp8_rows(dev(x), M, K, c, e)
    y = torch.full((M * K + 24,), 7.0, dtype=torch.bfloat16, device=DEV)
    ss.subspec_fp8_read(c, e, M, K, y)
    torch.cuda.synchronize()
    assert bool((c[M * K:] == 0x5A).all()) and bool((e[(K + 511) // 512 * M:] == 0x5A5A5A5A).all()) and bool((y[M * K:] == 7).all())
    rc, rs = oracle.fp8_rows(f64(x))
    gc, gs, _ = values8(c, e, M, K)
    assert np.array_equal(gs, rs)
    bad = np.isnan(oracle.E4M3[rc])
    assert np.array_equal(gc[~bad], rc[~bad]) and np.isnan(oracle.E4M3[gc[bad]]).all()
    # bytes past the last block are left as they were
    if K % 512:
        last = e[((K + 511) // 512 - 1) * M: (K + 511) // 512 * M].cpu().numpy().view(np.uint8).reshape(M, 4)
        assert (last[:, K // 128 % 4:] == 0x5A).all()
    with np.errstate(over="ignore"):
        ref = f64(bf16(oracle.fp8_values(rc, rs)))
    assert np.array_equal(f64(host(y[: M * K])).reshape(M, K), ref, equal_nan=True)


def test_every_code_reads_as_its_value():
    c = torch.arange(256, dtype=torch.uint8, device=DEV).view(2, 128)
    for byte in (1, 64, 127, 200, 240):
        e = torch.full((1, 2), byte, dtype=torch.int32, device=DEV)
        y = torch.empty((2, 128), dtype=torch.bfloat16, device=DEV)
        ss.subspec_fp8_read(c.view(torch.float8_e4m3fn), e, 2, 128, y)
        ref = f64(bf16(oracle.E4M3.reshape(2, 128) * 2.0 ** (byte - 127)))
        assert np.array_equal(f64(host(y)), ref, equal_nan=True), byte


def test_row_operators_on_another_stream_captured_and_replayed():
    M, K = 37, 1280
    x, res, w = _rand(40, M, K), _rand(41, M, K, 3.0), _rand(42, 1, K, 0.2, 1.0)[0]
    want = _norm(x, res, w, 1e-6)
    s = torch.cuda.Stream()
    got = _norm(x, res, w, 1e-6, stream=s)
    assert np.array_equal(want[0], got[0]) and np.array_equal(want[1], got[1])
    xd, rd, wd = dev(x), dev(res), dev(w)
    y, h = torch.empty_like(xd), torch.empty((M, K // 2), dtype=torch.bfloat16, device=DEV)
    c, e = rows8(M, K // 2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ss.subspec_add_norm(xd, rd, wd, 1e-6, M, K, None, y, None, None)
        ss.subspec_silu_mul(y, M, K // 2, h, c, e)
    for k in range(3):
        xd.copy_(dev(np.roll(x, k, 0)))
        rd.copy_(dev(np.roll(res, k, 0)))
        h.zero_(), c.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(host(y), np.roll(want[1], k, 0)), k
        h2, (c2, e2) = torch.empty_like(h), rows8(M, K // 2)
        ss.subspec_silu_mul(y, M, K // 2, h2, c2, e2)
        assert torch.equal(h.view(torch.int16), h2.view(torch.int16)) and torch.equal(c, c2)
        assert np.array_equal(values8(c, e, M, K // 2)[1], values8(c2, e2, M, K // 2)[1])
