"""Every kind of launch of the product in 8-bit floating point, held sharply: whole numbers exactly, each
cut of eight products where the 8-bit matrix units make it, bf16 rows bit for bit as their 8-bit rows, and rows
and blocks of zeros.  About 200 rows and columns of each result, the ends of every tile's among them.

Tolerances.  Whole numbers up to 256 have no rounding.  Else, against sums in 64 bits of the products as the
units leave them (above EXACT rows cut towards zero to a multiple of 2^(E - 13), E the largest sum of two
exponents among eight neighbouring k): K / 128 + 32 roundings of 2^-23 W, W the sum of magnitudes, and
one to bf16, 2^-8."""
import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss

from test_gpu_fp8 import DEV, EXACT, KINDS, _random_rows, _tiled_weight, codes_to, linear, weight
from test_gpu_rows import bf16, dev, rows8

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# the few rows' kernel: eight and sixteen wavefronts around the lines between them, two tiles a wavefront, parts of K
FEW = [(1, 272, 2048), (5, 272, 2176), (1, 3584, 4096), (16, 3584, 4224), (2, 4096, 5120), (9, 48, 8192), (3, 4112, 8192), (7, 48, 8320),
       (16, 8208, 640), (4, 512, 9216), (30, 512, 640), (33, 272, 2176), (64, 16, 4096)]


def _pick(n):
    """The first and last rows, and the ends of tiles between."""
    step = max(32, n // 64 // 32 * 32)
    return np.unique(np.r_[np.arange(min(n, 35)), np.arange(max(0, n - 70), n), np.arange(31, n, step), np.arange(32, n, step)])


def _some(y, m, n):
    return y[torch.from_numpy(m).to(DEV)][:, torch.from_numpy(n).to(DEV)].double().cpu().numpy()


@pytest.mark.parametrize("M,N,K", [*KINDS, *FEW])
def test_whole_numbers_are_exact(M, N, K):
    rng = np.random.default_rng([71, M, N, K])
    p = rng.integers(-30, 31, K // 128)  # powers that differ from block to block and cancel
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


def _cut_sums(x8, w8, cut):
    """(sums of the products as the units leave them, sums of magnitudes) in 64 bits, on the GPU."""
    def side(codes, bytes_):
        e = np.maximum((codes >> 3 & 15).astype(int), 1) - 7 + np.repeat(bytes_.astype(int) - 127, 128, 1)
        return torch.from_numpy(oracle.fp8_values(codes, bytes_)).to(DEV), torch.from_numpy(e.astype(np.float64)).to(DEV)
    (xv, xe), (wv, we) = side(*x8), side(*w8)
    ref, size = (torch.empty((len(xv), len(wv)), dtype=torch.float64, device=DEV) for _ in range(2))
    for m in range(len(xv)):
        p = (xv[m] * wv).view(len(wv), -1, 8)
        size[m] = p.abs().sum((1, 2))
        if cut:
            grid = torch.exp2((xe[m] + we).view(len(wv), -1, 8).amax(-1, keepdim=True) - 13.0)
            p = torch.trunc(p / grid) * grid
        ref[m] = p.sum((1, 2))
    return ref.cpu().numpy(), size.cpu().numpy()


def _check(y, x8, w8, M, K):
    ref, size = _cut_sums(x8, w8, M > EXACT)
    err, tol = np.abs(y - ref), 2.0 ** -8 * np.abs(ref) + (K / 128 + 32) * 2.0 ** -23 * size
    assert np.all(err <= tol), (float((err / np.maximum(tol, 1e-300)).max()), np.argwhere(err > tol)[:4].tolist())


@pytest.mark.parametrize("M,N,K", [*KINDS, *FEW])
def test_every_cut_and_nothing_else(M, N, K):
    rng = np.random.default_rng([72, M, N, K])
    x8, w8 = _random_rows(rng, M, K), _tiled_weight(rng, N, K)
    y = linear(*codes_to(*x8), *weight(*w8), M, N, K)
    m, n = _pick(M), _pick(N)
    _check(_some(y, m, n), tuple(a[m] for a in x8), tuple(a[n] for a in w8), M, K)


@pytest.mark.parametrize("M,N,K", [*KINDS, *FEW])
def test_bf16_rows_give_the_bits_of_their_8_bit_rows_in_every_kind(M, N, K):
    rng = np.random.default_rng([73, M, N, K])
    x = rng.standard_normal((M, K)) * np.repeat(np.exp2(rng.integers(-4, 5, (M, K // 128))), 128, 1)
    x[rng.random((M, K)) < 0.01] *= 500.0  # and some far larger ones
    xd = dev(bf16(x))
    t, ws = weight(*_tiled_weight(rng, N, K))
    c, s = rows8(M, K)
    ss.subspec_fp8_rows(xd, M, K, c, s)
    y8 = linear(c, s, t, ws, M, N, K).view(torch.int16)
    assert ss.subspec_fp8_linear_plan(M, N, K)[0] == (KINDS[M, N, K][0] if (M, N, K) in KINDS else 0)
    for _ in range(2):  # codes and partial sums share the workspace
        assert torch.equal(linear(xd, None, t, ws, M, N, K).view(torch.int16), y8)


# few rows in their launches of one and two tiles a wavefront, and what the exact small and large tiles take
ZEROS = [(5, 512, 2304), (16, 5120, 1152), (7, 512, 18944), (30, 512, 640), (40, 272, 2176)] + [k for k in KINDS if k[0] <= 200]


@pytest.mark.parametrize("M,N,K", ZEROS)
def test_rows_and_blocks_of_zeros_change_no_bit_of_the_others(M, N, K):
    rng = np.random.default_rng([74, M, N, K])
    x8, w8 = _random_rows(rng, M, K), _tiled_weight(rng, N, K)
    KB = K // 128
    y = linear(*codes_to(*x8), *weight(*w8), M, N, K)
    xz, wz = (tuple(a.copy() for a in r) for r in (x8, w8))
    empty, dead = np.arange(M) % 3 == 1, np.arange(N) % 5 == 2  # padding rows, columns of a weight that was cut away
    xz[0][empty], xz[1][empty] = 0, 1  # as subspec_fp8_rows makes them
    wz[0][dead], wz[1][dead] = 0x80, 1  # negative zeros too
    z = linear(*codes_to(*xz), *weight(*wz), M, N, K)
    off = torch.from_numpy(empty[:, None] | dead[None]).to(DEV)
    assert not bool(z[off].any())
    assert torch.equal(z[~off].view(torch.int16), y[~off].view(torch.int16))
    # a block of zeros in some rows and columns: the product without it
    xz, wz = (tuple(a.copy() for a in r) for r in (x8, w8))
    at = KB // 2
    xz[0][empty, 128 * at:128 * at + 128], xz[1][empty, at] = 0, 1
    wz[0][dead, :128], wz[1][dead, 0] = 0, 1
    z = linear(*codes_to(*xz), *weight(*wz), M, N, K)
    m, n = _pick(M), _pick(N)
    _check(_some(z, m, n), tuple(a[m] for a in xz), tuple(a[n] for a in wz), M, K)
    assert torch.equal(z[~off].view(torch.int16), y[~off].view(torch.int16))
    if M <= 32:  # bf16 rows of zeros, turned into codes on the way
        x = bf16(rng.standard_normal((M, K)))
        t, ws = weight(*w8)
        y = linear(dev(x), None, t, ws, M, N, K)
        x[empty] = 0
        z = linear(dev(x), None, t, ws, M, N, K)
        off = torch.from_numpy(empty).to(DEV)
        assert not bool(z[off].any()) and torch.equal(z[~off].view(torch.int16), y[~off].view(torch.int16))
