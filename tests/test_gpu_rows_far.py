"""The gated activation at gates far below zero, where sigmoid(g) leaves fp32's normal numbers and a large
second factor brings the result back.

Tolerances: those of test_gpu_rows.py (|g| 2^-23 + 2^-20 before the rounding to bf16, 2^-133 absolute where
the result is below bf16's normal numbers).  For |g| < 256 the first is below 2^-14."""
import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss

from test_gpu_rows import DEV, _act_ref, bf16, check8, dev, f64, host, rows8

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TOP = 3.3895e38  # bf16's largest


def _run(g, u):
    """(h, codes, scales) of gates and second factors [M][I]."""
    M, I = g.shape
    x = bf16(np.concatenate([g, u], 1))
    h, (c, e) = torch.empty((M, I), dtype=torch.bfloat16, device=DEV), rows8(M, I)
    ss.subspec_silu_mul(dev(x), M, I, h, c, e)
    torch.cuda.synchronize()
    return f64(x[:, :I]), f64(x[:, I:]), f64(host(h)), c, e


@pytest.mark.parametrize("u", [TOP, -TOP, 1e38, -2.0 ** 122, 2.0 ** 110, 1.0])
def test_silu_mul_below_the_smallest_sigmoid(u):
    g = np.concatenate([np.linspace(-195.0, -130.0, 251), [-256.0, -1e4, -TOP, 0.0, -0.0]])[None]
    g, uu, h, c, e = _run(g, np.full(g.shape, u))
    ref, add = _act_ref(g, uu)
    if abs(u) == TOP:  # what the test is for: results of normal size past the gate where the sigmoid is not
        assert np.any((g < -175) & (np.abs(ref) > 2.0 ** -120))
    err, tol = np.abs(h - ref), 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -8) + add + 2.0 ** -133
    assert np.all(err <= tol), (g[err > tol], h[err > tol], ref[err > tol])
    check8(c, e, 1, 256, ref, 2.0 ** -14)


def test_far_gates_leave_the_others_as_they_are():
    # the same values with and without a far gate beside them
    rng = np.random.default_rng(70)
    g, u = rng.standard_normal((4, 1280)) * 20, rng.standard_normal((4, 1280)) * 50
    _, _, h0, c0, e0 = _run(g, u)
    far = np.zeros(g.shape, bool)
    far[:, ::97] = True
    _, _, h1, _, _ = _run(np.where(far, -180.0, g), u)
    assert np.array_equal(h0[~far], h1[~far])
    _, _, h2, _, _ = _run(np.where(far, -np.inf, g), u)
    assert np.array_equal(h0[~far], h2[~far]) and np.isnan(h2[far]).all()
    _, _, h3, _, _ = _run(np.where(far, 0.0, g), np.where(far, 0.0, u))
    assert np.array_equal(h0[~far], h3[~far]) and not h3[far].any()
