"""The preparation of queries, keys and values where a head is rotated in part: dimensions past `rot`
come through as they are, infinities and NaN included, and keep to themselves."""
import numpy as np
import pytest

import oracle
from test_gpu_rope import _check, _inputs, _run

pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [3, 330])  # a workgroup for every 16 heads, or one a token
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [16, 64, 96, 112])
def test_qkv_rope_passes_what_it_does_not_rotate(M, rot, interleaved):
    Hq, Hkv = 3, 2
    x = _inputs(M, Hq, Hkv, rot, False, False, 5000, 6)
    rows = x["qkv"].reshape(M, Hq + 2 * Hkv, 128)
    clean = _run(x, M, Hq, Hkv, rot, interleaved, 1e-6)
    rng = np.random.default_rng([rot, interleaved])
    odd = np.array([0x7F80, 0xFF80, 0x7FC0], np.uint16)  # infinities and NaN
    where = np.zeros(rows.shape, bool)
    where[..., rot:] = rng.random((M, Hq + 2 * Hkv, 128 - rot)) < 0.2
    rows[where] = rng.choice(odd, int(where.sum()))
    got = _run(x, M, Hq, Hkv, rot, interleaved, 1e-6)
    src = oracle.bf16_bits_to_f64(rows)
    h0 = 0
    for o, c in zip(got, clean):
        h1 = h0 + o.shape[1]
        assert np.array_equal(o[..., rot:], src[:, h0:h1, rot:], equal_nan=True)
        assert np.array_equal(o[..., :rot], c[..., :rot])
        h0 = h1


@pytest.mark.parametrize("rot,interleaved", [(128, False), (64, False), (96, True), (0, False)])
def test_qkv_rope_a_workgroup_that_takes_its_tokens_heads_in_turns(rot, interleaved):
    """From 320 tokens on a workgroup takes 64 heads at a time: 80 heads take a second turn.  The bits are
    those of the same rows in smaller batches, which the oracle is compared with."""
    M, Hq, Hkv = 323, 64, 8
    x = _inputs(M, Hq, Hkv, max(rot, 2), True, True, 100000, 7)
    got = _run(x, M, Hq, Hkv, rot, interleaved, 1e-6)
    for r0, r1 in ((0, 300), (300, M)):
        part = dict(x, qkv=x["qkv"][r0:r1], pos=x["pos"][r0:r1])
        for o, p in zip(got, _run(part, r1 - r0, Hq, Hkv, rot, interleaved, 1e-6)):
            assert np.array_equal(o[r0:r1], p)
    few = dict(x, qkv=x["qkv"][319:], pos=x["pos"][319:])
    for o, p in zip(got, _check(few, 4, Hq, Hkv, rot, interleaved)):
        assert np.array_equal(o[319:], p)
