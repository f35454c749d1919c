"""GPU parity of the preparation of queries, keys and values against the fp64 oracle.

Tolerance, from the arithmetic: outputs are rounded once to bf16 (2^-8 relative).  Before
that, in fp32: the bias sum (2^-24 of a value below its rounding's scale), the norm (a sum of
128 squares in a tree, a root, a division, two products: at most 16 roundings, 2^-20
relative), cos and sin (the angle's fraction of a turn to 2^-25, so 2^-22 absolute, and 2 ulp
of the function), two products and a sum.  All of it is below 2^-19 of |a| + |b| of a
pair, which does not shrink when the pair's two products cancel.  Value heads carry one fp32 sum
of two bf16 numbers: 2^-24 of |row| + |bias|."""
import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss
from paper_2509_18344_amd import synth

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"


def _bits(rng, *shape, scale=1.0, mean=0.0):
    a = (rng.standard_normal(shape, dtype=np.float32) * np.float32(scale) + np.float32(mean))
    return synth.bf16_bits(torch.from_numpy(a).to(torch.bfloat16))


def _dev(bits):
    return None if bits is None else torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(DEV)


def _inputs(M, Hq, Hkv, rot, bias, norm, far, seed, pad=0):
    rng = np.random.default_rng([M, Hq, Hkv, rot, seed])
    heads = Hq + 2 * Hkv
    return dict(qkv=_bits(rng, M, heads * 128 + pad, scale=1.5), bias=_bits(rng, heads * 128, scale=2.0) if bias else None,
                qw=_bits(rng, 128, scale=0.2, mean=1.0) if norm else None,
                kw=_bits(rng, 128, scale=0.2, mean=1.0) if norm else None,
                pos=rng.integers(0, far, M).astype(np.int32),
                freq=np.array([1e6 ** (-2.0 * i / rot) for i in range(rot // 2)], np.float64))


def _run(x, M, Hq, Hkv, rot, interleaved, eps, stream=None):
    new = lambda h: torch.full((M + 1, h, 128), -7, dtype=torch.int16, device=DEV)  # noqa: E731
    q, k, v = new(Hq), new(Hkv), new(Hkv)
    torch.cuda.synchronize()  # the call may run on another stream
    ss.subspec_qkv_rope(_dev(x["qkv"]), x["qkv"].shape[1], _dev(x["bias"]), _dev(x["qw"]), _dev(x["kw"]), eps,
                        torch.from_numpy(x["pos"]).to(DEV), torch.from_numpy(x["freq"]).to(DEV) if rot else None, rot,
                        interleaved, M, Hq, Hkv, q, k, v, stream)
    torch.cuda.synchronize()
    for t in (q, k, v):
        assert bool((t[M] == -7).all())  # rows past the last are left as they were
    return [oracle.bf16_bits_to_f64(t[:M].cpu().numpy().view(np.uint16)) for t in (q, k, v)]


def _check(x, M, Hq, Hkv, rot, interleaved, eps=1e-6):
    got = _run(x, M, Hq, Hkv, rot, interleaved, eps)
    ref = oracle.qkv_rope(x["qkv"], x["bias"], x["qw"], x["kw"], eps, x["pos"], x["freq"], rot, interleaved, Hq, Hkv)
    still = oracle.qkv_rope(x["qkv"], x["bias"], x["qw"], x["kw"], eps, x["pos"], x["freq"], 0, interleaved, Hq, Hkv)
    for name, o, r, s in zip("qkv", got, ref, still):
        pair = np.abs(s)
        if rot and name != "v":
            a, b = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if interleaved else (np.arange(rot // 2), np.arange(rot // 2, rot))
            both = np.abs(s[..., a]) + np.abs(s[..., b])
            pair[..., a], pair[..., b] = both, both
        tol = 2.0 ** -8 * np.abs(r) + 2.0 ** -19 * pair
        if name == "v" and x["bias"] is not None:
            tol = tol + 2.0 ** -23 * 16
        err = np.abs(o - r)
        assert np.all(err <= tol), (name, float(err.max()), float((err / tol).max()))
    return got


@pytest.mark.parametrize("M,Hq,Hkv,rot,interleaved,bias,norm,far", [
    (1, 28, 4, 128, False, True, False, 131072),   # a single token, Qwen2.5-7B
    (6, 28, 4, 128, False, True, True, 3000),
    (37, 40, 8, 128, False, False, True, 32768),   # Qwen2.5-32B heads
    (5, 1, 1, 128, False, True, True, 100),        # three heads: most of a workgroup idle
    (3, 7, 3, 128, True, True, False, 70000),
    (4, 16, 16, 64, False, False, True, 5000),     # a part of the head rotates
    (4, 5, 2, 96, True, True, True, 5000),
    (2, 12, 2, 16, False, False, False, 200),
    (2, 12, 2, 0, False, True, True, 200),         # no rotation
    (3, 4, 2, 128, False, False, False, 2 ** 31 - 1),  # positions to the end of int32
])
def test_qkv_rope_matches_oracle(M, Hq, Hkv, rot, interleaved, bias, norm, far):
    _check(_inputs(M, Hq, Hkv, max(rot, 2), bias, norm, far, 1), M, Hq, Hkv, rot, interleaved)


def test_qkv_rope_row_stride_and_positions_of_either_sign():
    x = _inputs(9, 6, 2, 128, True, True, 4096, 2, pad=72)
    x["pos"][:3] = [0, -1, -70000]
    _check(x, 9, 6, 2, 128, False)


def test_qkv_rope_zero_row_and_values_near_the_types_ends():
    x = _inputs(4, 3, 1, 128, False, True, 64, 3)
    f = oracle.bf16_bits_to_f64(x["qkv"])
    f[0] = 0.0          # norm of nothing: eps keeps it finite
    f[1] *= 2.0 ** -60  # squares below fp32's range next to eps
    f[2] *= 2.0 ** 50
    x["qkv"] = oracle.bf16_round_bits(f.astype(np.float32))
    got = _check(x, 4, 3, 1, 128, False)
    assert not got[0][0].any()


def test_qkv_rope_many_rows_on_a_stream_of_its_own():
    M, Hq, Hkv = 700, 3, 1
    x = _inputs(M, Hq, Hkv, 128, True, True, 100000, 4)
    a = _check(x, M, Hq, Hkv, 128, False)
    s = torch.cuda.Stream()
    b = _run(x, M, Hq, Hkv, 128, False, 1e-6, s)
    for u, w in zip(a, b):
        assert np.array_equal(u, w)
