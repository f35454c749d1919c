"""CPU checks of the row operators and of the product in 8-bit floating point: refusals before any GPU
work, what the binding checks, workspace sizes, and pins of their oracle."""
import math

import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss
from test_binding_checks_cpu import BF, F32, I32, U8, Fake, calls  # noqa: F401

torch = pytest.importorskip("torch")
A = 4096  # an aligned address that no call may touch


def refused(kind):
    return pytest.raises(ss.SubspecError, match=kind)


def _norm(**kw):
    a = dict(x=A, res=A, w=A, eps=1e-6, M=1, K=256, sum=A, y=2 * A, codes=3 * A, scales=4 * A)
    a.update(kw)
    return ss.subspec_add_norm(a["x"], a["res"], a["w"], a["eps"], a["M"], a["K"], a["sum"], a["y"], a["codes"], a["scales"], stream=0)


@pytest.mark.parametrize("kw,kind", [
    (dict(x=None), "EINVAL"), (dict(w=None), "EINVAL"), (dict(codes=None), "EINVAL"), (dict(scales=None), "EINVAL"),
    (dict(y=None, codes=None, scales=None), "EINVAL"), (dict(x=A + 8), "EINVAL"), (dict(res=A + 2), "EINVAL"), (dict(w=A + 4), "EINVAL"),
    (dict(sum=A + 8), "EINVAL"), (dict(y=A + 8), "EINVAL"), (dict(codes=A + 8), "EINVAL"), (dict(scales=A + 2), "EINVAL"),
    (dict(sum=A, y=A), "EINVAL"), (dict(eps=-1.0), "EINVAL"), (dict(eps=math.nan), "EINVAL"), (dict(eps=math.inf), "EINVAL"),
    (dict(M=0), "EUNSUPPORTED"), (dict(M=(1 << 20) + 1), "EUNSUPPORTED"), (dict(K=0), "EUNSUPPORTED"), (dict(K=264), "EUNSUPPORTED"),
    (dict(K=65664), "EUNSUPPORTED"), (dict(codes=None, scales=None, K=260), "EUNSUPPORTED"), (dict(K=-128), "EUNSUPPORTED"),
])
def test_add_norm_refusals(kw, kind):
    with refused(kind):
        _norm(**kw)


def _act(**kw):
    a = dict(gu=A, M=1, I=256, h=A, codes=A, scales=A)
    a.update(kw)
    return ss.subspec_silu_mul(a["gu"], a["M"], a["I"], a["h"], a["codes"], a["scales"], stream=0)


@pytest.mark.parametrize("kw,kind", [
    (dict(gu=None), "EINVAL"), (dict(gu=A + 8), "EINVAL"), (dict(codes=None), "EINVAL"), (dict(scales=None), "EINVAL"),
    (dict(h=None, codes=None, scales=None), "EINVAL"), (dict(h=A + 4), "EINVAL"), (dict(codes=A + 8), "EINVAL"),
    (dict(scales=A + 1), "EINVAL"), (dict(M=0), "EUNSUPPORTED"), (dict(M=(1 << 20) + 1), "EUNSUPPORTED"), (dict(I=0), "EUNSUPPORTED"),
    (dict(I=136), "EUNSUPPORTED"), (dict(I=(1 << 23) + 128), "EUNSUPPORTED"), (dict(codes=None, scales=None, I=12), "EUNSUPPORTED"),
])
def test_silu_mul_refusals(kw, kind):
    with refused(kind):
        _act(**kw)


@pytest.mark.parametrize("args,kind", [
    ((None, 1, 128, A, A), "EINVAL"), ((A, 1, 128, None, A), "EINVAL"), ((A, 1, 128, A, None), "EINVAL"),
    ((A + 8, 1, 128, A, A), "EINVAL"), ((A, 1, 128, A + 8, A), "EINVAL"), ((A, 1, 128, A, A + 2), "EINVAL"),
    ((A, 0, 128, A, A), "EUNSUPPORTED"), ((A, (1 << 20) + 1, 128, A, A), "EUNSUPPORTED"), ((A, 1, 0, A, A), "EUNSUPPORTED"),
    ((A, 1, 192, A, A), "EUNSUPPORTED"), ((A, 1, (1 << 24) + 128, A, A), "EUNSUPPORTED"), ((A, 1 << 20, 1 << 21, A, A), "EUNSUPPORTED"),
])
def test_fp8_rows_and_read_refusals(args, kind):
    x, M, K, codes, scales = args
    with refused(kind):
        ss.subspec_fp8_rows(x, M, K, codes, scales, stream=0)
    with refused(kind):
        ss.subspec_fp8_read(codes, scales, M, K, x, stream=0)


@pytest.mark.parametrize("args,kind", [
    ((None, 16, 128, A), "EINVAL"), ((A, 16, 128, None), "EINVAL"), ((A, 16, 128, A), "EINVAL"), ((A + 8, 16, 128, 2 * A), "EINVAL"),
    ((A, 16, 128, 2 * A + 4), "EINVAL"), ((A, 8, 128, 2 * A), "EUNSUPPORTED"), ((A, 0, 128, 2 * A), "EUNSUPPORTED"),
    ((A, 16, 64, 2 * A), "EUNSUPPORTED"), ((A, (1 << 24) + 16, 128, 2 * A), "EUNSUPPORTED"), ((A, 1 << 24, 1 << 17, 2 * A), "EUNSUPPORTED"),
])
def test_fp8_pack_refusals(args, kind):
    with refused(kind):
        ss.subspec_fp8_pack(*args, stream=0)


def _linear(**kw):
    a = dict(x=A, xs=A, w=A, ws=A, M=1, N=16, K=128, y=A)
    a.update(kw)
    return ss.subspec_fp8_linear(a["x"], a["xs"], a["w"], a["ws"], a["M"], a["N"], a["K"], a["y"], stream=0)


@pytest.mark.parametrize("kw,kind", [
    (dict(x=None), "EINVAL"), (dict(w=None), "EINVAL"), (dict(ws=None), "EINVAL"), (dict(y=None), "EINVAL"), (dict(x=A + 8), "EINVAL"),
    (dict(w=A + 8), "EINVAL"), (dict(y=A + 8), "EINVAL"), (dict(xs=A + 2), "EINVAL"), (dict(ws=A + 1), "EINVAL"),
    (dict(M=0), "EUNSUPPORTED"), (dict(M=(1 << 20) + 1), "EUNSUPPORTED"), (dict(N=0), "EUNSUPPORTED"), (dict(N=24), "EUNSUPPORTED"),
    (dict(N=(1 << 24) + 16), "EUNSUPPORTED"), (dict(K=0), "EUNSUPPORTED"), (dict(K=192), "EUNSUPPORTED"), (dict(K=(1 << 24) + 128), "EUNSUPPORTED"),
    (dict(M=1 << 20, K=1 << 21), "EUNSUPPORTED"), (dict(N=1 << 20, K=1 << 21), "EUNSUPPORTED"), (dict(M=1 << 20, N=1 << 21), "EUNSUPPORTED"),
])
def test_fp8_linear_refusals(kw, kind):
    with refused(kind):
        _linear(**kw)
    if "M" in kw or "N" in kw or "K" in kw:
        assert ss.subspec_fp8_linear_workspace_bytes(kw.get("M", 1), kw.get("N", 16), kw.get("K", 128), 0) == 0


def test_fp8_linear_workspace():
    # whatever else it holds: bf16 rows of a large batch leave their codes and scales there
    for M, N, K in ((4096, 512, 1280), (300, 16, 128)):
        assert ss.subspec_fp8_linear_workspace_bytes(M, N, K, 0) >= M * K + 4 * M * ((K + 511) // 512)
    assert ss.subspec_fp8_linear_workspace_bytes(4096, 512, 1280, 2) == 0


def test_every_kind_of_launch_is_reached():
    from test_gpu_fp8 import KINDS
    for (M, N, K), (kernel, rows, columns, shared, several) in KINDS.items():
        k, r, c, groups, sharing = ss.subspec_fp8_linear_plan(M, N, K)
        assert (k, r, c, sharing > 1) == (kernel, rows, columns, shared), (M, N, K)
        tiles = -(-M // rows) * -(-N // columns)
        assert (groups > 256 if k == 1 else tiles > groups) == several, (M, N, K, groups)
        assert groups <= tiles * sharing
    kinds = {v[:3] for v in KINDS.values()}
    rng = np.random.default_rng(0)
    for _ in range(3000):  # and no other is
        M, N, K = (int(np.exp(rng.uniform(np.log(lo), np.log(hi)))) for lo, hi in ((1, 5000), (1, 4000), (1, 220)))
        p = ss.subspec_fp8_linear_plan(M, 16 * N, 128 * K)
        assert p[:3] in kinds if p[0] else p[1] == (M + 15) // 16 * 16 and M <= 64 and p[2] in (16, 32), (M, N, K, p)


@pytest.mark.parametrize("shape", [(0, 16, 128), (1, 24, 128), (1, 16, 192), (1 << 20, 1 << 21, 128)])
def test_fp8_linear_plan_refusals(shape):
    with refused("EUNSUPPORTED"):
        ss.subspec_fp8_linear_plan(*shape)


# --- what the binding checks ----------------------------------------------------------------

M, K, I, N = 3, 640, 384, 48
CALLS = {
    "norm": (lambda a: ss.subspec_add_norm(a["x"], a["res"], a["w"], 1e-6, M, K, a["sum"], a["y"], a["codes"], a["scales"]),
             dict(x=(BF, M * K), res=(BF, M * K), w=(BF, K), sum=(BF, M * K), y=(BF, M * K), codes=(U8, M * K), scales=(I32, 2 * M))),
    "act": (lambda a: ss.subspec_silu_mul(a["gu"], M, I, a["h"], a["codes"], a["scales"]),
            dict(gu=(BF, 2 * M * I), h=(BF, M * I), codes=(U8, M * I), scales=(I32, M))),
    "rows": (lambda a: ss.subspec_fp8_rows(a["x"], M, K, a["codes"], a["scales"]),
             dict(x=(BF, M * K), codes=(U8, M * K), scales=(I32, 2 * M))),
    "read": (lambda a: ss.subspec_fp8_read(a["codes"], a["scales"], M, K, a["y"]),
             dict(codes=(U8, M * K), scales=(I32, 2 * M), y=(BF, M * K))),
    "pack": (lambda a: ss.subspec_fp8_pack(a["codes"], N, K, a["tiles"]), dict(codes=(U8, N * K), tiles=(U8, N * K))),
    "linear": (lambda a: ss.subspec_fp8_linear(a["x"], None, a["w"], a["ws"], M, N, K, a["y"]),
               dict(x=(BF, M * K), w=(U8, N * K), ws=(I32, 2 * N), y=(BF, M * N))),
    "linear8": (lambda a: ss.subspec_fp8_linear(a["x"], a["xs"], a["w"], a["ws"], M, N, K, a["y"]),
                dict(x=(U8, M * K), xs=(I32, 2 * M), w=(U8, N * K), ws=(I32, 2 * N), y=(BF, M * N))),
}
EACH = [(call, name) for call in CALLS for name in CALLS[call][1]]
OTHER = {BF: [torch.float16, F32, U8], I32: [torch.int64, F32, torch.int16], U8: [BF, I32, torch.float8_e5m2]}


def _args(call, **changed):
    return {n: changed.get(n, Fake(*spec)) for n, spec in CALLS[call][1].items()}


@pytest.mark.parametrize("call", CALLS)
def test_tensors_of_exactly_the_size_needed_pass(calls, call):  # noqa: F811
    CALLS[call][0](_args(call))
    assert len(calls) == 1
    for name, (dtype, n) in CALLS[call][1].items():
        if dtype == U8:  # codes under their own type
            CALLS[call][0](_args(call, **{name: Fake(torch.float8_e4m3fn, n)}))
        if dtype == I32:  # scales as bytes
            for t in (U8, torch.float8_e8m0fnu):
                CALLS[call][0](_args(call, **{name: Fake(t, 4 * n)}))


@pytest.mark.parametrize("call,name", EACH)
def test_a_tensor_too_small_or_of_another_type_is_refused(calls, call, name):  # noqa: F811
    dtype, n = CALLS[call][1][name]
    for bad in [Fake(dtype, n - 1)] + [Fake(t, n) for t in OTHER[dtype]] + [Fake(U8, 4 * n - 1)] * (dtype == I32):
        with refused("EINVAL"):
            CALLS[call][0](_args(call, **{name: bad}))
    assert not calls


# --- pins of the oracle ---------------------------------------------------------------------

def test_codes_are_torchs_e4m3_numbers():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oracle.E4M3, t, equal_nan=True)
    rng = np.random.default_rng(3)
    v = np.concatenate([rng.uniform(-448, 448, 2000), rng.uniform(-0.02, 0.02, 2000), oracle.E4M3[:127],
                        (oracle.E4M3[:126] + oracle.E4M3[1:127]) / 2, [0.0, -0.0, 2.0 ** -10, -2.0 ** -10, 448.0]]).astype(np.float32)
    assert np.array_equal(oracle.e4m3_code(v), torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_blocks_take_the_smallest_power_that_holds_them():
    x = np.zeros((1, 896))
    for b, top in enumerate((448.0, 448.0001, 1.75, 0.0, 2.0 ** -133, 3.3895e38, -7.0)):
        x[0, 128 * b + 5] = top
    codes, s = oracle.fp8_rows(x)
    assert s.tolist() == [[127, 128, 119, 1, 1, 247, 121]]
    assert np.allclose(oracle.fp8_values(codes, s)[0, 5::128], x[0, 5::128], rtol=2.0 ** -4, atol=2.0 ** -136)
    w = oracle.scale_words(s, fill=9)
    assert w.tolist() == [[127 | 128 << 8 | 119 << 16 | 1 << 24], [1 | 247 << 8 | 121 << 16 | 9 << 24]]
    assert np.array_equal(oracle.scale_bytes(w, 896), s)


def test_weight_tiles_hold_every_code_once():
    c = np.arange(32 * 256).reshape(32, 256)
    t = np.empty(32 * 256, np.int64)
    n, k = np.divmod(c, 256)
    at = oracle.weight_tiles((c % 251).astype(np.uint8))
    t = [(16 * (i // 4096) + i % 256 // 16) * 256 + 128 * (i // 2048 % 2) + 64 * (i // 1024 % 2) + 16 * (i // 256 % 4) + i % 16 for i in range(32 * 256)]
    assert sorted(t) == list(range(32 * 256))
    assert np.array_equal(at, (np.array(t) % 251).astype(np.uint8)) and n.max() == 31 and k.max() == 255


def test_oracle_of_the_row_operators():
    x = np.array([[3.0, 4.0]])
    s, y = oracle.add_norm(x, np.array([[0.0, -8.0]]), np.array([1.0, 2.0]), 0.0)
    assert np.allclose(s, [[3, -4]]) and np.allclose(y, np.array([[3, -8]]) / math.sqrt(12.5))
    assert np.allclose(oracle.silu_mul(np.array([0.0, 1.0, -1.0, -800.0]), np.array([5.0, 2.0, 3.0, 1.0])),
                       [0.0, 2 / (1 + math.exp(-1)), -3 / (1 + math.e), 0.0])
