"""CPU checks of the 8-bit product with exact products at any number of rows: refusals before any GPU work,
its plans and workspace, and what the binding checks."""
import pytest

import paper_2509_18344_amd as ss
from test_binding_checks_cpu import BF, I32, U8, Fake, calls  # noqa: F401

torch = pytest.importorskip("torch")
A = 4096


def _linear(**kw):
    a = dict(x=A, xs=A, w=A, ws=A, M=1, N=16, K=128, y=A)
    a.update(kw)
    return ss.subspec_fp8_linear_exact(a["x"], a["xs"], a["w"], a["ws"], a["M"], a["N"], a["K"], a["y"], stream=0)


@pytest.mark.parametrize("kw,kind", [
    (dict(x=None), "EINVAL"), (dict(w=None), "EINVAL"), (dict(ws=None), "EINVAL"), (dict(y=None), "EINVAL"), (dict(x=A + 8), "EINVAL"),
    (dict(y=A + 8), "EINVAL"), (dict(xs=A + 2), "EINVAL"), (dict(ws=A + 1), "EINVAL"), (dict(M=0), "EUNSUPPORTED"),
    (dict(M=(1 << 20) + 1), "EUNSUPPORTED"), (dict(N=24), "EUNSUPPORTED"), (dict(K=192), "EUNSUPPORTED"), (dict(M=1 << 20, N=1 << 21), "EUNSUPPORTED"),
])
def test_refusals(kw, kind):
    with pytest.raises(ss.SubspecError, match=kind):
        _linear(**kw)
    if not {"M", "N", "K"}.isdisjoint(kw):
        shape = kw.get("M", 1), kw.get("N", 16), kw.get("K", 128)
        assert ss.subspec_fp8_linear_exact_workspace_bytes(*shape, 0) == 0
        with pytest.raises(ss.SubspecError, match=kind):
            ss.subspec_fp8_linear_exact_plan(*shape)


def test_every_kind_of_launch_is_reached():
    from test_gpu_fp8_exact import KINDS
    for (M, N, K), (kernel, rows, columns, shared, several) in KINDS.items():
        k, r, c, groups, sharing = ss.subspec_fp8_linear_exact_plan(M, N, K)
        assert (k, r, c, sharing > 1) == (kernel, rows, columns, shared), (M, N, K)
        tiles = -(-M // rows) * -(-N // columns)
        assert (groups > 256 if k == 1 else tiles > groups) == several, (M, N, K, groups)
        assert groups <= tiles * sharing


@pytest.mark.parametrize("M", [65, 100, 289, 1000, 4096, 100000, 1 << 20])
@pytest.mark.parametrize("N,K", [(16, 128), (3584, 18944), (55296, 5120), (1 << 20, 256)])
def test_a_launch_for_every_size(M, N, K):
    kernel, rows, columns, groups, sharing = ss.subspec_fp8_linear_exact_plan(M, N, K)
    assert kernel in (1, 2) and rows in (32, 64) and groups >= 1 and sharing >= 1
    codes = M * K + 4 * M * ((K + 511) // 512)
    parts = ss.subspec_fp8_linear_exact_workspace_bytes(M, N, K, 1)
    assert (parts > 0) == (sharing > 1)
    assert ss.subspec_fp8_linear_exact_workspace_bytes(M, N, K, 0) >= codes + parts


@pytest.mark.parametrize("M,N,K", [(1, 3584, 3584), (16, 512, 18944), (40, 512, 512), (64, 37888, 3584)])
def test_up_to_64_rows_plans_are_the_same(M, N, K):
    assert ss.subspec_fp8_linear_exact_plan(M, N, K) == ss.subspec_fp8_linear_plan(M, N, K)
    for rows8 in (0, 1):
        assert ss.subspec_fp8_linear_exact_workspace_bytes(M, N, K, rows8) == ss.subspec_fp8_linear_workspace_bytes(M, N, K, rows8)


M, N, K = 70, 48, 640
TENSORS = dict(x=(U8, M * K), xs=(I32, 2 * M), w=(U8, N * K), ws=(I32, 2 * N), y=(BF, M * N))


def test_the_binding_checks_every_tensor(calls):  # noqa: F811
    def call(**changed):
        a = {n: changed.get(n, Fake(*spec)) for n, spec in TENSORS.items()}
        ss.subspec_fp8_linear_exact(a["x"], a["xs"], a["w"], a["ws"], M, N, K, a["y"])

    call()
    assert [name for name, _ in calls] == ["subspec_fp8_linear_exact"]
    for name, (dtype, n) in TENSORS.items():
        for bad in (Fake(dtype, n - 1), Fake(torch.float16, n)):
            with pytest.raises(ss.SubspecError, match="EINVAL"):
                call(**{name: bad})
    ss.subspec_fp8_linear_exact(Fake(BF, M * K), None, Fake(U8, N * K), Fake(I32, 2 * N), M, N, K, Fake(BF, M * N))
    assert len(calls) == 2
