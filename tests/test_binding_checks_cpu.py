"""CPU checks of what the binding refuses before a kernel could read or write past a tensor: one that
is smaller than the call needs, and one of another type than the kernel takes it for.  Stand-ins for
device tensors, with addresses that no call may touch; both ways through the binding, the one with
torch's methods mapped over the tensors and the one that names the fault."""
import numpy as np
import pytest

import paper_2509_18344_amd as ss
from paper_2509_18344_amd import _binding

torch = pytest.importorskip("torch")
A = 4096


class Fake:
    """A contiguous tensor on the current device, by its word."""

    def __init__(self, dtype, n):
        self.dtype, self.n = dtype, n

    def get_device(self):
        return _binding._current_device(None)

    def is_contiguous(self):
        return True

    def numel(self):
        return self.n

    def data_ptr(self):
        return A


BF, I32, F32, F64, U8 = torch.bfloat16, torch.int32, torch.float32, torch.float64, torch.uint8
M, Hq, Hkv, LD, S, P, T, N, V = 3, 4, 2, 1032, 96, 40, 30, 6, 1024
CACHE = ss.subspec_kv4_bytes(Hkv, S, 64)


def _rope(a, **kw):
    return ss.subspec_qkv_rope(a["qkv"], LD, a["bias"], a["qw"], a["kw"], 1e-6, a["pos"], a["freq"], kw.get("rot", 96), 0, M, Hq, Hkv,
                               a["q"], a["k"], a["v"])


def _append(a, **kw):
    return ss.subspec_kv4_append(a["k"], a["v"], 8, a["rows"], a["count"], 5, Hkv, S, 7, kw.get("group", 64), a["kc"], a["vc"])


def _read(a):
    return ss.subspec_kv4_read(a["kc"], a["vc"], Hkv, S, 7, 5, 64, a["k"], a["v"])


def _attend(a):
    return ss.subspec_tree_attention_kv4(a["q"], a["kc"], a["vc"], a["mask"], M, Hq, Hkv, S, P, T, 64, 0.1, a["out"])


def _verify(a, **kw):
    return ss.subspec_tree_verify(a["logits"], a["parent"], a["token"], a["u"], N, V, kw.get("T", 0.6), a["path"], a["acc"], a["nxt"])


# every tensor of every call: its type and the elements the header gives it
CALLS = {
    "rope": (_rope, dict(qkv=(BF, 2 * LD + 8 * 128), bias=(BF, 8 * 128), qw=(BF, 128), kw=(BF, 128), pos=(I32, M), freq=(F64, 48),
                         q=(BF, M * Hq * 128), k=(BF, M * Hkv * 128), v=(BF, M * Hkv * 128))),
    "append": (_append, dict(k=(BF, 8 * Hkv * 128), v=(BF, 8 * Hkv * 128), rows=(I32, 5), count=(I32, 1), kc=(U8, CACHE), vc=(U8, CACHE))),
    "read": (_read, dict(kc=(U8, CACHE), vc=(U8, CACHE), k=(BF, 5 * Hkv * 128), v=(BF, 5 * Hkv * 128))),
    "attend": (_attend, dict(q=(BF, M * Hq * 128), kc=(U8, CACHE), vc=(U8, CACHE), mask=(I32, M * 2), out=(BF, M * Hq * 128))),
    "verify": (_verify, dict(logits=(BF, (N + 1) * V), parent=(I32, N), token=(I32, N), u=(F32, N + 1), path=(I32, N), acc=(I32, 1),
                             nxt=(I32, 1))),
}
EACH = [(call, name) for call in CALLS for name in CALLS[call][1]]
RAW = {BF: [torch.int16], I32: [], F32: [], F64: [], U8: [torch.int8]}
OTHER = {BF: [torch.float16, F32, U8], I32: [torch.int64, F32, torch.int16], F32: [F64, torch.float16, I32],
         F64: [F32, torch.int64], U8: [BF, I32, torch.float32]}


@pytest.fixture(params=["mapped", "named"])
def calls(request, monkeypatch):
    """The library's calls replaced by one that records them."""
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.append((name, args)) or 0

    monkeypatch.setattr(_binding, "load_library", lambda: Library())
    monkeypatch.setattr(_binding, "_current_device", lambda stream: 0)
    monkeypatch.setattr(_binding, "_stream", lambda stream: 0)
    mapped = request.param == "mapped"
    for name, value in dict(_torch=torch, _raw_stream=lambda dev: 0, _device=lambda: 0, _get_device=Fake.get_device if mapped else None,
                            _is_contiguous=Fake.is_contiguous, _data_ptr=Fake.data_ptr, _dtype=lambda t: t.dtype,
                            _numel=Fake.numel).items():
        monkeypatch.setattr(_binding, name, value, raising=False)
    if not mapped:
        monkeypatch.setattr(_binding, "_raw_stream", None)
    return seen


def _args(call, **changed):
    return {n: changed.get(n, Fake(*spec)) for n, spec in CALLS[call][1].items()}


@pytest.mark.parametrize("call", CALLS)
def test_tensors_of_exactly_the_size_needed_pass(calls, call):
    CALLS[call][0](_args(call))
    for name, (dtype, n) in CALLS[call][1].items():
        for raw in RAW[dtype]:
            CALLS[call][0](_args(call, **{name: Fake(raw, n + 1)}))
    assert len(calls) == 1 + sum(len(RAW[d]) for d, _ in CALLS[call][1].values())
    assert all(A in args for _, args in calls)


@pytest.mark.parametrize("call,name", EACH)
def test_a_tensor_with_an_element_too_few_is_refused(calls, call, name):
    dtype, n = CALLS[call][1][name]
    with pytest.raises(ss.SubspecError, match="needs %d" % n):
        CALLS[call][0](_args(call, **{name: Fake(dtype, n - 1)}))
    assert not calls


@pytest.mark.parametrize("call,name", EACH)
def test_a_tensor_of_another_type_is_refused(calls, call, name):
    dtype, n = CALLS[call][1][name]
    for other in OTHER[dtype]:
        with pytest.raises(ss.SubspecError, match="needs one of"):
            CALLS[call][0](_args(call, **{name: Fake(other, 8 * n)}))
    assert not calls


def test_missing_tensors_keep_the_checks_of_the_others(calls):
    none = dict(bias=None, qw=None, kw=None)
    _rope(_args("rope", **none))
    with pytest.raises(ss.SubspecError, match="needs 48"):
        _rope(_args("rope", **none, freq=Fake(F64, 47)))
    with pytest.raises(ss.SubspecError, match="int64"):
        _rope(_args("rope", **none, pos=Fake(torch.int64, M)))
    _append(_args("append", rows=None, count=None))
    with pytest.raises(ss.SubspecError, match="needs %d" % CACHE):
        _append(_args("append", rows=None, count=None, vc=Fake(U8, CACHE - 1)))
    assert [args[3] for name, args in calls if "append" in name] == [None]


def test_what_a_call_does_not_read_is_not_checked(calls):
    _rope(_args("rope", pos=Fake(torch.int64, 0), freq=Fake(F32, 0)), rot=0)
    _verify(_args("verify", u=Fake(F64, 0)), T=0.0)
    assert len(calls) == 2


def test_groups_of_128_need_the_smaller_cache(calls):
    n = Hkv * (S // 32) * 2176
    _append(_args("append", kc=Fake(U8, n), vc=Fake(U8, n)), group=128)
    with pytest.raises(ss.SubspecError, match="needs %d" % n):
        _append(_args("append", kc=Fake(U8, n - 1), vc=Fake(U8, n)), group=128)


def test_sizes_of_caches_agree_with_the_library():
    for Hkv_, S_, group in ((1, 32, 64), (1, 32, 128), (8, 131072, 64), (65535, 1 << 20, 128)):
        assert _binding._kv4_size(Hkv_, S_, group) == ss.subspec_kv4_bytes(Hkv_, S_, group)


def test_arrays_are_no_device_tensors(calls):
    with pytest.raises(TypeError):
        _append(_args("append", k=np.zeros(8 * Hkv * 128, np.int16)))


@pytest.mark.parametrize("call", CALLS)
def test_calls_without_any_tensor_reach_the_librarys_refusal(monkeypatch, call):
    # the mapped way is there from the first call on a device on
    for name, value in dict(_torch=torch, _get_device=Fake.get_device, _device=lambda: 0, _raw_stream=lambda dev: 0).items():
        monkeypatch.setattr(_binding, name, value)
    monkeypatch.setattr(_binding, "_current_device", lambda stream: 0)
    monkeypatch.setattr(_binding, "_stream", lambda stream: 0)
    with pytest.raises(ss.SubspecError, match="EINVAL.*null pointer"):
        CALLS[call][0](dict.fromkeys(CALLS[call][1]))
