"""CPU-only checks of the operators around the 4-bit cache: refusals before any GPU work,
sizes and launch shapes, and pins of their oracles."""
import itertools
import math

import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss

A = 4096  # an aligned address that no call may touch


def refused(kind):
    return pytest.raises(ss.SubspecError, match=kind)


# --- queries, keys and values ---------------------------------------------------------------

def _rope(**kw):
    a = dict(qkv=A, ld=36 * 128, bias=None, qw=None, kw=None, eps=1e-6, pos=A, freq=A, rot=128, il=0, M=1, Hq=28, Hkv=4,
             q=A, k=A, v=A)
    a.update(kw)
    return ss.subspec_qkv_rope(a["qkv"], a["ld"], a["bias"], a["qw"], a["kw"], a["eps"], a["pos"], a["freq"], a["rot"],
                               a["il"], a["M"], a["Hq"], a["Hkv"], a["q"], a["k"], a["v"], stream=0)


@pytest.mark.parametrize("kw,kind", [
    (dict(qkv=None), "EINVAL"), (dict(q=None), "EINVAL"), (dict(k=None), "EINVAL"), (dict(v=None), "EINVAL"),
    (dict(pos=None), "EINVAL"), (dict(freq=None), "EINVAL"), (dict(qkv=A + 8), "EINVAL"), (dict(bias=A + 2), "EINVAL"),
    (dict(qw=A + 4), "EINVAL"), (dict(v=A + 8), "EINVAL"), (dict(pos=A + 2), "EINVAL"), (dict(freq=A + 4), "EINVAL"),
    (dict(ld=36 * 128 - 8), "EINVAL"), (dict(ld=36 * 128 + 4), "EINVAL"), (dict(il=2), "EINVAL"),
    (dict(eps=-1.0), "EINVAL"), (dict(eps=math.nan), "EINVAL"), (dict(eps=math.inf), "EINVAL"),
    (dict(rot=8), "EUNSUPPORTED"), (dict(rot=144), "EUNSUPPORTED"), (dict(rot=-16), "EUNSUPPORTED"),
    (dict(M=0), "EUNSUPPORTED"), (dict(M=(1 << 20) + 1), "EUNSUPPORTED"), (dict(Hq=0), "EUNSUPPORTED"),
    (dict(Hkv=0), "EUNSUPPORTED"), (dict(Hq=65535), "EUNSUPPORTED"),
])
def test_qkv_rope_refusals(kw, kind):
    with refused(kind):
        _rope(**kw)


def test_rope_oracle_pins():
    rng = np.random.default_rng(0)
    x = rng.standard_normal(128)
    freq = [1e4 ** (-i / 64) for i in range(64)]
    assert np.array_equal(oracle.rope_head(x, None, 0.0, 0, freq, 128, False), x)
    # a rotation keeps every pair's length, and q.k depends on the distance of positions alone
    y = oracle.rope_head(x, None, 0.0, 77, freq, 128, False)
    assert np.allclose(y[:64] ** 2 + y[64:] ** 2, x[:64] ** 2 + x[64:] ** 2)
    z = rng.standard_normal(128)
    for il in (False, True):
        dots = [oracle.rope_head(x, None, 0.0, p + 5, freq, 128, il) @ oracle.rope_head(z, None, 0.0, p, freq, 128, il)
                for p in (0, 9, 1000)]
        assert np.allclose(dots, dots[0])
    # a quarter turn of the pair (0, 1) interleaved
    e = np.zeros(128)
    e[0] = 1.0
    assert np.allclose(oracle.rope_head(e, None, 0.0, 1, [math.pi / 2] + [0.0] * 63, 128, True)[:2], [0.0, 1.0])
    # complex form
    c = (x[:64] + 1j * x[64:]) * np.exp(1j * 77 * np.array(freq))
    assert np.allclose(y, np.concatenate([c.real, c.imag]))
    w = rng.standard_normal(128)
    assert np.allclose(oracle.rope_head(3 * x, w, 0.0, 0, freq, 0, False), x * w / math.sqrt((x * x).mean()))


# --- rows of the 4-bit cache -------------------------------------------------------------------

def _append(**kw):
    a = dict(k=A, v=A, src=8, rows=None, count=None, n=8, Hkv=4, S=64, pos=0, group=64, kc=A, vc=A)
    a.update(kw)
    return ss.subspec_kv4_append(a["k"], a["v"], a["src"], a["rows"], a["count"], a["n"], a["Hkv"], a["S"], a["pos"], a["group"],
                                 a["kc"], a["vc"], stream=0)


def _read(**kw):
    a = dict(kc=A, vc=A, Hkv=4, S=64, pos=0, n=8, group=64, k=A, v=A)
    a.update(kw)
    return ss.subspec_kv4_read(a["kc"], a["vc"], a["Hkv"], a["S"], a["pos"], a["n"], a["group"], a["k"], a["v"], stream=0)


SHARED = [(dict(group=32), "EUNSUPPORTED"), (dict(Hkv=0), "EUNSUPPORTED"), (dict(Hkv=65536), "EUNSUPPORTED"),
          (dict(S=0), "EUNSUPPORTED"), (dict(S=48), "EUNSUPPORTED"), (dict(S=(1 << 30) + 32), "EUNSUPPORTED"),
          (dict(pos=-1), "EUNSUPPORTED"), (dict(pos=57), "EUNSUPPORTED"), (dict(n=-1), "EUNSUPPORTED"),
          (dict(S=1 << 30, n=(1 << 28) + 1), "EUNSUPPORTED"), (dict(pos=2 ** 31 - 1), "EUNSUPPORTED"),
          (dict(k=None), "EINVAL"), (dict(v=None), "EINVAL"), (dict(kc=None), "EINVAL"), (dict(vc=None), "EINVAL"),
          (dict(k=A + 8), "EINVAL"), (dict(vc=A + 4), "EINVAL")]


@pytest.mark.parametrize("kw,kind", SHARED)
def test_kv4_rows_refusals(kw, kind):
    with refused(kind):
        _append(**kw)
    with refused(kind):
        _read(**kw)


def test_kv4_append_refusals_and_empty_calls():
    for kw in (dict(rows=A + 2), dict(count=A + 1), dict(src=7), dict(rows=A, src=-1)):
        with refused("EINVAL"):
            _append(**kw)
    assert _append(n=0) == 0 and _read(n=0) == 0 and _append(n=0, pos=64, src=0) == 0


def test_kv4_bytes():
    assert ss.subspec_kv4_bytes(1, 32, 128) == 2048 + 128
    assert ss.subspec_kv4_bytes(8, 131072, 64) == 8 * 4096 * 2304 == oracle.kv4_bytes(8, 131072, 64)
    for bad in [(0, 32, 64), (4, 16, 64), (4, 32, 32), (4, 33, 64), (65536, 32, 64)]:
        assert ss.subspec_kv4_bytes(*bad) == 0


def test_kv4_oracle_pins():
    # places: every nibble and every half of a tile exactly once
    from oracle.kv4 import kv4_places
    for group, value in itertools.product((64, 128), (False, True)):
        byte, bit, scale = kv4_places(64, group, value)
        tile = 2048 + 128 * (128 // group)
        spots = 2 * byte.astype(np.int64) + bit // 4
        assert np.unique(spots).size == 64 * 128 and set(np.unique(bit)) == {0, 4}
        assert (byte[:32] < 2048).all() and ((byte[32:] >= tile) & (byte[32:] < tile + 2048)).all()
        halves = np.concatenate([scale[:, ::group].ravel(), scale[:, ::group].ravel() + 16])
        assert np.unique(halves).size == 2 * 64 * (128 // group) and (halves % 2 == 0).all()
        assert halves[np.argsort(halves)][0] == 2048 and halves.max() == 2 * tile - 2
    # the stated examples: position 17, dimension 37 of a key: block 1, slice 16 * 0 + 1, word 1, code 5
    byte, bit, _ = kv4_places(32, 64, False)
    assert byte[17, 37] == 1024 + 16 * 1 + 4 + 16 // 8 + 8 // 8 and bit[17, 37] == 0
    byte, bit, scale = kv4_places(32, 64, True)
    # a value: half 0, lane 16 * 0 + 5, word 2, code 1 + 4
    assert byte[17, 37] == 16 * 5 + 4 * 2 + 16 // 8 + 8 // 8 and bit[17, 37] == 0
    assert scale[17, 37] == 2048 + 2 * 5 and scale[17, 64] == 2048 + 32 + 2 * 5
    # a row on the grid comes back as it is; the ends of a range are met
    x = 2.0 + 0.25 * (np.arange(128) % 16).astype(np.float32)
    c, s, m = oracle.kv4_quantize(x, 128)
    assert s[0] == 0.25 and m[0] == 2.0 and np.array_equal(oracle.kv4_value(c, s, m), x)
    rng = np.random.default_rng(1)
    x = rng.standard_normal((100, 128)).astype(np.float32)
    c, s, m = oracle.kv4_quantize(x, 64)
    err = np.abs(oracle.kv4_value(c, s, m) - x).reshape(100, 2, 64)
    assert (err <= s.astype(np.float64)[..., None] * 0.51 + 2e-3).all() and c.min() == 0 and c.max() == 15
    c, s, m = oracle.kv4_quantize(np.full((1, 128), -7.5, np.float32), 64)
    assert not c.any() and not s.any() and (m == -7.5).all()


# --- attention over it ------------------------------------------------------------------------------

def _attend(**kw):
    a = dict(q=A, kc=A, vc=A, mask=A, M=6, Hq=28, Hkv=4, S=2400, P=2048, T=282, group=64, scale=0.088, out=A)
    a.update(kw)
    return ss.subspec_tree_attention_kv4(a["q"], a["kc"], a["vc"], a["mask"], a["M"], a["Hq"], a["Hkv"], a["S"], a["P"], a["T"],
                                         a["group"], a["scale"], a["out"], stream=0)


@pytest.mark.parametrize("kw,kind", [
    (dict(q=None), "EINVAL"), (dict(kc=None), "EINVAL"), (dict(vc=None), "EINVAL"), (dict(mask=None), "EINVAL"),
    (dict(out=None), "EINVAL"), (dict(q=A + 8), "EINVAL"), (dict(kc=A + 8), "EINVAL"), (dict(mask=A + 2), "EINVAL"),
    (dict(out=A + 2), "EINVAL"), (dict(scale=math.inf), "EINVAL"), (dict(scale=math.nan), "EINVAL"),
    (dict(scale=3e38), "EINVAL"), (dict(S=2335), "EUNSUPPORTED"), (dict(S=2304), "EUNSUPPORTED"),
    (dict(group=32), "EUNSUPPORTED"), (dict(Hq=30), "EUNSUPPORTED"), (dict(Hkv=0), "EUNSUPPORTED"),
    (dict(M=0), "EUNSUPPORTED"), (dict(M=10), "EUNSUPPORTED"), (dict(P=-1), "EUNSUPPORTED"), (dict(T=-1), "EUNSUPPORTED"),
    (dict(M=64, Hq=4, T=1100, S=4096), "EUNSUPPORTED"),
])
def test_kv4_attention_refusals(kw, kind):
    with refused(kind):
        _attend(**kw)


def test_kv4_attention_plan():
    for M, Hq, Hkv, P, T in [(1, 1, 1, 0, 0), (6, 28, 4, 2048, 282), (6, 40, 8, 131072, 60), (16, 32, 8, 8191, 200),
                             (8, 16, 2, 33, 7), (1, 16, 16, 1000000, 0), (1, 65535, 65535, 100, 0), (1, 1, 1, 1 << 29, 0)]:
        s, t = ss.subspec_tree_attention_kv4_plan(M, Hq, Hkv, P, T)
        tiles = -(-(P + T + M) // 32)
        assert t >= 1 and 1 <= s <= 512 and (s - 1) * t < tiles <= s * t, (M, Hq, Hkv, P, T, s, t)
        pad = 16 * -(-(Hq // Hkv * M) // 16)
        expect = 0 if s == 1 else 65536 + Hkv * s * pad * (128 + 2) * 4
        assert ss.subspec_tree_attention_kv4_workspace_bytes(M, Hq, Hkv, P, T) == expect
    for M, Hq, Hkv, P, T in [(6, 30, 4, 10, 0), (0, 28, 4, 10, 0), (10, 28, 4, 10, 0), (6, 28, 4, -1, 0), (1, 65536, 65536, 9, 0)]:
        with refused("EUNSUPPORTED"):
            ss.subspec_tree_attention_kv4_plan(M, Hq, Hkv, P, T)
        assert ss.subspec_tree_attention_kv4_workspace_bytes(M, Hq, Hkv, P, T) == 0


def test_kv4_attention_oracle_agrees_with_the_bf16_caches():
    from paper_2509_18344_amd import synth
    M, Hq, Hkv, P, T = 3, 4, 2, 20, 9
    S = P + T + M
    x = synth.tree_attn_inputs(M, Hq, Hkv, 128, S, 3)
    mask = synth.tree_levels_mask(T, 3, M, 3)
    ref, kc, vc = oracle.tree_attention(x["q"], x["k_cache"], x["v_cache"], P, T, x["k_new"], x["v_new"], mask, 0.1)
    wabs = oracle.weighted_abs_v(x["q"], x["k_cache"], x["v_cache"], P, T, x["k_new"], x["v_new"], mask, 0.1)
    K, V = (oracle.bf16_bits_to_f64(c).transpose(1, 0, 2) for c in (kc, vc))
    out, w = oracle.tree_attention_values(x["q"], K, V, P, T, mask, 0.1)
    assert np.allclose(out, ref, rtol=0, atol=1e-13) and np.allclose(w, wabs, rtol=0, atol=1e-13)


# --- verification ------------------------------------------------------------------------------------

def _verify(**kw):
    a = dict(logits=A, parent=A, token=A, u=A, N=6, V=1024, T=0.6, path=A, acc=A, nxt=A)
    a.update(kw)
    return ss.subspec_tree_verify(a["logits"], a["parent"], a["token"], a["u"], a["N"], a["V"], a["T"], a["path"], a["acc"],
                                  a["nxt"], stream=0)


@pytest.mark.parametrize("kw,kind", [
    (dict(logits=None), "EINVAL"), (dict(parent=None), "EINVAL"), (dict(token=None), "EINVAL"), (dict(u=None), "EINVAL"),
    (dict(path=None), "EINVAL"), (dict(acc=None), "EINVAL"), (dict(nxt=None), "EINVAL"), (dict(logits=A + 8), "EINVAL"),
    (dict(parent=A + 2), "EINVAL"), (dict(u=A + 1), "EINVAL"), (dict(path=A + 2), "EINVAL"),
    (dict(T=-0.5), "EINVAL"), (dict(T=math.nan), "EINVAL"), (dict(T=math.inf), "EINVAL"), (dict(T=1e-39), "EINVAL"),
    (dict(N=-1), "EUNSUPPORTED"), (dict(N=1025), "EUNSUPPORTED"), (dict(V=0), "EUNSUPPORTED"), (dict(V=1020), "EUNSUPPORTED"),
    (dict(V=(1 << 20) + 8), "EUNSUPPORTED"),
])
def test_tree_verify_refusals(kw, kind):
    with refused(kind):
        _verify(**kw)


def test_tree_verify_workspace():
    for N, V in [(0, 8), (0, 1 << 20), (4, 32000), (288, 152064), (1024, 1 << 20)]:
        n = ss.subspec_tree_verify_workspace_bytes(N, V)
        assert 65536 + 16 + 8 * -(-V // 2048) + 8 * (N + 1) <= n < 65536 + 16 * 1024 + 8 * 4096 + 8 * 1024
    for N, V in [(-1, 8), (1025, 8), (4, 12), (4, 0), (4, (1 << 20) + 8)]:
        assert ss.subspec_tree_verify_workspace_bytes(N, V) == 0


def test_tree_verify_oracle_samples_the_target():
    """The law of (first token) over uniform numbers is the target's distribution, whatever was
    drafted; the law of the second one that of the row that follows it."""
    rng = np.random.default_rng(0)
    V = 8
    logits = oracle.bf16_round_bits(rng.standard_normal((3, V)).astype(np.float32))
    l = oracle.bf16_bits_to_f64(logits)
    p = np.exp(l - l.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    steps = 4000
    first = np.zeros(V)
    for u in (np.arange(steps) + 0.5) / steps:
        path, nxt, _ = oracle.tree_verify(logits, [-1, -1], [6, 2], [u, 0.3, 0.6], 1.0)
        assert path in ([], [0], [1])
        first[[6, 2][path[0]] if path else nxt] += 1
    assert np.abs(first / steps - p[0]).max() <= 2.0 / steps
    assert oracle.tree_verify(logits, [-1, 0], [6, 1], None, 0.0)[0] == ([0] if p[0].argmax() == 6 else [])


# --- the binding's own checks ----------------------------------------------------------------------------

def test_binding_refuses_tensors_that_a_kernel_cannot_read():
    torch = pytest.importorskip("torch")
    host = torch.zeros(1 << 16, dtype=torch.int16)
    with refused("EINVAL"):
        _rope(qkv=host)
    with refused("EINVAL"):
        _attend(q=host)
    with pytest.raises(TypeError):
        _append(k=np.zeros(1 << 16, np.int16))

    class Strided:  # on the right device by its word, but not whole
        def get_device(self):
            return -2

        def is_contiguous(self):
            return False

        def data_ptr(self):
            return A
    with refused("not contiguous"):
        _verify(logits=Strided())
    with refused("current device"):
        _verify(logits=torch.zeros(8))
