"""The operators together, as a draft pass and the verification after it call them: a
substitute q|k|v projection, its preparation, the new rows into the 4-bit cache, the tree
attention over it, a substitute output projection as logits, the tree expansion; then the
verification of the drafted tokens and the accepted rows into the cache.  Eager, each step
against its oracle on the step's own inputs, and captured into a graph of the caller's,
replayed several times with eager work in between."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss
from paper_2509_18344_amd import synth
from helpers import bf16_to_f64, device_projection, run_qlinear

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"
Hq, Hkv, M, P, T, S, V, GROUP = 28, 4, 6, 200, 18, 256, 2048, 64
HEADS = Hq + 2 * Hkv


class Pass:
    """One layer's draft pass and a verification on fixed buffers."""

    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
        bf = lambda *s: torch.from_numpy(rng.standard_normal(s, dtype=np.float32)).to(torch.bfloat16).to(DEV)  # noqa: E731
        self.qkv_proj = device_projection(dev(synth.weights_np(HEADS * 128, 256, seed, 1, std=0.1)), 4, 64)
        self.out_proj = device_projection(dev(synth.weights_np(V, Hq * 128, seed, 2, std=0.1)), 4, 64)
        self.x, self.bias = bf(M, 256), bf(HEADS * 128)
        self.pos = dev(np.array([P + 3] * M, np.int32))
        self.freq = dev(np.array([1e6 ** (-i / 64) for i in range(64)]))
        self.mask_host = synth.tree_levels_mask(T, 6, M, seed)
        self.mask = dev(self.mask_host.view(np.int32))
        n = ss.subspec_kv4_bytes(Hkv, S, GROUP)
        self.kc, self.vc = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
        ss.subspec_kv4_append(bf(P + T, Hkv, 128), bf(P + T, Hkv, 128), P + T, None, None, P + T, Hkv, S, 0, GROUP, self.kc, self.vc)
        self.start = self.kc.clone(), self.vc.clone()
        # a verification of the T + M drafted tokens: the target's logits, keys and values of each
        N = self.N = T + M
        parent = np.full(N, -1, np.int32)
        for j in range(6, N):
            parent[j] = (j // 6 - 1) * 6 + rng.integers(0, 6)
        token = rng.choice(V, N, replace=False).astype(np.int32)
        logits = rng.standard_normal((N + 1, V), dtype=np.float32) * 2
        for j in range(N):
            logits[parent[j] + 1, token[j]] += 9.0
        self.tree = parent, token, rng.random(N + 1, dtype=np.float32)
        self.logits = torch.from_numpy(logits).to(torch.bfloat16).to(DEV)
        self.parent, self.token, self.u = (dev(a) for a in self.tree)
        self.tk, self.tv = bf(N, Hkv, 128), bf(N, Hkv, 128)
        e = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device=DEV)  # noqa: E731
        self.qkv, self.q, self.k, self.v, self.o = e(M, HEADS * 128), e(M, Hq, 128), e(M, Hkv, 128), e(M, Hkv, 128), e(M, Hq, 128)
        self.draft_logits, self.parent_logp = e(M, V), e(M, dtype=torch.float32)
        self.next_parent, self.next_token = e(6, dtype=torch.int32), e(6, dtype=torch.int32)
        self.next_score = e(6, dtype=torch.float32)
        self.path, self.accepted, self.bonus = e(N, dtype=torch.int32), e(1, dtype=torch.int32), e(1, dtype=torch.int32)
        self.outputs = [self.qkv, self.q, self.k, self.v, self.o, self.draft_logits, self.next_parent, self.next_token,
                        self.next_score, self.path, self.accepted, self.bonus, self.kc, self.vc]

    def workspace(self):
        return max(ss.subspec_qlinear_plan(M, HEADS * 128, 256, 4, 64)["workspace_bytes"],
                   ss.subspec_qlinear_plan(M, V, Hq * 128, 4, 64)["workspace_bytes"],
                   ss.subspec_tree_attention_kv4_workspace_bytes(M, Hq, Hkv, P, T), ss.subspec_tree_workspace_bytes(M, V, 6),
                   ss.subspec_tree_verify_workspace_bytes(self.N, V))

    def reset(self):
        for t in self.outputs:
            t.zero_()
        self.kc.copy_(self.start[0])
        self.vc.copy_(self.start[1])

    def _linear(self, p, x, y):
        ss.subspec_qlinear(x, p["qweight"], p["scales"], p["zeros"], 4, 64, M, p["N"], p["K"], y)

    def draft(self):
        self._linear(self.qkv_proj, self.x, self.qkv)
        ss.subspec_qkv_rope(self.qkv, HEADS * 128, self.bias, None, None, 1e-6, self.pos, self.freq, 128, False, M, Hq, Hkv,
                            self.q, self.k, self.v)
        ss.subspec_kv4_append(self.k, self.v, M, None, None, M, Hkv, S, P + T, GROUP, self.kc, self.vc)
        ss.subspec_tree_attention_kv4(self.q, self.kc, self.vc, self.mask, M, Hq, Hkv, S, P, T, GROUP, 1 / math.sqrt(128), self.o)
        self._linear(self.out_proj, self.o, self.draft_logits)
        ss.subspec_tree_expand(self.draft_logits, self.parent_logp, M, V, 0.2, 6, self.next_parent, self.next_token, self.next_score)

    def verify(self):
        ss.subspec_tree_verify(self.logits, self.parent, self.token, self.u, self.N, V, 0.6, self.path, self.accepted, self.bonus)
        ss.subspec_kv4_append(self.tk, self.tv, self.N, self.path, self.accepted, self.N, Hkv, S, P, GROUP, self.kc, self.vc)


def _bits(t):
    return t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def test_a_draft_pass_and_its_verification_match_the_oracles():
    p = Pass(1)
    p.draft()
    torch.cuda.synchronize()
    # q|k|v and its preparation
    y = run_qlinear(p.qkv_proj, p.x)
    assert torch.equal(y, p.qkv)
    q, k, v = oracle.qkv_rope(_bits(p.qkv), _bits(p.bias), None, None, 1e-6, p.pos.cpu().numpy(), p.freq.cpu().numpy(), 128,
                              False, Hq, Hkv)
    size = np.abs(bf16_to_f64(p.qkv)).max() + np.abs(bf16_to_f64(p.bias)).max()
    for got, ref in ((p.q, q), (p.k, k), (p.v, v)):
        assert np.all(np.abs(bf16_to_f64(got) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * size)
    # the cache: everything before the pass, and its own rows
    start = [t.cpu().numpy().reshape(Hkv, -1) for t in p.start]
    for got, was, rows, value in ((p.kc, start[0], p.k, False), (p.vc, start[1], p.v, True)):
        ref = was.copy()
        oracle.kv4_write(ref, range(P + T, P + T + M), *oracle.kv4_quantize(bf16_to_f64(rows), GROUP), GROUP, value)
        assert np.array_equal(got.cpu().numpy().reshape(Hkv, -1), ref)
    # attention over what the cache holds; bounds as in the attention's own tests, coarser
    K, W = (oracle.kv4_value(*oracle.kv4_read(c.cpu().numpy().reshape(Hkv, -1), GROUP, value))[:P + T + M]
            for c, value in ((p.kc, False), (p.vc, True)))
    ref, wabs = oracle.tree_attention_values(_bits(p.q), K, W, P, T, p.mask_host, 1 / math.sqrt(128))
    assert np.all(np.abs(bf16_to_f64(p.o) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -8 * (wabs + np.abs(W).max() * 2.0 ** -4))
    # the next leaves
    pi, tok, sc = oracle.tree_expand(_bits(p.draft_logits), np.zeros(M), 0.2, 6)
    assert np.all(np.abs(p.next_score.cpu().numpy() - sc) <= 2e-4 + 1e-6 * np.abs(sc))
    # verification, and the accepted tokens' rows over the tree's first positions
    before = [t.cpu().numpy().reshape(Hkv, -1).copy() for t in (p.kc, p.vc)]
    p.verify()
    torch.cuda.synchronize()
    path, nxt, margin = oracle.tree_verify(_bits(p.logits), *p.tree[:2], p.tree[2], float(np.float32(0.6)))
    assert margin > 2.0 ** -17 and 1 <= len(path) < T
    n = int(p.accepted.item())
    assert p.path.cpu().tolist() == path + [-1] * (p.N - len(path)) and n == len(path) and p.bonus.item() == nxt
    for got, was, rows, value in ((p.kc, before[0], p.tk, False), (p.vc, before[1], p.tv, True)):
        oracle.kv4_write(was, range(P, P + n), *oracle.kv4_quantize(bf16_to_f64(rows)[path], GROUP), GROUP, value)
        assert np.array_equal(got.cpu().numpy().reshape(Hkv, -1), was)


def test_captured_passes_replay_after_the_workspace_has_grown():
    """A graph of the caller's own over all calls: replays equal the eager pass, with eager work
    between them, and after a larger call has replaced the workspace buffer and
    subspec_reserve has freed what it may (the graph's buffer is not among it)."""
    p = Pass(2)
    ss.subspec_reserve(p.workspace())
    p.reset()
    p.draft()
    p.verify()
    torch.cuda.synchronize()
    expect = [t.clone() for t in p.outputs]
    p.reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        p.draft()
        p.verify()
    size = ss.subspec_workspace_info()["bytes"]
    for rep in range(4):
        if rep == 2:
            ss.subspec_reserve(2 * size + (1 << 20))
            ss.subspec_reserve(1)
            assert ss.subspec_workspace_info()["retired"] >= 1
            junk = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)  # whoever frees, reuses
        p.reset()
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip(p.outputs, expect):
            assert torch.equal(got.view(torch.uint8), ref.view(torch.uint8)), rep
        other = Pass(3)  # eager work of other sizes and values between the replays
        other.draft()
        other.verify()
        torch.cuda.synchronize()
    del junk


GROWTH = """
import torch, paper_2509_18344_amd as ss
big = 1 << 15
q = torch.zeros((1, 28, 128), dtype=torch.bfloat16, device="cuda")
kc, vc = (torch.zeros(ss.subspec_kv4_bytes(4, big, 64), dtype=torch.uint8, device="cuda") for _ in range(2))
mask, out = torch.ones((1, 1), dtype=torch.int32, device="cuda"), torch.empty_like(q)
torch.cuda.synchronize()
assert ss.subspec_tree_attention_kv4_workspace_bytes(1, 28, 4, big - 1, 0) > 0 == ss.subspec_workspace_info()["bytes"]
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
    try:
        ss.subspec_tree_attention_kv4(q, kc, vc, mask, 1, 28, 4, big, big - 1, 0, 64, 0.1, out)
    except ss.SubspecError as e:
        assert "ECAPTURE" in str(e), e
        print("refused")
"""


def test_workspace_growth_is_refused_during_capture():
    """In a process of its own, whose workspace no other test has grown."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", GROWTH], cwd=root, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "refused" in r.stdout, r.stderr[-2000:]
