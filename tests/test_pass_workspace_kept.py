"""Graphs of the caller's own over each kind of call alone: the workspace buffer that a call was
captured with stays allocated when a larger one replaces it and subspec_reserve frees what it may,
so that replays write no memory that belongs to others by then.  In a process of its own, whose
workspace starts empty and which no other test's captures have marked."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = """
import math, sys
sys.path[:0] = [{root!r}, {tests!r}]
import numpy as np, torch
import paper_2509_18344_amd as ss
from paper_2509_18344_amd import synth
from helpers import device_projection
from test_pass_together import Pass

D = "cuda"
rng = np.random.default_rng(5)
bf = lambda *s: torch.from_numpy(rng.standard_normal(s, dtype=np.float32)).to(torch.bfloat16).to(D)
empty = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device=D)


def linear():
    M, N, K = 40, 1024, 2048
    p = device_projection(torch.from_numpy(synth.weights_np(N, K, 9, 3, 128)).to(D), 3, 128)
    x, y, need = bf(M, K), empty(M, N), ss.subspec_qlinear_plan(M, N, K, 3, 128)["workspace_bytes"]
    call = lambda: ss.subspec_qlinear(x, p["qweight"], p["scales"], p["zeros"], 3, 128, M, N, K, y)
    return need, call, [y]


def stack():
    M, N, K = 40, 1024, 2048
    p = device_projection(torch.from_numpy(synth.weights_np(N, K, 9, 3, 128)).to(D), 3, 128)
    x, y, need = bf(M, K), empty(M, N), ss.subspec_qlinear_plan(M, N, K, 3, 128)["workspace_bytes"]
    one = [dict(x=x, qweight=p["qweight"], scales=p["scales"], zeros=p["zeros"], y=y, N=N, K=K)]
    return need, lambda: ss.subspec_stack_forward(one, 3, 128, M), [y]


def attention():
    M, Hq, Hkv, P, T = 6, 28, 4, 2048, 60
    S = P + T + M
    q, kc, vc, k, v, out = bf(M, Hq, 128), bf(S, Hkv, 128), bf(S, Hkv, 128), bf(M, Hkv, 128), bf(M, Hkv, 128), empty(M, Hq, 128)
    mask = torch.from_numpy(synth.tree_levels_mask(T, 6, M, 3).view(np.int32)).to(D)
    call = lambda: ss.subspec_tree_attention(q, kc, vc, k, v, mask, M, Hq, Hkv, S, P, T, 1 / math.sqrt(128), out)
    return ss.subspec_tree_attention_workspace_bytes(M, Hq, Hkv, P, T), call, [out]


def expand():
    R, V, k = 6, 152064, 6
    logits, logp = bf(R, V), torch.zeros(R, dtype=torch.float32, device=D)
    outs = [empty(k, dtype=torch.int32), empty(k, dtype=torch.int32), empty(k, dtype=torch.float32)]
    return ss.subspec_tree_workspace_bytes(R, V, k), lambda: ss.subspec_tree_expand(logits, logp, R, V, 0.2, k, *outs), outs


def draft():
    p = Pass(4)  # whose attention needs no workspace
    assert ss.subspec_tree_attention_kv4_workspace_bytes(6, 28, 4, 200, 18) == 0
    return p.workspace(), p.draft, p.outputs


def attention_kv4():
    M, Hq, Hkv, P = 1, 40, 8, 8191
    S = P + M
    kc, vc = (torch.zeros(ss.subspec_kv4_bytes(Hkv, S, 64), dtype=torch.uint8, device=D) for _ in range(2))
    ss.subspec_kv4_append(bf(S, Hkv, 128), bf(S, Hkv, 128), S, None, None, S, Hkv, S, 0, 64, kc, vc)
    q, mask, out = bf(M, Hq, 128), torch.ones((1, 1), dtype=torch.int32, device=D), empty(M, Hq, 128)
    call = lambda: ss.subspec_tree_attention_kv4(q, kc, vc, mask, M, Hq, Hkv, S, P, 0, 64, 0.088, out)
    return ss.subspec_tree_attention_kv4_workspace_bytes(M, Hq, Hkv, P, 0), call, [out]


def info():
    return ss.subspec_workspace_info()


for make in (linear, stack, attention, expand, draft, attention_kv4):
    need, call, outs = make()
    assert need > 0
    ss.subspec_reserve(max(need, info()["bytes"] + 1))  # a buffer that no graph holds
    ss.subspec_reserve(1)
    held, size = info()["retired"], info()["bytes"]
    call()
    torch.cuda.synchronize()
    expect = [t.clone() for t in outs]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call()
    ss.subspec_reserve(size + 1)
    ss.subspec_reserve(1)
    assert info()["bytes"] > size and info()["retired"] == held + 1, (make.__name__, held, info())
    junk = torch.full((size,), 0xFF, dtype=torch.uint8, device=D)  # whoever frees, reuses
    for rep in range(3):
        for t in outs:
            if make is not draft:
                t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip(outs, expect):
            assert torch.equal(got.view(torch.uint8), ref.view(torch.uint8)), (make.__name__, rep)
        assert bool((junk == 0xFF).all())
        call()  # on the larger buffer
        torch.cuda.synchronize()
    print(make.__name__, "kept", flush=True)

# the library's own graphs keep theirs only as long as they live
M, N, K = 40, 1024, 2048
need, call, outs = linear()
p = device_projection(torch.from_numpy(synth.weights_np(N, K, 9, 3, 128)).to(D), 3, 128)
x, y = bf(M, K), empty(M, N)
ss.subspec_reserve(info()["bytes"] + 1)
ss.subspec_reserve(1)
held, size = info()["retired"], info()["bytes"]
side = torch.cuda.Stream()
with torch.cuda.stream(side):
    g = ss.subspec_stack_capture([dict(x=x, qweight=p["qweight"], scales=p["scales"], zeros=p["zeros"], y=y, N=N, K=K)], 3, 128, M, side)
ss.subspec_reserve(size + 1)
assert info()["retired"] == held + 1
ss.subspec_graph_destroy(g)
assert info()["retired"] == held
print("done", info()["bytes"])
"""


def test_a_callers_graph_keeps_its_buffer_whatever_call_it_holds():
    script = SCRIPT.format(root=ROOT, tests=os.path.join(ROOT, "tests"))
    r = subprocess.run([sys.executable, "-c", script], cwd=ROOT, capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "done" in r.stdout, (r.stdout[-500:], r.stderr[-2000:])
