"""The 8-bit product in graphs that the caller captures, on other streams and beside other calls that
use the workspace.  Such graphs keep their buffers until the process ends, so these tests come after those
that count the buffers kept, or run in a process of their own."""
import os
import subprocess
import sys

import numpy as np
import pytest

import paper_2509_18344_amd as ss

from test_gpu_fp8 import _layer, _mlp, _mlp_buffers, _random_rows, linear, weight
from test_gpu_rows import bf16, dev, host

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("M", [1, 13, 200])
def test_mlp_on_another_stream_captured_and_replayed(M):
    rng = np.random.default_rng([59, M])
    l = _layer(rng, 768, 640)
    xs = [bf16(rng.standard_normal((M, 768))) for _ in range(4)]
    res = bf16(4 * rng.standard_normal((M, 768)))
    out = _mlp_buffers(l, M)
    want = []
    for x in xs:
        want.append(host(_mlp(l, dev(x), dev(res), M, out)))
    s = torch.cuda.Stream()
    rd, xd = dev(res), dev(xs[1])
    s.wait_stream(torch.cuda.current_stream())
    y = _mlp(l, xd, rd, M, out, s)
    s.synchronize()
    assert np.array_equal(host(y), want[1])
    need = max(ss.subspec_fp8_linear_workspace_bytes(M, n, k, 1) for n, k in ((1280, 768), (768, 640)))
    ss.subspec_reserve(max(need, 1))
    allocations = ss.subspec_workspace_info()["allocations"]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _mlp(l, xd, rd, M, out)
    for x, w in zip(xs, want):
        xd.copy_(dev(x))
        rd.copy_(dev(res))
        out["y"].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(host(out["y"]), w)
        assert np.array_equal(host(_mlp(l, dev(x), dev(res), M, _mlp_buffers(l, M))), w)  # eager between replays
    assert ss.subspec_workspace_info()["allocations"] == allocations


def test_bf16_rows_captured_next_to_other_calls_that_use_the_workspace():
    from helpers import device_projection, run_qlinear
    rng = np.random.default_rng(60)
    M, N, K = 40, 512, 1024
    wc, wb = _random_rows(rng, N, K)
    t, ws = weight(wc, wb)
    x = dev(bf16(rng.standard_normal((M, K))))
    p = device_projection(torch.from_numpy(rng.standard_normal((512, 3584)).astype(np.float32)).to(DEV), 4, 64)
    xq = dev(bf16(rng.standard_normal((M, 3584))))
    q0, y0 = run_qlinear(p, xq), linear(x, None, t, ws, M, N, K)
    ss.subspec_reserve(max(ss.subspec_fp8_linear_workspace_bytes(M, N, K, 0), ss.subspec_qlinear_plan(M, 512, 3584, 4, 64)["workspace_bytes"]))
    y, g = torch.empty((M, N), dtype=torch.bfloat16, device=DEV), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ss.subspec_fp8_linear(x, None, t, ws, M, N, K, y)
    for _ in range(4):
        y.zero_()
        g.replay()
        q = run_qlinear(p, xq)
        torch.cuda.synchronize()
        assert torch.equal(y.view(torch.int16), y0.view(torch.int16)) and torch.equal(q.view(torch.int16), q0.view(torch.int16))
        assert torch.equal(linear(x, None, t, ws, M, N, K).view(torch.int16), y0.view(torch.int16))


SCRIPT = """
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import numpy as np, torch
import paper_2509_18344_amd as ss
from paper_2509_18344_amd import prepare

D, rng = "cuda", np.random.default_rng(5)
bf = lambda *s: torch.from_numpy(rng.standard_normal(s, dtype=np.float32)).to(torch.bfloat16).to(D)
info = ss.subspec_workspace_info


def few():  # parts of K, of few rows
    return 4, 512, 9216


def small():  # codes, and parts of a small tile
    return 200, 512, 4096


def large():  # codes, and parts of a large tile
    return 516, 26448, 2560


for make in (few, small, large):
    M, N, K = make()
    p = prepare.fp8_weight(bf(N, K))
    x, y = bf(M, K), torch.empty((M, N), dtype=torch.bfloat16, device=D)
    need = ss.subspec_fp8_linear_workspace_bytes(M, N, K, 0)
    call = lambda: ss.subspec_fp8_linear(x, None, p["w"], p["w_scales"], M, N, K, y)
    assert need > 0 and ss.subspec_fp8_linear_plan(M, N, K)[4] > 1, make.__name__
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    if make is few:  # nothing reserved yet: a capture that would have to allocate is refused, and goes on
        assert info()["bytes"] == 0
        side.wait_stream(torch.cuda.current_stream())
        refused = torch.cuda.CUDAGraph()
        with torch.cuda.graph(refused, stream=side):
            y.zero_()
            try:
                call()
                raise SystemExit("a call that allocates was captured")
            except ss.SubspecError as e:
                assert e.status == -4, e
        refused.replay()
    ss.subspec_reserve(max(need, info()["bytes"] + 1))  # a buffer that no graph holds
    ss.subspec_reserve(1)
    held, size = info()["retired"], info()["bytes"]
    call()
    torch.cuda.synchronize()
    expect = y.clone()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call()
    ss.subspec_reserve(size + 1)
    ss.subspec_reserve(1)
    assert info()["bytes"] > size and info()["retired"] == held + 1, (make.__name__, held, info())
    junk = torch.full((size,), 0xFF, dtype=torch.uint8, device=D)  # whoever frees, reuses
    for rep in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.view(torch.int16), expect.view(torch.int16)), (make.__name__, rep)
        assert bool((junk == 0xFF).all())
        call()  # on the larger buffer
        torch.cuda.synchronize()
        assert torch.equal(y.view(torch.int16), expect.view(torch.int16)), (make.__name__, rep)
    print(make.__name__, "kept", flush=True)
print("done")
"""


def test_a_callers_graph_keeps_its_buffer():
    script = SCRIPT.format(root=ROOT, tests=os.path.join(ROOT, "tests"))
    r = subprocess.run([sys.executable, "-c", script], cwd=ROOT, capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "done" in r.stdout, (r.stdout[-500:], r.stderr[-2000:])
