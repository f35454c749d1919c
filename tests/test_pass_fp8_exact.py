"""The 8-bit product with exact products captured into a graph and replayed, with eager calls of both products
between the replays: codes, partial sums and counters share one workspace."""
import numpy as np
import pytest

import paper_2509_18344_amd as ss

from test_gpu_fp8 import _tiled_weight, weight
from test_gpu_rows import bf16, dev

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", [(113, 1952, 1152), (197, 18800, 1920), (333, 10880, 640)])  # parts of small and of large tiles, none
def test_captured_and_replayed(M, N, K):
    rng = np.random.default_rng([90, M, N, K])
    xs = [dev(bf16(rng.standard_normal((M, K)))) for _ in range(3)]
    t, ws = weight(*_tiled_weight(rng, N, K))
    ss.subspec_reserve(max(f(M, N, K, 0) for f in (ss.subspec_fp8_linear_exact_workspace_bytes, ss.subspec_fp8_linear_workspace_bytes)))
    y, z = (torch.empty((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    want = []
    for x in xs:
        ss.subspec_fp8_linear_exact(x, None, t, ws, M, N, K, y)
        want.append(y.clone())
    torch.cuda.synchronize()
    allocations = ss.subspec_workspace_info()["allocations"]
    x, g = torch.empty_like(xs[0]), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ss.subspec_fp8_linear_exact(x, None, t, ws, M, N, K, y)
    for k in (0, 1, 2, 0):
        x.copy_(xs[k])
        y.zero_()
        g.replay()
        ss.subspec_fp8_linear(xs[k], None, t, ws, M, N, K, z)
        torch.cuda.synchronize()
        assert torch.equal(y.view(torch.int16), want[k].view(torch.int16)), k
        ss.subspec_fp8_linear_exact(xs[k], None, t, ws, M, N, K, z)
        assert torch.equal(z.view(torch.int16), want[k].view(torch.int16)), k
    assert ss.subspec_workspace_info()["allocations"] == allocations
