"""prepare.fp8_weight on another stream while that stream is behind: temporary inputs, results dropped
early, and the null stream's handle.  The work ahead of it is ordinary products of a few milliseconds."""
import pytest

from paper_2509_18344_amd import prepare

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"
N, K = 2048, 4096


def _weight(seed, n=N):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn((n, K), generator=g, device=DEV).to(torch.bfloat16)


def _expect(w):
    p = prepare.fp8_weight(w)
    torch.cuda.synchronize()
    return p["w"].clone(), p["w_scales"].clone()


def _behind(a, times=40):
    """Work on the current stream; its last result."""
    for _ in range(times):
        b = torch.mm(a, a)
    return b


@pytest.mark.parametrize("given", ["stream", "handle"])
def test_a_temporary_weight_lives_until_the_stream_has_read_it(given):
    g, u = _weight(1, N // 2), _weight(2, N // 2)
    want = _expect(torch.cat([g, u]))
    a, s = torch.zeros((8192, 8192), dtype=torch.bfloat16, device=DEV), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        _behind(a)
    p = prepare.fp8_weight(torch.cat([g, u]), s if given == "stream" else s.cuda_stream)
    junk = [torch.full((N, K), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(8)]  # whoever frees, reuses
    torch.cuda.synchronize()
    assert torch.equal(p["w"], want[0]) and torch.equal(p["w_scales"], want[1]) and len(junk) == 8


def test_a_weight_dropped_early_writes_into_nobody():
    w = _weight(3)
    a, s = torch.zeros((8192, 8192), dtype=torch.bfloat16, device=DEV), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        _behind(a)
    p = prepare.fp8_weight(w, s)
    sizes = [(p[k].numel(), p[k].dtype) for k in ("w", "w_scales")]
    del p
    junk = [torch.full((n,), 77, dtype=t, device=DEV) for n, t in sizes for _ in range(4)]
    torch.cuda.synchronize()
    assert all(bool((j == 77).all()) for j in junk)


def test_the_null_streams_handle_waits_for_the_current_stream():
    w = _weight(4)
    want = _expect(w)
    a, s = torch.zeros((8192, 8192), dtype=torch.bfloat16, device=DEV), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        late = torch.zeros_like(w)
        _behind(a)
        late.copy_(w)
        p = prepare.fp8_weight(late, 0)
    torch.cuda.synchronize()
    assert torch.equal(p["w"], want[0]) and torch.equal(p["w_scales"], want[1])
