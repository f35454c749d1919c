"""The verification's 32-bit sums over long rows whose logits repeat, so that roundings add up instead
of averaging out: a uniform number 2^-18 of a drafted token's border away is decided rightly.

The bound, from the arithmetic: a term 2^(c (l - r)) is off by the rounding of c, twice, of its product and of
the exponential, (3 |x| ln 2 + 2) 2^-24 for an exponent x, of which those that weigh lie within
2^-24 .. 1 of the row's: below 2^-18.6 of the sum, and of a drafted token's share, of which the other part's
half counts at a border; sums of 8 such terms add 3 roundings, and those over the row and over its
drafted tokens run in 64 bits."""
import numpy as np
import pytest

import oracle
import paper_2509_18344_amd as ss
from test_gpu_verify import _bf16

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"


def _rows(kind, V):
    """Row 0 of the logits, in bf16."""
    i = np.arange(V)
    if kind == "flat":  # every thread's first load is large, all others the same
        x = np.where(i < 2048, 0.0, -1.5)
    elif kind == "rising":  # the maximum moves in most loads
        x = -4.0 + 4.0 * (i // 2048) / max(1, V // 2048)
    elif kind == "steps":  # it moves far, a few times
        x = -60.0 + 20.0 * np.minimum(i * 4 // V, 2) + np.where(i % 3 == 0, 0.3, 0.0)
    else:
        x = np.where(i % 2 == 0, 0.7, -0.4)
    return x.astype(np.float32)


@pytest.mark.parametrize("T", [1.0, 0.6, 8.0])
@pytest.mark.parametrize("kind", ["flat", "rising", "steps", "two"])
@pytest.mark.parametrize("N,V", [(700, 1 << 20), (640, 152064), (288, 152064), (300, 32000), (1024, 40960)])
def test_tree_verify_borders_on_long_rows_of_repeated_logits(N, V, kind, T):
    x = _rows(kind, V)
    x[V - 9] = T * np.log(np.exp((x.astype(np.float64) - x.max()) / T).sum()) + x.max()  # half of the row
    bits = _bf16(x)
    l = oracle.bf16_bits_to_f64(bits)
    p = np.exp((l - l.max()) / float(np.float32(T)))
    p /= p.sum()
    share = p[V - 9]
    assert 0.4 < share < 0.6
    logits = torch.zeros((N + 1, V), dtype=torch.int16, device=DEV)
    logits[0] = torch.from_numpy(bits.view(np.int16)).to(DEV)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    parent, token = torch.full((N,), -2, dtype=torch.int32, device=DEV), torch.zeros(N, dtype=torch.int32, device=DEV)
    parent[5], token[5] = -1, V - 9
    path, acc, nxt = torch.empty(N, dtype=torch.int32, device=DEV), i32(-9), i32(-9)
    for side in (-1, 1):
        u = np.float32(share * (1 + side * 2.0 ** -18))
        assert abs(float(u) / share - 1) > 2.0 ** -18.5 and (float(u) < share) == (side < 0)
        uniform = torch.full((N + 1,), float(u), dtype=torch.float32, device=DEV)
        ss.subspec_tree_verify(logits, parent, token, uniform, N, V, T, path, acc, nxt)
        assert acc.item() == (1 if side < 0 else 0), (side, acc.item(), nxt.item())


@pytest.mark.parametrize("top", [5.0, 5.875, 7.0])
def test_tree_verify_borders_between_many_equal_children(top):
    """The borders lie at multiples of one probability: a thousand sums of the same two numbers."""
    N, V, T = 1024, 152064, 1.0
    x = np.zeros(V, np.float32)
    token = np.arange(N, dtype=np.int32) * 148 + 3
    x[token] = top
    bits = _bf16(x)
    l = oracle.bf16_bits_to_f64(bits)
    p = np.exp(l - l.max())
    p /= p.sum()
    edge = np.cumsum(p[token])
    logits = torch.zeros((N + 1, V), dtype=torch.int16, device=DEV)
    logits[0] = torch.from_numpy(bits.view(np.int16)).to(DEV)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    parent, token = torch.full((N,), -1, dtype=torch.int32, device=DEV), torch.from_numpy(token).to(DEV)
    path, acc, nxt = torch.empty(N, dtype=torch.int32, device=DEV), i32(-9), i32(-9)
    for k in (10, 100, 300, 511, 700, 900, 1000, 1022):
        for side in (-1, 1):
            u = np.float32(edge[k] * (1 + side * 2.0 ** -18))
            assert (float(u) < edge[k]) == (side < 0) and abs(float(u) / edge[k] - 1) > 2.0 ** -18.5
            uniform = torch.full((N + 1,), float(u), dtype=torch.float32, device=DEV)
            ss.subspec_tree_verify(logits, parent, token, uniform, N, V, T, path, acc, nxt)
            assert path[0].item() == (k if side < 0 else k + 1), (k, side, path[0].item())
