"""What the 8-bit product's large tiles ask of the workspace: a place for every tile's sums that one of
its workgroups writes, and none that no workgroup does."""
import pytest

import paper_2509_18344_amd as ss

CUS = 256
COUNTERS = 65536


def _sharers(left, KB):
    """Workgroups of each way to share the left tiles."""
    return {min(CUS // left * left, left * KB), min(CUS, left * KB)}


@pytest.mark.parametrize("M,N,K", [(1000, 37888, 3584), (18, 16448, 4864), (34, 19536, 7808), (144, 18000, 5248), (1233, 14800, 6016),
                                   (516, 26448, 2560), (1175, 15008, 6016), (2048, 5120, 27648)])
def test_places_of_the_large_tiles_sums(M, N, K):
    kernel, rows, columns, groups, sharing = ss.subspec_fp8_linear_plan(M, N, K)
    assert kernel == 2
    got = ss.subspec_fp8_linear_workspace_bytes(M, N, K, 1)
    if sharing == 1:
        assert got == 0
        return
    left = -(-M // rows) * -(-N // columns) % CUS
    # a workgroup's run lies in one tile where every tile has as many workgroups, else it may end in a second
    allowed = {COUNTERS + s * (1 if s % left == 0 else 2) * rows * columns * 4 for s in _sharers(left, K // 128) if s > left}
    assert got in allowed, (got, allowed)
    # bf16 rows: their codes and scales too, in whole 256 bytes
    codes = M * K + 4 * M * ((K + 511) // 512)
    assert ss.subspec_fp8_linear_workspace_bytes(M, N, K, 0) - got == -(-codes // 256) * 256


def test_a_run_of_equal_ones_lies_in_one_tile():
    # the arithmetic behind it: worker w of c a tile has blocks floor(w left KB / (c left)) .. of tiles of KB
    for left in range(1, 129):
        for KB in (1, 2, 3, 7, 20, 28, 40, 216):
            s = min(CUS // left * left, left * KB)
            assert s % left == 0
            for w in range(s):
                a, b = w * left * KB // s, (w + 1) * left * KB // s
                assert a < b and a // KB == (b - 1) // KB == w // (s // left)
