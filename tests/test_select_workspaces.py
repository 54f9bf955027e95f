"""Sizes of the workspaces of the selective layer's operators, on the CPU: what serves a call serves every smaller one where that is
promised, and none is larger than what its call keeps."""
import pytest

from paper_2607_05583_amd import _lib as L

LENGTHS = sorted({0, 1, 7, 8, 9, 63, 64, 65, 300, 777, 1024, 1025, 2001, 4096, 4097, 6464, 6528, 6529, 8192, 12000, 16384, 32768, 65536, 131072, 1 << 20})


def conv(B, T, D, K):
    return L.lib().resonator_short_conv_workspace_bytes(B, T, D, K)


@pytest.mark.parametrize("K", [1, 4, 16])
@pytest.mark.parametrize("D", [1, 64, 130, 640, 5000])
def test_conv_workspace_serves_smaller_calls(D, K):
    for B in (1, 2, 5, 64):
        sizes = [conv(B, T, D, K) for T in LENGTHS]
        assert sizes[0] > 0 and sizes == sorted(sizes), (B, D, K)
    for T in (1, 300, 6528, 8192):
        for wider in ([conv(B, T, D, K) for B in range(1, 200)], [conv(3, T, d, K) for d in range(D, D + 300)], [conv(3, T, D, k) for k in range(1, 17)]):
            assert wider == sorted(wider), (T, D, K)
