"""The selective layer's operators with workspaces that the caller keeps."""
import pytest
import torch

from paper_2607_05583_amd import _lib, ops

from gpu_util import say

pytestmark = pytest.mark.gpu


def test_convolution_of_shorter_rows_in_the_longest_ones_workspace():
    say("conv, one workspace for rows of any length")
    B, D, K = 1, 640, 4
    ws = torch.full((_lib.lib().resonator_short_conv_workspace_bytes(B, 8192, D, K),), 255, dtype=torch.uint8, device="cuda")
    r = torch.Generator(device="cuda").manual_seed(0)
    n = lambda *s, dtype=torch.float32: torch.randn(s, generator=r, device="cuda").to(dtype)  # noqa: E731
    w, bias = n(D, K), n(D)
    for L in (8192, 6528, 4097, 300, 1):
        x, dy = n(B, L, D, dtype=torch.bfloat16), n(B, L, D, dtype=torch.bfloat16)
        a, b = (ops.resonator_short_conv_bwd(x, w, dy, bias, ws=v) for v in (ws, None))
        assert all(torch.equal(a[k], b[k]) for k in b), L
