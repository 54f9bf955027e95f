"""The selective layer's operators with workspaces that the caller keeps."""
import pytest
import torch

from paper_2607_05583_amd import _lib, ops

from gpu_util import say
from select_util import DT, Scan, gpu, within

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


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("sizes", [(2, 300, 6, 40, 2, 50), (2, 300, 3, 64, 3, 64), (1, 200, 2, 128, 2, 128), (1, 130, 5, 20, 5, 100), (2, 300, 10, 16, 1, 40),
                                   (2, 300, 6, 40, 2, 24), (1, 200, 3, 64, 3, 32), (2, 130, 1, 100, 1, 1), (1, 70, 9, 30, 1, 16)])
def test_scan_of_few_heads_a_group_stays_in_its_workspace(sizes, act):
    """The backward with a workspace of just the bytes that it asks for: what lies around them is left alone."""
    say(f"scan backward {act} {sizes} in its own bytes")
    s = Scan(act, *sizes, seed=3)
    a, m, dy, dh = s.tensors(), s.more(), gpu(s.dy, act), gpu(s.dh)
    _, carry = ops.resonator_selective_scan_fwd(*a, **m, save=True)
    n = _lib.lib().resonator_selective_scan_workspace_bytes(1, ops._DT[DT[act]], *sizes)
    room = torch.full((n + 8192,), 0x5A, dtype=torch.uint8, device="cuda")
    g = ops.resonator_selective_scan_bwd(*a, dy, **m, dh_out=dh, carry=carry, want_dh0=True, ws=room[4096:4096 + n])
    assert (room[:4096] == 0x5A).all() and (room[4096 + n:] == 0x5A).all()
    for k, v in g.items():
        within(v, s.grads[k], s.bound[k], k)
