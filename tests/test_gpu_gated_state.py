"""The gated scan that advances its state in place (h_out is h0): a chain's last tile overwrites the state that its first tile
begins with, however many tiles lie between and however late one of them is.  What comes out is, bit for bit, what comes out
with a state of its own.
"""
import numpy as np
import pytest
import torch

from gpu_util import say

pytestmark = pytest.mark.gpu

ops = None
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def setup_module(module):
    global ops
    from paper_2607_05583_amd import ops as _ops
    ops = _ops


# chains of one tile of any size, of two (256 steps each), of three to eight (fewer than are looked back over), of nine and
# more; enough chains that a chain's tiles run beside each other, and few
@pytest.mark.parametrize("B,L,D", [(3, 31, 64), (3, 256, 40), (2, 257, 64), (2, 600, 64), (5, 1025, 72), (1, 2048, 64), (64, 2000, 256),
                                   (4, 2049, 64), (2, 9000, 200)])
@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_state_in_place(act, B, L, D):
    say(f"state in place {act} {B} {L} {D}")
    r = np.random.default_rng(L)
    t = lambda *s: torch.from_numpy(r.normal(size=s).astype(np.float32)).cuda()  # noqa: E731
    x, gates = t(B, L, D).to(DT[act]), t(B, L, 2 * D).to(DT[act]).split(D, dim=-1)
    # dampings so small that the first state is still felt in the last
    gamma = torch.linspace(1e-5, 2e-3, D, device="cuda")
    h0 = 10.0 * t(B, D)
    lengths = torch.from_numpy(r.integers(0, L + 1, B).astype(np.int32)).cuda()
    for n in (None, lengths):
        y, h, carry = ops.resonator_gated_scan_fwd(x, *gates, gamma, h0=h0, lengths=n, return_state=True, save=True)
        state = h0.clone()
        ws = ops.gated_scan_workspace(DT[act], B, L, D, "cuda")
        y2, h2, carry2 = ops.resonator_gated_scan_fwd(x, *gates, gamma, h0=state, lengths=n, return_state=True, save=True,
                                                      h_out=state, ws=ws)
        assert h2.data_ptr() == state.data_ptr()
        assert torch.equal(y, y2) and torch.equal(h, h2) and torch.equal(carry, carry2)
        assert ops.resonator_fwd_status(ws) == 0
