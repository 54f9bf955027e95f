"""The short convolution's state, written over by the call that reads it, with every number of taps: whatever tiles the steps go in,
no tile may read what another one has overwritten."""
import pytest
import torch

from paper_2607_05583_amd import ops

from gpu_util import say
from select_util import gpu, within
from test_gpu_short_conv import Conv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("K", [5, 9, 10, 13, 16])
@pytest.mark.parametrize("sizes,lengths", [
    ((2, 9, 640), None), ((2, 17, 130), None), ((1, 300, 1283), None), ((3, 40, 640), [40, 9, 0]), ((4, 33, 515), [17, 33, 8, 2])])
def test_state_in_place(sizes, lengths, K, dt):
    """640 channels are more than a work-group's, so that a row's second tile is in another one than its first."""
    B, L, D = sizes
    say(f"conv in place {dt} {sizes} {K} taps {lengths}")
    c = Conv(dt, B, L, D, K, lengths=lengths, seed=K)
    x, w, bias = c.tensors(3)
    m = c.more()
    start = m.pop("state")
    apart = ops.resonator_short_conv_fwd(x, w, bias, state=start, **m)
    within(apart, c.y, c.bound["y"], "y")
    for _ in range(4):
        s = start.clone()
        y = ops.resonator_short_conv_fwd(x, w, bias, state=s, state_out=s, **m)
        assert torch.equal(y, apart) and torch.equal(s, gpu(c.last, dt))


@pytest.mark.parametrize("K", [4, 10, 16])
def test_prompt_in_pieces(K):
    """A prompt in pieces of any length, its state moved on in place, is the whole prompt bit for bit."""
    say(f"conv in pieces, {K} taps")
    c = Conv("bf16", 2, 200, 700, K, seed=20 + K)
    x, w, bias = c.tensors()
    s, at, ys = gpu(c.state, "bf16"), 0, []
    whole = ops.resonator_short_conv_fwd(x, w, bias, act=c.act, state=s.clone())
    for n in (1, 16, 9, 40, 64, 3, 67):
        ys.append(ops.resonator_short_conv_fwd(x[:, at:at + n], w, bias, act=c.act, state=s, state_out=s))
        at += n
    assert at == 200 and torch.equal(torch.cat(ys, 1), whole) and torch.equal(s, gpu(c.last, "bf16"))
