"""The largest scales of the token log probabilities, on the CPU: one whose product with log2 e is beyond float32 is refused."""
import pytest

from paper_2607_05583_amd import _lib as L

from test_select_abi import err, lp_bwd, lp_fwd


@pytest.mark.parametrize("call", [lp_fwd, lp_bwd])
@pytest.mark.parametrize("scale", [3.4e38, 2.5e38, 1.7015e38])
def test_refused(call, scale):
    assert call(scale=scale) == L.RES_ERR_INVALID_ARG and "scale" in err()


def test_largest_is_taken():
    """Without rows nothing is launched."""
    for scale in (2.0 ** 127, 2.0 ** -126):
        assert lp_fwd(R=0, x=None, tok=None, logp=None, ids=None, tlp=None, scale=scale) == L.RES_OK
        assert lp_bwd(R=0, x=None, tok=None, stats=None, dx=None, scale=scale) == L.RES_OK


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_largest_scale(dt):
    """All of the probability is the largest logits', in equal parts; no difference times the scale is beyond float32's 2^128 but as
    an infinite one, and the gradient is at most the scale."""
    import math

    import torch

    from paper_2607_05583_amd import ops
    from select_util import DT

    print(f"logprobs {dt}, the largest scale", flush=True)
    z = torch.zeros(3, 700, dtype=DT[dt], device="cuda")
    z[0, [5, 300, 699]], z[1, :], z[2, 17] = 1.0, -2.0, 8.0
    t = torch.tensor([300, 4, 3], device="cuda")
    scale = 2.0 ** 127
    r = ops.resonator_token_logprobs_fwd(z, t, top=3, entropy=True, scale=scale)
    near = lambda a, b: abs(a - b) <= 8 * 2.0 ** -24 * max(1.0, abs(b))  # noqa: E731  (a logarithm of the unit, and its terms' sum)
    for k, n in ((0, 3), (1, 700)):
        assert near(r.logp[k].item(), -math.log(n)) and near(r.entropy[k].item(), math.log(n))
    assert r.logp[2].item() == -math.inf and r.entropy[2].item() == 0
    assert r.top_ids.tolist() == [[5, 300, 699], [0, 1, 2], [17, 0, 1]] and r.top_logp[2].tolist() == [0, -math.inf, -math.inf]
    g = ops.resonator_token_logprobs_bwd(z, t, r, torch.ones(3, device="cuda"), scale=scale).double()
    want = torch.zeros(3, 700, dtype=torch.float64, device="cuda")
    want[0, [5, 699]], want[0, 300] = -scale / 3, scale * 2 / 3
    want[1], want[1, 4] = -scale / 700, scale * 699 / 700
    want[2, 17], want[2, 3] = -scale, scale
    # p is exp(log p), off by some roundings of log p (at most 6.6 here), below 2^-20 in all and scale times that in 1 - p; a rounding to
    # bf16 is off by 2^-8
    off = (2.0 ** -8 if dt == "bf16" else 0) + 2.0 ** -24 * 64
    assert ((g - want).abs() <= off * want.abs() + scale * 2.0 ** -20 * (want != 0)).all()
