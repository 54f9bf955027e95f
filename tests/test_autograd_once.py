"""The autograd forms on the CPU, with the library's calls replaced by products of the same interface: a second derivative, which
the library's backwards do not have, raises instead of being left out."""
import pytest
import torch

from paper_2607_05583_amd import ops


@pytest.fixture
def calls(monkeypatch):
    """Forward and backward calls that compute on the CPU what no graph sees, as the library's do."""
    @torch.no_grad()
    def linear_fwd(x, W, bias=None, act="none", residual=None, save=False):
        y = x @ W
        return (y, ops.LinearSaved(None, bias)) if save else y

    @torch.no_grad()
    def linear_bwd(x, W, dy, pre=None, act="none", residual=None, want_dx=True, want_dw=True, want_db=False):
        return dict(dx=dy @ W.t(), dW=x.t() @ dy)

    @torch.no_grad()
    def scan_fwd(x, r, i, gamma, h0=None, lengths=None, return_state=False, save=False):
        return x * r, x[:, -1].clone(), x.clone()

    @torch.no_grad()
    def scan_bwd(x, r, i, gamma, dy, lengths=None, dh_out=None, carry=None, want_dh0=False):
        return dict(dx=dy * r, dr=dy * x, di=torch.zeros_like(i), dgamma=torch.zeros_like(gamma))

    @torch.no_grad()
    def layer_fwd(x, p, h0=None, lengths=None, act="gelu_tanh", return_state=False, save=False):
        return x * p.gamma, x[:, -1].clone(), dict(u=x, y=x, carry=x, z=x, m=x, pre=ops.LinearSaved(None, p.b1))

    @torch.no_grad()
    def layer_bwd(x, p, dout, saved, lengths=None, dh=None, act="gelu_tanh", want_dh0=False):
        return dict(dx=dout * p.gamma, dp=ops.GatedLayerParams(*(torch.zeros_like(t) for t in p)))

    @torch.no_grad()
    def mix_fwd(x, gamma, omega, amp, phase):
        return x * 2

    @torch.no_grad()
    def mix_bwd(x, dy, gamma, omega, amp, phase):
        return dict(dx=dy * 2, dgamma=gamma * 0, domega=omega * 0, damp=amp * 0, dphase=phase * 0)

    @torch.no_grad()
    def map_fwd(tg, tw, alpha_min):
        return tg.exp(), tw * 2

    @torch.no_grad()
    def map_bwd(tg, tw, dg, dw):
        return dg * tg.exp(), dw * 2

    for name, f in dict(resonator_linear_fwd=linear_fwd, resonator_linear_bwd=linear_bwd, resonator_gated_scan_fwd=scan_fwd,
                        resonator_gated_scan_bwd=scan_bwd, resonator_gated_layer_fwd=layer_fwd, resonator_gated_layer_bwd=layer_bwd,
                        resonator_mix_fwd=mix_fwd, resonator_mix_bwd=mix_bwd, resonator_params_map=map_fwd,
                        resonator_params_map_bwd=map_bwd).items():
        monkeypatch.setattr(ops, name, f)


def leaf(*s):
    return torch.randn(*s, dtype=torch.float64).requires_grad_()


FORMS = {
    "linear": lambda: (x := leaf(4, 3), ops.resonator_linear(x, leaf(3, 5))),
    "scan": lambda: (x := leaf(2, 4, 3), ops.resonator_gated_scan(x, leaf(2, 4, 3), leaf(2, 4, 3), leaf(3))[0]),
    "layer": lambda: (x := leaf(2, 4, 3), ops.resonator_gated_layer(x, ops.GatedLayerParams(
        leaf(3, 9), leaf(9), leaf(3), leaf(3, 3), leaf(3), leaf(3, 12), leaf(12), leaf(12, 3), leaf(3)))[0]),
    "mix": lambda: (x := leaf(2, 4, 3), ops.resonator_mix(x, *(leaf(3, 2) for _ in range(4)))),
    "parameter map": lambda: (x := leaf(3, 2), ops.ResonatorParamMapFunction.apply(x, leaf(3, 2))[0]),
}


@pytest.mark.parametrize("form", FORMS)
def test_gradients_come_once(calls, form):
    x, y = FORMS[form]()
    (g,) = torch.autograd.grad((y ** 2).sum(), x)
    assert g.shape == x.shape and g.any()


@pytest.mark.parametrize("form", FORMS)
def test_a_gradient_penalty_raises(calls, form):
    """Its gradient would lack the penalty's term."""
    x, y = FORMS[form]()
    (g,) = torch.autograd.grad((y ** 2).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (y.sum() + (g ** 2).sum()).backward()
