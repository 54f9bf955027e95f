"""The autograd forms of the selective layer and of the token probabilities on the CPU, with the library's calls replaced: nothing is
kept for a backward that cannot come, gradients come once, and a second derivative raises instead of being left out."""
import pytest
import torch

from paper_2607_05583_amd import ops


@pytest.fixture
def kept(monkeypatch):
    """What each scan or product was asked to keep; the calls compute something of the right shape that no graph sees."""
    log = []

    @torch.no_grad()
    def linear_fwd(x, W, bias=None, act="none", residual=None, save=False):
        log.append(save)
        y = x @ W
        return (y, ops.LinearSaved(y, bias)) if save else y

    @torch.no_grad()
    def linear_bwd(x, W, dy, pre=None, act="none", residual=None, want_dx=True, want_dw=True, want_db=False):
        return dict(dx=dy @ W.t(), dW=x.flatten(0, -2).t() @ dy.flatten(0, -2), db=dy.flatten(0, -2).sum(0))

    @torch.no_grad()
    def conv_fwd(x, w, bias=None, act="silu", state=None, lengths=None, return_state=False):
        return x * w[:, 0], x[:, -1:].clone()

    @torch.no_grad()
    def conv_bwd(x, w, dy, bias=None, act="silu", state=None, lengths=None, dstate_out=None, want_dstate=False, out=None):
        dx = dy * w[:, 0]
        if out is not None:
            out.copy_(dx)
        return dict(dx=dx, dw=torch.zeros_like(w), dbias=dy.sum((0, 1)))

    @torch.no_grad()
    def scan_fwd(x, dt, b, c, gamma, dt_bias=None, skip=None, h0=None, lengths=None, return_state=False, save=False, ws=None):
        log.append(save)
        return (x * 2, x[:, -1].clone()) + ((x.clone(),) if save else ())

    @torch.no_grad()
    def scan_bwd(x, dt, b, c, gamma, dy, dt_bias=None, skip=None, h0=None, lengths=None, dh_out=None, carry=None, want_dh0=False, out=None, ws=None):
        g = dict(dx=dy * 2, ddt=torch.zeros_like(dt), db=torch.zeros_like(b), dc=torch.zeros_like(c), dgamma=torch.zeros_like(gamma),
                 ddt_bias=torch.zeros_like(gamma), dskip=torch.zeros_like(gamma))
        if out is not None:
            for o, k in zip(out, ("dx", "ddt", "db", "dc")):
                o.copy_(g[k])
        return g

    @torch.no_grad()
    def logprobs_fwd(logits, tokens, top=0, entropy=False, scale=1.0):
        log.append(logits.requires_grad)
        return ops.TokenLogprobs(logits.sum(-1), logits.sum(-1) if entropy else None, None, None, logits[..., :2].clone())

    @torch.no_grad()
    def logprobs_bwd(logits, tokens, saved, dlogp=None, dentropy=None, scale=1.0):
        return dlogp[..., None].expand_as(logits).clone()

    for name, f in dict(resonator_linear_fwd=linear_fwd, resonator_linear_bwd=linear_bwd, resonator_short_conv_fwd=conv_fwd,
                        resonator_short_conv_bwd=conv_bwd, resonator_selective_scan_fwd=scan_fwd, resonator_selective_scan_bwd=scan_bwd,
                        resonator_token_logprobs_fwd=logprobs_fwd, resonator_token_logprobs_bwd=logprobs_bwd).items():
        monkeypatch.setattr(ops, name, f)
    return log


def leaf(*s, grad=True):
    return torch.randn(*s, dtype=torch.float64).requires_grad_(grad)


def params(grad=True):
    t = lambda *s: leaf(*s, grad=grad)  # noqa: E731
    return ops.SelectiveLayerParams(t(3, 10), t(10), t(8, 2), t(8), t(2), t(2), t(2), t(4, 3), t(3), t(3, 12), t(12), t(12, 3), t(3))


FORMS = {
    "conv": lambda g=True: (x := leaf(2, 4, 3, grad=g), ops.resonator_short_conv(x, leaf(3, 2, grad=g), leaf(3, grad=g))[0]),
    "scan": lambda g=True: (x := leaf(2, 4, 2, 3, grad=g), ops.resonator_selective_scan(
        x, leaf(2, 4, 2, grad=g), leaf(2, 4, 1, 3, grad=g), leaf(2, 4, 1, 3, grad=g), leaf(2, grad=g), leaf(2, grad=g), leaf(2, grad=g))[0]),
    "layer": lambda g=True: (x := leaf(2, 4, 3, grad=g), ops.resonator_selective_layer(x, params(g))[0]),
    "logprobs": lambda g=True: (x := leaf(4, 5, grad=g), ops.resonator_token_logprobs(x, torch.zeros(4, dtype=torch.int64))),
}


@pytest.mark.parametrize("form", FORMS)
def test_gradients_come_once(kept, form):
    x, y = FORMS[form]()
    assert y.requires_grad
    (g,) = torch.autograd.grad((y ** 2).sum(), x)
    assert g.shape == x.shape and g.any()


@pytest.mark.parametrize("form", FORMS)
def test_a_gradient_penalty_raises(kept, form):
    x, y = FORMS[form]()
    (g,) = torch.autograd.grad((y ** 2).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (y.sum() + (g ** 2).sum()).backward()


@pytest.mark.parametrize("form", ["scan", "layer"])
def test_nothing_is_kept_without_gradients(kept, form):
    with torch.no_grad():
        assert not FORMS[form]()[1].requires_grad
    assert kept and not any(kept)
    del kept[:]
    assert not FORMS[form](False)[1].requires_grad and kept and not any(kept)
    del kept[:]
    with torch.inference_mode():
        FORMS[form]()
    assert kept and not any(kept)
    del kept[:]
    assert FORMS[form]()[1].requires_grad and any(kept)


def test_columns_that_do_not_fit_are_refused(kept):
    p = params()
    with pytest.raises(ValueError, match="columns"):
        ops.resonator_selective_layer(leaf(2, 4, 3), p, groups=3)
