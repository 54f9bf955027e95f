"""The autograd forms without gradients, on the CPU, with the library's calls replaced: nothing is kept for a backward that cannot
come (the scan's states, the products' pre), and with gradients it is."""
import pytest
import torch

from paper_2607_05583_amd import ops


@pytest.fixture
def kept(monkeypatch):
    """What each forward call was asked to keep."""
    log = []

    def linear_fwd(x, W, bias=None, act="none", residual=None, save=False):
        log.append(save)
        y = x.detach() @ W.detach()
        return (y, ops.LinearSaved(y, bias)) if save else y

    def scan_fwd(x, r, i, gamma, h0=None, lengths=None, return_state=False, save=False, ws=None):
        log.append(save)
        x = x.detach()
        return (x.clone(), x[:, -1].clone()) + ((x,) if save else ())

    monkeypatch.setattr(ops, "resonator_linear_fwd", linear_fwd)
    monkeypatch.setattr(ops, "resonator_gated_scan_fwd", scan_fwd)
    return log


def forms(grad):
    t = lambda *s: torch.randn(*s).requires_grad_(grad)  # noqa: E731
    p = ops.GatedLayerParams(t(3, 9), t(9), t(3), t(3, 3), t(3), t(3, 12), t(12), t(12, 3), t(3))
    return [lambda: ops.resonator_linear(t(4, 3), t(3, 5), t(5), "silu"), lambda: ops.resonator_gated_scan(*(t(2, 4, 3),) * 3, t(3))[0],
            lambda: ops.resonator_gated_layer(t(2, 4, 3), p)[0]]


@pytest.mark.parametrize("k", range(3))
def test_nothing_is_kept_without_gradients(kept, k):
    with torch.no_grad():
        out = forms(True)[k]()
    assert not out.requires_grad and kept and not any(kept)
    del kept[:]
    out = forms(False)[k]()
    assert not out.requires_grad and kept and not any(kept)
    del kept[:]
    with torch.inference_mode():
        forms(True)[k]()
    assert kept and not any(kept)


@pytest.mark.parametrize("k", range(3))
def test_with_gradients_it_is(kept, k):
    assert forms(True)[k]().requires_grad and any(kept)
