"""What the gated recurrent layer's calls write into a caller's tensors counts as a change for autograd: a graph that kept the old
values raises when its backward comes, as after any operation in place."""
import pytest
import torch

from gpu_util import say

pytestmark = pytest.mark.gpu

ops = None


class _Off:
    """Stands in for the native module: takes nothing, so the Python code runs."""

    def __getattr__(self, name):
        return lambda *a: None


def setup_module(module):
    global ops
    from paper_2607_05583_amd import ops as _ops
    ops = _ops


@pytest.fixture(params=["native", "python"])
def path(request, monkeypatch):
    monkeypatch.setattr(ops, "_NATIVE", ops._native() if request.param == "native" else _Off())
    return request.param


def t(*s, dtype=torch.float32):
    return torch.randn(*s, device="cuda").to(dtype)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_step_between_forward_and_backward_raises(path, bits, dtype):
    """Two losses of one graph, and a step after the first: the second's gradient would be of the new weights."""
    say(f"step and backward {path} {bits} {dtype}")
    W = t(64, 32, dtype=dtype).requires_grad_()
    st = ops.adamw_state([W], bits=bits)
    y = ops.resonator_linear(t(8, 64, dtype=dtype), W, act="gelu_tanh")
    y.sum().backward(retain_graph=True)
    ops.resonator_adamw_step([W.detach()], [W.grad], st, step=1, lr=0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def versions(*tensors):
    return [v._version for v in tensors]


@pytest.mark.parametrize("bits", [8, 32])
def test_step_counts_for_what_it_writes(path, bits):
    say(f"versions of a step {path} {bits}")
    p, g = [t(300, dtype=torch.bfloat16), t(5, dtype=torch.bfloat16)], [t(300), t(5)]
    st = ops.adamw_state(p, bits=bits)
    every = [*p, *st.values()]
    was, was_g = versions(*every), versions(*g)
    ops.resonator_adamw_step(p, g, st, step=1, lr=0.1)
    assert versions(*every) == [v + 1 for v in was] and versions(*g) == was_g
    new, new_st = [v.clone() for v in p], {k: v.clone() for k, v in st.items()}
    was, was_new = versions(*every), versions(*new, *new_st.values())
    ops.resonator_adamw_step(p, g, st, step=2, lr=0.1, out=(new, new_st))
    assert versions(*every) == was and versions(*new, *new_st.values()) == [v + 1 for v in was_new]


def test_scan_and_product_count_for_what_they_write(path):
    say(f"versions of scan and product {path}")
    x, r, i, gamma = t(2, 40, 16), t(2, 40, 16), t(2, 40, 16), torch.rand(16, device="cuda")
    h, y, dx = t(2, 16), t(2, 40, 16), [t(2, 40, 16) for _ in range(3)]
    ins = x, r, i, gamma
    was = versions(*ins, h)
    _, carry = ops.resonator_gated_scan_fwd(*ins, h0=h, save=True)
    assert versions(*ins, h) == was
    v = versions(h, y)
    ops.resonator_gated_scan_fwd(*ins, h0=h, out=y, h_out=h)
    assert versions(h, y) == [k + 1 for k in v]
    v = versions(*dx)
    ops.resonator_gated_scan_bwd(*ins, y, carry=carry, out=dx)
    assert versions(*dx) == [k + 1 for k in v]
    tok, out = t(2, 16), t(2, 16)
    v = versions(h, out)
    ops.resonator_gated_scan_step(tok, tok.clone(), tok.clone(), gamma, h, out=out)
    assert versions(h, out) == [k + 1 for k in v]
    h2 = t(2, 16)
    v = versions(h, h2)
    ops.resonator_gated_scan_step(tok, tok.clone(), tok.clone(), gamma, h, h_out=h2)
    assert versions(h, h2) == [v[0], v[1] + 1]
    v = versions(out)
    ops.resonator_linear_fwd(tok, t(16, 16), residual=out, out=out)
    assert versions(out) == [v[0] + 1]
    assert versions(*ins) == was[:4]


def test_tensors_of_inference_mode(path):
    """They have no versions, and are taken as before."""
    say(f"inference mode {path}")
    with torch.inference_mode():
        p, g, h, x = [t(40)], [t(40)], t(2, 16), t(2, 16)
        st = ops.adamw_state(p)
        ops.resonator_adamw_step(p, g, st, step=1, lr=0.1)
        ops.resonator_gated_scan_step(x, x.clone(), x.clone(), x[0].abs().clone(), h)
    ops.resonator_adamw_step(p, g, st, step=2, lr=0.1)
    ops.resonator_gated_scan_step(x, x.clone(), x.clone(), x[0].abs().clone(), h)
    assert torch.isfinite(p[0]).all() and torch.isfinite(h).all()
