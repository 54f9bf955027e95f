"""The selective layer with a part of the state before the call, against the whole state whose other part is zeros."""
import pytest
import torch

from paper_2607_05583_amd import ops

from gpu_util import say
from test_gpu_selective_layer import problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("given", [(True, False), (False, True)])
def test_part_of_a_state(given, act):
    """What is not given is zero: the same bits forward, and the same gradients of all that is given."""
    say(f"selective layer, state {given} {act}")
    q = problem(act, 2, 70, 32, 4, 16, 2, 16, 4, 64, seed=5)
    parts = [t if g else None for t, g in zip(q["gstate"], given)]
    full = ops.SelectiveState(*(t if g else torch.zeros_like(t) for t, g in zip(q["gstate"], given)))
    out, last = ops.resonator_selective_layer(q["gx"], q["gp"], 2, state=ops.SelectiveState(*parts))
    for state in (parts, full):
        leaves = [None if t is None else t.clone().requires_grad_() for t in (q["gx"], *state, *q["gp"])]
        o, st = ops.resonator_selective_layer(leaves[0], ops.SelectiveLayerParams(*leaves[3:]), 2, state=ops.SelectiveState(*leaves[1:3]))
        assert torch.equal(o, out) and torch.equal(st.conv, last.conv) and torch.equal(st.h, last.h)
        kept = [0] + [1 + k for k in range(2) if given[k]] + list(range(3, len(leaves)))
        grads = torch.autograd.grad((o, *st), [leaves[k] for k in kept], (q["gdout"], *q["gdstate"]))
        if state is parts:
            first = grads
    assert all(torch.equal(a, b) for a, b in zip(first, grads))
