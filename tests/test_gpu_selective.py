"""The selective scan on the GPU against its float64 oracle."""
import numpy as np
import pytest
import torch

from paper_2607_05583_amd import ops

from gpu_util import say
from select_util import Scan, gpu, host, rounded, within

pytestmark = pytest.mark.gpu
ACTS = ["bf16", "f32"]
# one and odd sizes, chunks of 64 steps that end inside, several segments, padded states (16, 32, 64, 128), row blocks of 64
# (P over 64 has two), more heads in a group than a work-group of the backward takes
SIZES = [(1, 1, 1, 1, 1, 1), (2, 63, 2, 16, 1, 16), (1, 64, 3, 64, 1, 32), (2, 65, 4, 40, 2, 24), (1, 200, 4, 64, 2, 64),
         (2, 257, 2, 128, 1, 128), (1, 130, 11, 33, 1, 33), (3, 129, 2, 65, 2, 100), (1, 600, 18, 17, 2, 65), (1, 321, 9, 70, 1, 8)]


def check_forward(s, fused=False, **kw):
    y, h, carry = ops.resonator_selective_scan_fwd(*s.tensors(fused), return_state=True, save=True, **s.more(), **kw)
    within(y, s.y, s.bound["y"], "y")
    within(h, s.h, s.bound["h"], "h")
    return y, h, carry


def check_backward(s, fused=False, carry=None, **kw):
    g = ops.resonator_selective_scan_bwd(*s.tensors(fused), gpu(s.dy, s.act), dh_out=None if s.dh is None else gpu(s.dh),
                                         carry=carry, want_dh0=True, **s.more(), **kw)
    for k, b in s.bound.items():
        if k in g:
            within(g[k], s.grads[k], b, k)
    return g


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("sizes", SIZES)
def test_forward_and_backward(sizes, act):
    say(f"selective {act} {sizes}")
    s = Scan(act, *sizes, seed=sum(sizes))
    carry = check_forward(s)[2]
    check_backward(s, carry=carry)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("lengths", [[0, 1, 300], [64, 128, 5], [300, 65, 0]])
def test_rows_of_unequal_length(lengths, act):
    say(f"selective {act} lengths {lengths}")
    s = Scan(act, 3, 300, 3, 24, 1, 40, seed=sum(lengths), lengths=lengths)
    y, h, carry = check_forward(s, fused=True)
    for r, n in enumerate(lengths):
        assert not y[r, n:].any()
        if n == 0:
            assert torch.equal(h[r], gpu(s.h0)[r])
    g = check_backward(s, fused=True, carry=carry)
    for r, n in enumerate(lengths):
        for k in ("dx", "ddt", "db", "dc"):
            assert not g[k][r, n:].any()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("at,width", [(-40.0, 1.0), (60.0, 5.0), (0.0, 30.0), (4.0, 0.0)])
def test_steps_of_any_size(at, width, act):
    """Steps of next to nothing, steps that forget everything, both next to each other."""
    say(f"selective {act} steps at {at} +- {width}")
    s = Scan(act, 1, 150, 2, 16, 1, 16, seed=9, dt_at=at, dt_width=width)
    check_backward(s, carry=check_forward(s)[2])


@pytest.mark.parametrize("act", ACTS)
def test_without_anything_optional(act):
    s = Scan(act, 2, 270, 2, 20, 1, 20, seed=3, h0=False, bias=False, skip=False)
    say(f"selective {act} without options")
    y = ops.resonator_selective_scan_fwd(*s.tensors())
    within(y, s.y, s.bound["y"], "y")
    g = ops.resonator_selective_scan_bwd(*s.tensors(), gpu(s.dy, act))  # (the carry is made again)
    assert set(g) == {"dx", "ddt", "db", "dc", "dgamma", "ddt_bias", "dskip"}
    for k in g:
        within(g[k], s.grads[k], s.bound[k], k)


@pytest.mark.parametrize("act", ACTS)
def test_no_steps(act):
    say(f"selective {act} no steps")
    s = Scan(act, 2, 0, 2, 3, 1, 5, seed=1)
    y, h, carry = check_forward(s)
    assert torch.equal(h, gpu(s.h0))
    g = check_backward(s, carry=carry)
    assert torch.equal(g["dh0"], gpu(s.dh)) and not g["dgamma"].any() and not g["dskip"].any()


@pytest.mark.parametrize("act", ACTS)
def test_state_in_place_and_gradients_as_columns(act):
    say(f"selective {act} in place")
    B, L, H, P, G, N = sizes = (2, 140, 2, 24, 1, 16)
    s = Scan(act, *sizes, seed=5)
    a, m = s.tensors(True), s.more()
    h = m["h0"].clone()
    y = ops.resonator_selective_scan_fwd(*a, **{**m, "h0": h}, h_out=h)
    y1, h1 = ops.resonator_selective_scan_fwd(*a, **m, return_state=True)
    assert torch.equal(y, y1) and torch.equal(h, h1)
    cols = (H * P, G * N, G * N, H)
    du = torch.full((B, L, sum(cols) + 3), 7.0, device="cuda", dtype=a[0].dtype)
    dx, db, dc, dd, rest = du.split((*cols, 3), dim=-1)
    out = dx.unflatten(-1, (H, P)), dd, db.unflatten(-1, (G, N)), dc.unflatten(-1, (G, N))
    g = check_backward(s, True, out=out)
    g2 = check_backward(s, False)
    assert all(torch.equal(g[k], g2[k]) for k in g) and (rest == 7.0).all()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("sizes", [(1, 1, 1, 1, 1), (3, 2, 5, 1, 7), (2, 6, 64, 2, 64), (5, 4, 33, 4, 100), (2, 2, 128, 1, 128), (4, 3, 16, 1, 16)])
def test_step_is_the_scan_of_one(sizes, act):
    B, H, P, G, N = sizes
    say(f"selective step {act} {sizes}")
    s = Scan(act, B, 1, H, P, G, N, seed=sum(sizes))
    x, dt, b, c, gamma = s.tensors(True)
    m = s.more()
    h = m["h0"].clone()
    h2 = torch.empty_like(h)
    a = x[:, 0], dt[:, 0], b[:, 0], c[:, 0], gamma, h
    y = ops.resonator_selective_scan_step(*a, dt_bias=m["dt_bias"], skip=m["skip"], h_out=h2)
    assert torch.equal(h, m["h0"])
    y2 = ops.resonator_selective_scan_step(*a, dt_bias=m["dt_bias"], skip=m["skip"])
    assert torch.equal(y, y2) and torch.equal(h, h2)
    within(y, s.y[:, 0], s.bound["y"][:, 0], "y")
    within(h, s.h, s.bound["h"], "h")


def test_prompt_then_steps_is_the_whole():
    say("selective prompt then steps")
    s = Scan("f32", 2, 90, 2, 16, 1, 16, seed=8)
    x, dt, b, c, gamma = s.tensors()
    m = s.more()
    k = 70
    y, h = ops.resonator_selective_scan_fwd(*(v[:, :k].contiguous() for v in (x, dt, b, c)), gamma, **m, return_state=True)
    ys = [y]
    for t in range(k, 90):
        ys.append(ops.resonator_selective_scan_step(x[:, t], dt[:, t], b[:, t], c[:, t], gamma, h, m["dt_bias"], m["skip"])[:, None])
    within(torch.cat(ys, 1), s.y, s.bound["y"], "y")
    within(h, s.h, s.bound["h"], "h")


def test_calls_repeat_bit_for_bit_whatever_the_workspace_holds():
    say("selective repeats")
    sizes = (2, 500, 9, 24, 1, 24)
    s = Scan("bf16", *sizes, seed=2)
    a, m = s.tensors(), s.more()
    dy = gpu(s.dy, "bf16")
    first = None
    for fill in (0, 255, 17):
        ws = ops.selective_scan_workspace(torch.bfloat16, *sizes, "cuda").fill_(fill)
        y, h, carry = ops.resonator_selective_scan_fwd(*a, **m, return_state=True, save=True, ws=ws)
        ws.fill_(fill)
        g = ops.resonator_selective_scan_bwd(*a, dy, **m, dh_out=gpu(s.dh), carry=carry, want_dh0=True, ws=ws)
        now = [y, h, *g.values()]
        first = first or now
        assert all(torch.equal(p, q) for p, q in zip(first, now))


def test_graph_replays_with_eager_calls_between():
    say("selective in a graph")
    sizes = (2, 300, 4, 32, 1, 32)
    s = Scan("bf16", *sizes, seed=4)
    a, m = s.tensors(), s.more()
    dy, dh = gpu(s.dy, "bf16"), gpu(s.dh)
    ws = ops.selective_scan_workspace(torch.bfloat16, *sizes, "cuda")

    def step():
        y, h, carry = ops.resonator_selective_scan_fwd(*a, **m, return_state=True, save=True, ws=ws)
        g = ops.resonator_selective_scan_bwd(*a, dy, **m, dh_out=dh, carry=carry, want_dh0=True, ws=ws)
        return [y, h, *g.values()]

    eager = [t.clone() for t in step()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for _ in range(3):
        for t in captured:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(eager, captured))
        assert all(torch.equal(p, q) for p, q in zip(eager, step()))


@pytest.mark.parametrize("act", ACTS)
def test_autograd_is_the_backward(act):
    say(f"selective autograd {act}")
    s = Scan(act, 2, 100, 2, 16, 1, 16, seed=6, lengths=[100, 37])
    m = s.more()
    leaves = [t.clone().requires_grad_() for t in (*s.tensors(), m["dt_bias"], m["skip"], m["h0"])]
    y, h = ops.resonator_selective_scan(*leaves, m["lengths"])
    dy, dh = gpu(s.dy, act), gpu(s.dh)
    got = torch.autograd.grad((y, h), leaves, (dy, dh))
    g = check_backward(s)
    for k, v in zip(("dx", "ddt", "db", "dc", "dgamma", "ddt_bias", "dskip", "dh0"), got):
        assert torch.equal(g[k], v), k
    with torch.no_grad():
        assert not ops.resonator_selective_scan(*leaves, m["lengths"])[0].requires_grad


def test_another_stream():
    say("selective on a stream")
    s = Scan("bf16", 2, 300, 2, 64, 1, 64, seed=7)
    a, m = s.tensors(), s.more()
    y0, h0 = ops.resonator_selective_scan_fwd(*a, **m, return_state=True)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        y, h = ops.resonator_selective_scan_fwd(*a, **m, return_state=True)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(y, y0) and torch.equal(h, h0)


def test_bad_arguments_are_refused():
    s = Scan("f32", 2, 10, 4, 8, 2, 8, seed=1)
    x, dt, b, c, gamma = s.tensors()
    f = ops.resonator_selective_scan_fwd
    for bad in [(x[0], dt, b, c, gamma), (x, dt[:, :5], b, c, gamma), (x, dt, b[:, :, :1], c, gamma), (x, dt, b, c.bfloat16(), gamma),
                (x, dt, b, c, gamma[:3]), (x, dt, b, c, gamma.double()), (x.transpose(2, 3), dt, b, c, gamma), (x, dt, b, c[0], gamma)]:
        with pytest.raises((ValueError, TypeError)):
            f(*bad)
    with pytest.raises((ValueError, TypeError)):
        f(x.half(), dt.half(), b.half(), c.half(), gamma)
    with pytest.raises(ValueError):
        f(x, dt, b, c, gamma, h0=gpu(np.zeros((2, 4, 8, 7))))
    with pytest.raises(ValueError):
        f(x, dt, b, c, gamma, lengths=torch.tensor([1, 2], device="cuda"))
    with pytest.raises(Exception, match="overlap"):
        f(x, dt, b, c, gamma, out=x)
    b3 = gpu(np.zeros((2, 10, 3, 8)))
    with pytest.raises(Exception, match="G divide H"):
        f(x, dt, b3, b3, gamma)
    with pytest.raises(Exception, match="workspace"):
        f(*(torch.zeros(2, 4096, *t.shape[2:], device="cuda") for t in (x, dt, b, c)), gamma, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    big = gpu(np.zeros((1, 2, 1, 129)))
    with pytest.raises(Exception, match="range"):
        f(big, gpu(np.zeros((1, 2, 1))), gpu(np.zeros((1, 2, 1, 4))), gpu(np.zeros((1, 2, 1, 4))), gpu(np.zeros(1)))


def test_a_value_that_is_not_finite_stays_in_its_row_and_behind():
    say("selective NaN")
    s = Scan("bf16", 2, 200, 2, 16, 1, 16, seed=11)
    x, dt, b, c, gamma = s.tensors()
    x[0, 100, 1, 3] = float("nan")
    y, h = ops.resonator_selective_scan_fwd(x, dt, b, c, gamma, **s.more(), return_state=True)
    bad = ~torch.isfinite(y)
    assert bad[0, 100, 1, 3] and bad[0, 128:, 1, 3].all() and not torch.isfinite(h[0, 1, 3]).any()
    assert not bad[1].any() and not bad[0, :64].any() and not bad[0, :, 0].any()  # (its 64 steps may be hit)
