"""The short causal convolution on the GPU against its float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import select_oracle as O
from paper_2607_05583_amd import ops

from gpu_util import say
from select_util import DT, HALF, gpu, rounded, within

pytestmark = pytest.mark.gpu
ACTS = ["bf16", "f32"]


class Conv:
    def __init__(self, dt, B, L, D, K, act="silu", state=True, lengths=None, bias=True, seed=0):
        r = np.random.default_rng(seed)
        f = lambda v: np.float32(v).astype(np.float64)  # noqa: E731
        n = lambda *s: rounded(r.standard_normal(s), dt)  # noqa: E731
        self.dt, self.act, self.lengths = dt, act, lengths
        self.x, self.dy = n(B, L, D), n(B, L, D)
        self.w, self.bias = f(r.standard_normal((D, K))), f(r.standard_normal(D)) if bias else None
        self.state, self.dlast = (n(B, K - 1, D), n(B, K - 1, D)) if state else (None, None)
        self.y, self.last = O.conv_fwd(self.x, self.w, self.bias, act, self.state, lengths)
        self.g = dict(zip(("dx", "dw", "dbias", "dstate"), O.conv_bwd(self.x, self.w, self.dy, self.bias, act, self.state, lengths, self.dlast)))
        # a handful of float32 roundings of pre's terms, and the activation's own (exp and 1/x of the unit: some 2^-22 each);
        # every activation's derivative is at most 1.2, its second at most 1.1
        a = lambda v: None if v is None else np.abs(v)  # noqa: E731
        e, half = (K + 24) * 2.0 ** -22, HALF[dt]
        pre, _ = O.conv_fwd(a(self.x), a(self.w), a(self.bias), "none", a(self.state), lengths)
        gain = 1.2 + 1.1 * pre  # how a dpre moves with its pre's error
        up = O.conv_bwd(a(self.x), a(self.w), a(self.dy) * gain, a(self.bias), "none", a(self.state), lengths, a(self.dlast))
        self.bound = dict(y=half * np.abs(self.y) + 1.2 * e * pre)
        # dw and dbias: sums over up to 128 steps of a thread, then over blocks in 64 bits
        for k, v in zip(("dx", "dw", "dbias", "dstate"), up):
            self.bound[k] = (half * np.abs(self.g[k]) if k in ("dx", "dstate") else 0) + (e + (150 * 2.0 ** -24 if k in ("dw", "dbias") else 0)) * v

    def tensors(self, pad=0):
        x = gpu(self.x, self.dt)
        if self.lengths is not None:
            for r, n in enumerate(self.lengths):
                x[r, max(0, n):] = float("nan")
        if pad:
            x = torch.cat([x, torch.full((*x.shape[:2], pad), float("nan"), device="cuda", dtype=x.dtype)], -1)[..., :x.shape[-1]]
        return x, gpu(self.w), None if self.bias is None else gpu(self.bias)

    def more(self):
        return dict(act=self.act, state=None if self.state is None else gpu(self.state, self.dt),
                    lengths=None if self.lengths is None else torch.tensor(self.lengths, dtype=torch.int32, device="cuda"))

    def check(self, pad=0):
        x, w, bias = self.tensors(pad)
        y, last = ops.resonator_short_conv_fwd(x, w, bias, return_state=True, **self.more())
        within(y, self.y, self.bound["y"], "y")
        assert torch.equal(last, gpu(self.last, self.dt))
        if self.lengths is not None:
            for r, n in enumerate(self.lengths):
                assert not y[r, max(0, n):].any()
        g = ops.resonator_short_conv_bwd(x, w, gpu(self.dy, self.dt), bias, want_dstate=True,
                                         dstate_out=None if self.dlast is None else gpu(self.dlast, self.dt), **self.more())
        for k in g:
            within(g[k], self.g[k], self.bound[k], k)
        return y, last, g


# vectors that end inside, tiles of steps that end inside, steps fewer than taps, every constant number of taps and others
@pytest.mark.parametrize("dt", ACTS)
@pytest.mark.parametrize("sizes", [(1, 1, 1, 1), (2, 1, 5, 4), (1, 2, 8, 4), (2, 33, 16, 4), (3, 65, 17, 3), (1, 200, 130, 4), (2, 100, 64, 2),
                                   (1, 70, 40, 7), (2, 130, 9, 16), (1, 64, 3, 5), (2, 31, 12, 1), (9, 70, 24, 4), (1, 10, 6, 16)])
def test_forward_and_backward(sizes, dt):
    say(f"conv {dt} {sizes}")
    Conv(dt, *sizes, seed=sum(sizes)).check(pad=sum(sizes) % 4)


# calls that fill the chip, whose threads take more steps: forward 8, 32, 16 and 8 of them, backward 64, 32, 32 and 16
@pytest.mark.parametrize("dt", ACTS)
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("sizes", [(700, 150, 3, 16), (150, 700, 90, 4), (100, 700, 90, 3), (60, 700, 90, 2)])
def test_large_calls(sizes, ragged, dt):
    say(f"conv {dt} {sizes} ragged {ragged}")
    B, L = sizes[:2]
    lengths = [int(v) for v in np.random.default_rng(7).integers(0, L + 1, B)] if ragged else None
    Conv(dt, *sizes, lengths=lengths, seed=sum(sizes)).check(pad=2)


@pytest.mark.parametrize("dt", ACTS)
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu_tanh"])
def test_activations(act, dt):
    say(f"conv {dt} {act}")
    c = Conv(dt, 2, 50, 20, 4, act=act, seed=3)
    if act == "relu":  # (its derivative has a step at 0: no pre may lie within its own error of it)
        pre, _ = O.conv_fwd(c.x, c.w, c.bias, "none", c.state)
        assert np.abs(pre).min() > 1e-5
    c.check()


@pytest.mark.parametrize("dt", ACTS)
@pytest.mark.parametrize("K", [3, 4, 9])
@pytest.mark.parametrize("lengths", [[0, 1, 2, 70], [70, 64, 65, 3], [8, 0, 32, 33]])
def test_rows_of_unequal_length(lengths, K, dt):
    say(f"conv {dt} {K} {lengths}")
    Conv(dt, 4, 70, 18, K, lengths=lengths, seed=K).check(pad=2)
    Conv(dt, 4, 70, 18, K, lengths=lengths, seed=K, state=False, bias=False).check()


@pytest.mark.parametrize("dt", ACTS)
def test_no_steps(dt):
    say(f"conv {dt} no steps")
    c = Conv(dt, 2, 0, 6, 4, seed=1)
    y, last, g = c.check()
    assert torch.equal(last, gpu(c.state, dt)) and torch.equal(g["dstate"], gpu(c.dlast, dt)) and not g["dw"].any()


@pytest.mark.parametrize("dt", ACTS)
@pytest.mark.parametrize("K", [1, 2, 4, 11])
def test_step_is_the_convolution_of_one(K, dt):
    say(f"conv step {dt} {K}")
    c = Conv(dt, 3, 12, 21, K, seed=K)
    x, w, bias = c.tensors(3)
    state = gpu(c.state, dt)
    ys = []
    for t in range(12):
        new = torch.empty_like(state)
        y = ops.resonator_short_conv_step(x[:, t], w, state, bias, act=c.act, state_out=new)
        y2 = ops.resonator_short_conv_step(x[:, t], w, state, bias, act=c.act)  # in place
        assert torch.equal(y, y2) and torch.equal(new, state)
        ys.append(y)
    within(torch.stack(ys, 1), c.y, c.bound["y"], "y")
    assert torch.equal(state, gpu(c.last, dt))


@pytest.mark.parametrize("dt", ACTS)
@pytest.mark.parametrize("L", [1, 2, 40])
def test_state_in_place_and_gradient_as_columns(L, dt):
    say(f"conv {dt} in place, {L} steps")
    c = Conv(dt, 2, L, 10, 4, seed=4)
    x, w, bias = c.tensors(6)
    s = gpu(c.state, dt)
    y = ops.resonator_short_conv_fwd(x, w, bias, act=c.act, state=s, state_out=s)
    within(y, c.y, c.bound["y"], "y")
    assert torch.equal(s, gpu(c.last, dt))
    wide = torch.full((2, L, 15), 7.0, device="cuda", dtype=DT[dt])
    g = ops.resonator_short_conv_bwd(x, w, gpu(c.dy, dt), bias, act=c.act, state=gpu(c.state, dt), dstate_out=gpu(c.dlast, dt), out=wide[..., 2:12])
    within(g["dx"], c.g["dx"], c.bound["dx"], "dx")
    assert (wide[..., :2] == 7).all() and (wide[..., 12:] == 7).all()


def test_repeats_bit_for_bit_and_in_a_graph():
    say("conv in a graph")
    c = Conv("bf16", 3, 300, 72, 4, seed=5)
    x, w, bias = c.tensors()
    dy, m = gpu(c.dy, "bf16"), c.more()

    def step():
        y, last = ops.resonator_short_conv_fwd(x, w, bias, return_state=True, **m)
        g = ops.resonator_short_conv_bwd(x, w, dy, bias, want_dstate=True, **m)
        return [y, last, *g.values()]

    eager = step()
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


@pytest.mark.parametrize("dt", ACTS)
def test_autograd_is_the_backward(dt):
    say(f"conv autograd {dt}")
    c = Conv(dt, 2, 40, 12, 4, lengths=[40, 2], seed=6)
    leaves = [t.clone().requires_grad_() for t in (*c.tensors(), gpu(c.state, dt))]
    y, last = ops.resonator_short_conv(*leaves[:3], c.act, leaves[3], c.more()["lengths"])
    got = torch.autograd.grad((y, last), leaves, (gpu(c.dy, dt), gpu(c.dlast, dt)))
    g = c.check()[2]
    for k, v in zip(("dx", "dw", "dbias", "dstate"), got):
        assert torch.equal(g[k], v), k


def test_values_that_are_not_finite_reach_their_taps_only():
    say("conv NaN")
    c = Conv("f32", 1, 80, 6, 3, act="none", seed=7)
    x, w, bias = c.tensors()
    x[0, 31, 2], x[0, 50, 4] = float("nan"), float("inf")
    y = ops.resonator_short_conv_fwd(x, w, bias, act="none", state=gpu(c.state))
    bad = ~torch.isfinite(y)
    assert bad.sum() == 6 and bad[0, 31:34, 2].all() and bad[0, 50:53, 4].all()


def test_bad_arguments_are_refused():
    c = Conv("f32", 2, 10, 8, 4, seed=1)
    x, w, bias = c.tensors()
    f = ops.resonator_short_conv_fwd
    for bad in [(x[0], w, bias), (x, w[:5], bias), (x, w.double(), bias), (x, w, bias[:3]), (x.transpose(1, 2), w, bias), (x.half(), w, bias)]:
        with pytest.raises((ValueError, TypeError)):
            f(*bad)
    with pytest.raises(ValueError, match="act"):
        f(x, w, bias, act="tanh")
    with pytest.raises(ValueError):
        f(x, w, bias, state=gpu(c.state)[:, :2])
    with pytest.raises(Exception, match="overlap"):
        f(x, w, bias, out=x)
    with pytest.raises(Exception, match="range"):
        f(x, torch.zeros(8, 17, device="cuda"))
    with pytest.raises(Exception, match="workspace"):
        ops.resonator_short_conv_bwd(x, w, gpu(c.dy), bias, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
