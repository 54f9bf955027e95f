"""GPU parity of the linear product with bias, activation and residual, and of its
gradients, against the float64 oracle.

Tolerances (largest error over max(|value|, rms)): a float32 sum of K random terms
is off by about 2^-24 sqrt(K) and at most 2^-24 K of the sum of sizes (K up to 5000:
1e-4); bfloat16 results and the rounding of dpre to bfloat16 are within 2^-8, 2e-2.
"""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_util import host, rel_err, say

pytestmark = pytest.mark.gpu

ops = None
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TOL = {"f32": 1e-4, "bf16": 2e-2}


def setup_module(module):
    global ops
    from paper_2607_05583_amd import ops as _ops
    ops = _ops


def problem(act, R, K, N, seed, bias=True, res=True, pad=0, shift=0):
    r = np.random.default_rng(seed)

    def t(*s):
        return torch.from_numpy(r.normal(size=s).astype(np.float32))

    buf = t(R * (K + pad) + shift).to(DT[act]).cuda()
    x = buf[shift:].view(R, K + pad)[:, :K]
    return dict(x=x, W=(t(K, N) / np.sqrt(K)).to(DT[act]).cuda(), b=t(N).cuda() if bias else None,
                res=t(R, N).to(DT[act]).cuda() if res else None, dy=t(R, N).to(DT[act]).cuda(),
                into=t(R, K).to(DT[act]).cuda() if res else None)


def check(q, act, fn, say_it):
    say(say_it)
    y, saved = ops.resonator_linear_fwd(q["x"], q["W"], q["b"], act=fn, residual=q["res"], save=True)
    g = ops.resonator_linear_bwd(q["x"], q["W"], q["dy"], pre=saved, act=fn, residual=q["into"], want_db=True)
    pre = saved.pre
    torch.cuda.synchronize()
    h = {k: None if v is None else host(v) for k, v in q.items()}
    yr, pr = O.linear_fwd(h["x"], h["W"], h["b"], fn, h["res"])
    gr = O.linear_bwd(h["x"], h["W"], h["dy"], h["b"], fn, h["into"])
    assert rel_err(host(y), yr) <= TOL[act]
    assert pre is None or rel_err(host(pre), pr) <= 1e-4
    if fn != "none":  # the other of the two ways: pre kept, or computed again
        if pre is None:
            pre = torch.from_numpy(pr.astype(np.float32)).cuda()
        again = ops.resonator_linear_bwd(q["x"], q["W"], q["dy"], pre=pre, act=fn, residual=q["into"], want_db=True)
        for k in ("dx", "dW"):
            assert rel_err(host(again[k]), gr[k]) <= TOL[act], k
        assert rel_err(host(again["db"]), gr["db"]) <= 1e-4
    for k in ("dx", "dW"):
        assert rel_err(host(g[k]), gr[k]) <= TOL[act], k
    assert rel_err(host(g["db"]), gr["db"]) <= 1e-4


SHAPES = [(1, 1, 1), (1, 64, 64), (3, 33, 17), (16, 256, 1024), (17, 200, 72), (64, 1000, 136), (65, 64, 320),
          (129, 130, 131), (256, 256, 256), (300, 512, 64), (1025, 96, 257), (2048, 320, 520), (4099, 64, 96)]


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("k", range(len(SHAPES)))
def test_linear_parity(act, k):
    R, K, N = SHAPES[k]
    fn = ("none", "relu", "silu", "gelu_tanh")[k % 4]
    q = problem(act, R, K, N, seed=k, bias=k % 3 != 1, res=k % 2 == 0)
    check(q, act, fn, f"linear {act} R={R} K={K} N={N} {fn}")


@pytest.mark.parametrize("act,R,K,N,fn,pad,shift", [
    ("bf16", 70, 128, 192, "silu", 8, 0), ("bf16", 70, 128, 192, "gelu_tanh", 3, 0), ("bf16", 300, 256, 256, "none", 0, 1),
    ("f32", 70, 128, 192, "silu", 4, 0), ("f32", 131, 64, 128, "relu", 1, 3), ("bf16", 1, 96, 64, "none", 5, 1),
    ("bf16", 5000, 128, 128, "relu", 0, 0), ("f32", 5000, 48, 80, "gelu_tanh", 0, 0), ("bf16", 7, 5000, 64, "none", 0, 0),
    ("f32", 2, 4096, 8, "silu", 0, 0), ("bf16", 20000, 32, 40, "silu", 8, 8)])
def test_linear_strides_alignment_and_long_sums(act, R, K, N, fn, pad, shift):
    q = problem(act, R, K, N, seed=R + K, pad=pad, shift=shift)
    check(q, act, fn, f"linear {act} R={R} K={K} N={N} {fn} pad={pad} shift={shift}")


@pytest.mark.parametrize("fn", ["relu", "silu", "gelu_tanh"])
def test_gradients_at_far_out_values(fn):
    """Arguments whose powers leave float32: values and slopes stay at their limits."""
    x = torch.tensor([[1e20], [-1e20], [30.0], [-30.0], [0.0]], device="cuda")
    W = torch.ones(1, 1, device="cuda")
    y, pre = ops.resonator_linear_fwd(x, W, act=fn, save=True)
    g = ops.resonator_linear_bwd(x, W, torch.ones_like(y), pre=pre, act=fn)
    assert torch.isfinite(y).all() and torch.isfinite(g["dx"]).all()
    with np.errstate(over="ignore"):
        want = O.act_value(host(x), fn)
    assert rel_err(host(y), want) <= 1e-6
    slope = np.array([1.0, 0.0, 1.0, 0.0, {"relu": 0.0}.get(fn, 0.5)])
    assert np.abs(host(g["dx"])[:, 0] - slope).max() <= 1e-6


def test_linear_is_reproducible_and_rows_do_not_depend_on_others():
    q = problem("bf16", 300, 256, 192, seed=3)
    y = ops.resonator_linear_fwd(q["x"], q["W"], q["b"], act="silu", residual=q["res"])
    assert torch.equal(y, ops.resonator_linear_fwd(q["x"], q["W"], q["b"], act="silu", residual=q["res"]))
    x2 = q["x"].clone()
    x2[100:] = float("nan")
    y2 = ops.resonator_linear_fwd(x2, q["W"], q["b"], act="silu", residual=q["res"])
    assert torch.equal(y2[:100], y[:100]) and torch.isnan(y2[100:]).all()


def test_linear_in_place_residual_and_batched_rows():
    q = problem("f32", 48, 64, 64, seed=4)
    want = ops.resonator_linear_fwd(q["x"], q["W"], q["b"], residual=q["res"])
    into = q["res"].clone()
    got = ops.resonator_linear_fwd(q["x"], q["W"], q["b"], residual=into, out=into)
    assert got.data_ptr() == into.data_ptr() and torch.equal(got, want)
    x3 = q["x"].view(4, 12, 64)
    assert torch.equal(ops.resonator_linear_fwd(x3, q["W"], q["b"], residual=q["res"].view(4, 12, 64)), want.view(4, 12, 64))
    wide = torch.zeros(4, 12, 80, device="cuda")
    wide[..., :64] = x3
    assert torch.equal(ops.resonator_linear_fwd(wide[..., :64], q["W"], q["b"]), ops.resonator_linear_fwd(x3, q["W"], q["b"]))


def test_linear_without_rows():
    W = torch.randn(8, 4, device="cuda")
    x = torch.empty(0, 8, device="cuda")
    y, pre = ops.resonator_linear_fwd(x, W, act="silu", save=True)
    assert y.shape == (0, 4)
    g = ops.resonator_linear_bwd(x, W, y, pre=pre, act="silu", want_db=True)
    assert g["dx"].shape == (0, 8) and torch.all(g["dW"] == 0) and torch.all(g["db"] == 0)


def test_linear_autograd():
    q = problem("f32", 70, 40, 24, seed=6)
    leaves = [v.clone().requires_grad_() for v in (q["x"], q["W"], q["b"], q["res"])]
    y = ops.resonator_linear(leaves[0], leaves[1], leaves[2], "gelu_tanh", leaves[3])
    y.backward(q["dy"])
    h = {k: host(v) for k, v in q.items()}
    gr = O.linear_bwd(h["x"], h["W"], h["dy"], h["b"], "gelu_tanh")
    for leaf, want in zip(leaves, (gr["dx"], gr["dW"], gr["db"], h["dy"])):
        assert rel_err(host(leaf.grad), want) <= 1e-4
    w = q["W"].clone().requires_grad_()
    ops.resonator_linear(q["x"], w).backward(q["dy"])
    assert rel_err(host(w.grad), O.linear_bwd(h["x"], h["W"], h["dy"])["dW"]) <= 1e-4


def test_linear_refusals():
    q = problem("f32", 8, 16, 12, seed=1)
    x, W, fwd, bwd = q["x"], q["W"], ops.resonator_linear_fwd, ops.resonator_linear_bwd
    bad = [
        (lambda: fwd(x, W, act="tanh"), ValueError),
        (lambda: fwd(x, W[:15]), ValueError),
        (lambda: fwd(x, W.t()), ValueError),
        (lambda: fwd(x, W.bfloat16()), ValueError),
        (lambda: fwd(x.half(), W.half()), TypeError),
        (lambda: fwd(x.cpu(), W), ValueError),
        (lambda: fwd(x.t().contiguous().t(), W), ValueError),
        (lambda: fwd(x[:1].expand(8, 16), W), ValueError),
        (lambda: fwd(x.view(2, 4, 16)[:, ::3], W), ValueError),
        (lambda: fwd(x, W, bias=q["b"][:5]), ValueError),
        (lambda: fwd(x, W, bias=q["b"].bfloat16()), ValueError),
        (lambda: fwd(x, W, residual=q["res"][:5]), ValueError),
        (lambda: fwd(x, torch.randn(16, 16, device="cuda"), out=x), Exception),
        (lambda: bwd(x, W, None), TypeError),
        (lambda: bwd(x, W, q["dy"], act="silu"), TypeError),
        (lambda: bwd(x, W, q["dy"][:3]), ValueError),
        (lambda: bwd(x, W, q["dy"], want_dx=False, want_dw=False), Exception),
        (lambda: bwd(x, W, q["dy"], residual=q["res"]), ValueError),
    ]
    for k, (call, kind) in enumerate(bad):
        with pytest.raises(kind):
            call()
            pytest.fail(f"case {k} was taken")
