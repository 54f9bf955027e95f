"""The linear product's large tiles against a float64 product, in every role that they have: the forward with bias, activation
and residual, dy act'(pre) with the sums of its columns, the data gradient, and the weight gradient with its sum cut in parts;
whole and odd sizes, tiles whose edges are not full, and more tiles than work-groups that stay.

Whole numbers: products and sums below 2^24 are exact in float32, so float32 results are equal and bfloat16 ones are the
exact result's rounding, bit for bit.

Bounds of the other test, element by element.  A float32 sum of K <= 40000 random terms, each rounding 2^-24 of the partial sum,
has an error of 2^-24 sqrt(K) / 2.4 of its size, 5e-6; five and a half of them with a factor of three for the activation are
below 1e-4 of max(|value|, rms).  A gradient's terms hold dy act'(pre) rounded to bfloat16, which is off by at most 2^-8 of it
(8 significant bits): independent errors, so that the sum is off by 2^-8 / sqrt(3) of the root of its terms' squares' sum, and
five and a half times that holds for 2 x 10^7 of them.  A bfloat16 result is the rounding of a value within these bounds, so it
lies between the bounds' roundings.
"""
import ctypes

import numpy as np
import pytest
import torch

from gpu_util import host, say

gpu = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SMALL, SQUARE, WIDE, DEEP = 0, 1, 2, 3

# act, R, K, N, and the tiles that are meant: of the forward, of dy act'(pre), dx and dW, with the parts of dW's sum
CASES = [
    ("bf16", 4100, 136, 1032, SQUARE, SQUARE, DEEP, SMALL, 10),
    ("bf16", 4100, 136, 1030, SQUARE, SQUARE, DEEP, SMALL, 10),   # outputs of any alignment
    ("f32", 4100, 136, 1032, SQUARE, SQUARE, SMALL, SMALL, 10),
    ("f32", 4100, 136, 1030, SQUARE, SQUARE, SMALL, SMALL, 10),
    ("bf16", 8200, 264, 1032, WIDE, SQUARE, WIDE, WIDE, 17),
    ("f32", 8200, 264, 1160, SQUARE, SQUARE, SQUARE, SQUARE, 8),  # more tiles than work-groups
    ("bf16", 13200, 264, 1288, WIDE, SQUARE, WIDE, WIDE, 14),     # more of all tiles
    ("bf16", 12000, 136, 1544, WIDE, SQUARE, WIDE, WIDE, 18),     # dx's sum is cut too
    ("bf16", 17000, 72, 520, WIDE, SQUARE, SQUARE, SQUARE, 49),
    ("f32", 17000, 72, 520, SQUARE, SQUARE, SQUARE, SQUARE, 51),
    ("f32", 5000, 1030, 1032, SQUARE, SQUARE, SQUARE, SQUARE, 3),
    ("bf16", 5000, 1030, 1032, WIDE, SQUARE, SQUARE, WIDE, 5),
    ("bf16", 40000, 40, 56, SMALL, SMALL, SMALL, SMALL, 63),      # more small tiles than work-groups
    ("f32", 40000, 40, 55, SMALL, SMALL, SMALL, SMALL, 63),
]


@pytest.mark.parametrize("act,R,K,N,fwd,dpre,dx,dW,parts", CASES)
def test_cases_reach_the_tiles(act, R, K, N, fwd, dpre, dx, dW, parts):
    """The library's rule (res::linear_plan) gives these tiles; where it changes, the cases have to follow."""
    from paper_2607_05583_amd import _lib
    plan = getattr(_lib.lib(), "_ZN3res11linear_planElllmbb")
    plan.restype, plan.argtypes = ctypes.c_uint64, [ctypes.c_int64] * 3 + [ctypes.c_size_t, ctypes.c_bool, ctypes.c_bool]
    es = DT[act].itemsize
    whole_n, whole_k = N * es % 16 == 0, K * es % 16 == 0
    got = [plan(R, N, K, es, False, whole_n), plan(R, N, K, es, True, False), plan(R, K, N, es, False, whole_k),
           plan(K, N, R, es, False, whole_n)]
    assert [v & 0xffffffff for v in got] == [fwd, dpre, dx, dW]
    assert got[3] >> 32 == parts


def _ops():
    from paper_2607_05583_amd import ops
    return ops


def _product(x, W, dy, b, into, fn):
    """(pre, dpre's function of a slope) and the gradients in 64 bits, from the device's inputs"""
    x, W, dy, b, into = (host(t) for t in (x, W, dy, b, into))
    pre = x @ W + b

    def grads(slope):
        d = dy * slope
        return dict(dx=d @ W.T + into, dW=x.T @ d, db=d.sum(0))

    return pre, grads


def _calls(ops, x, W, dy, b, res, into, fn):
    """The forward and the backward, twice: with what the forward keeps, and with pre the other way (kept, or computed again)."""
    y, saved = ops.resonator_linear_fwd(x, W, b, act=fn, residual=res, save=True)
    g = ops.resonator_linear_bwd(x, W, dy, pre=saved, act=fn, residual=into, want_db=True)
    other = g
    if fn != "none":
        pre = None if saved.pre is not None else torch.addmm(b, x.float(), W.float())
        other = ops.resonator_linear_bwd(x, W, dy, pre=ops.LinearSaved(pre, b), act=fn, residual=into, want_db=True)
    again = ops.resonator_linear_fwd(x, W, b, act=fn, residual=res)
    assert torch.equal(y, again)
    torch.cuda.synchronize()
    return y, saved, g, other


@gpu
@pytest.mark.parametrize("fn", ["none", "relu"])
@pytest.mark.parametrize("act,R,K,N", [c[:4] for c in CASES])
def test_whole_numbers(act, R, K, N, fn):
    ops = _ops()
    say(f"whole numbers {act} {R} {K} {N} {fn}")
    r = np.random.default_rng(R + K + N)

    def t(lo, hi, *s):
        return torch.from_numpy(r.integers(lo, hi + 1, s).astype(np.float32)).to(DT[act]).cuda()

    x, W, dy, res, into = t(-2, 2, R, K), t(-2, 2, K, N), t(-2, 2, R, N), t(-9, 9, R, N), t(-9, 9, R, K)
    b = torch.from_numpy(r.integers(-4, 5, N).astype(np.float32) + 0.5).cuda()  # (so that pre is never 0)
    y, saved, g, other = _calls(ops, x, W, dy, b, res, into, fn)
    pre, grads = _product(x, W, dy, b, into, fn)
    want = grads(pre > 0 if fn == "relu" else 1.0)
    want["y"] = (np.maximum(pre, 0.0) if fn == "relu" else pre) + host(res)

    def rounded(v, dtype):
        return torch.from_numpy(v.astype(np.float32)).to(dtype)

    assert torch.equal(y.cpu(), rounded(want["y"], DT[act]))
    if saved.pre is not None:
        assert torch.equal(saved.pre.cpu(), rounded(pre, torch.float32))
    for got in (g, other):
        for k in ("dx", "dW"):
            assert torch.equal(got[k].cpu(), rounded(want[k], DT[act])), k
        assert torch.equal(got["db"].cpu(), rounded(want["db"], torch.float32))


@gpu
@pytest.mark.parametrize("fn", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("act,R,K,N", [c[:4] for c in CASES])
def test_activations(act, R, K, N, fn):
    import oracle as O
    ops = _ops()
    say(f"activations {act} {R} {K} {N} {fn}")
    r = np.random.default_rng(R + K + N)

    def t(*s):
        return torch.from_numpy(r.normal(size=s).astype(np.float32))

    x, W, dy, res, into = (v.to(DT[act]).cuda() for v in (t(R, K), t(K, N) / K ** 0.5, t(R, N), t(R, N), t(R, K)))
    b = t(N).cuda()
    y, saved, g, other = _calls(ops, x, W, dy, b, res, into, fn)
    pre, grads = _product(x, W, dy, b, into, fn)
    slope = O.act_slope(pre, fn)
    want = grads(slope)

    def check(got, ref, dtype, off=0.0):
        off = off + 1e-4 * np.maximum(np.abs(ref), np.sqrt(np.mean(ref ** 2)))
        lo, hi = (host(torch.from_numpy(v).to(dtype)) for v in (ref - off, ref + off))  # (roundings keep the order)
        got = host(got)
        assert np.all((lo <= got) & (got <= hi)), np.max(np.abs(got - ref) / off)

    check(y, O.act_value(pre, fn) + host(res), DT[act])
    if saved.pre is not None:
        check(saved.pre, pre, torch.float32)
    d2 = (host(dy) * slope) ** 2
    each = 5.5 * 2.0 ** -8 / 3 ** 0.5 if act == "bf16" else 0.0
    off = dict(dx=each * np.sqrt(d2 @ (host(W) ** 2).T), dW=each * np.sqrt((host(x) ** 2).T @ d2))
    for got in (g, other):
        for k in ("dx", "dW"):
            check(got[k], want[k], DT[act], off[k])
        check(got["db"], want["db"], torch.float32)
