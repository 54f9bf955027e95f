"""The linear product for few rows, as decoding and small models call it: every sum in one work-group, or cut over several.

Tolerances (largest error over max(|value|, rms)): a float32 sum of K <= 4100 random terms is off by about 2^-24 sqrt(K) of
its size, and less than 1e-4 with a factor of twenty; a bfloat16 result is rounded once, 2^-9 of its size, 1e-2 with a factor
of five for results that are small beside their sum.
"""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_util import host, rel_err, say

pytestmark = pytest.mark.gpu

ops = None
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TOL = {"f32": 1e-4, "bf16": 1e-2}


def setup_module(module):
    global ops
    from paper_2607_05583_amd import ops as _ops
    ops = _ops


def problem(act, R, K, N, seed):
    r = np.random.default_rng(seed)

    def t(*s):
        return torch.from_numpy(r.normal(size=s).astype(np.float32)).cuda()

    return t(R, K).to(DT[act]), (t(K, N) / K ** 0.5).to(DT[act]), t(N), t(R, N).to(DT[act])


# K of less than a step, of fewer steps than waves, with a last step that is not whole; the borders of the rule; odd N
SIZES = [(1, 1, 1), (3, 31, 5), (64, 32, 64), (65, 33, 66), (2, 264, 40), (130, 250, 72), (16, 256, 768), (64, 1000, 64),
         (64, 1025, 128), (7, 2048, 200), (70, 2056, 70), (1, 4100, 33), (300, 520, 300)]


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("R,K,N", SIZES)
def test_few_rows(act, R, K, N):
    x, W, b, res = problem(act, R, K, N, 7 * R + K + N)
    for fn in ("none", "relu", "silu", "gelu_tanh"):
        say(f"few rows {act} {R} {K} {N} {fn}")
        y, saved = ops.resonator_linear_fwd(x, W, b, act=fn, residual=res, save=True)
        ry, rp = O.linear_fwd(host(x), host(W), host(b), fn, host(res))
        assert rel_err(host(y), ry) <= TOL[act]
        if saved.pre is not None:
            assert rel_err(host(saved.pre), rp) <= 1e-4
        assert torch.equal(y, ops.resonator_linear_fwd(x, W, b, act=fn, residual=res))  # the same every time
        bare = ops.resonator_linear_fwd(x, W, act=fn)
        assert rel_err(host(bare), O.linear_fwd(host(x), host(W), None, fn)[0]) <= TOL[act]


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("R,K,N", [(5, 40, 264), (64, 72, 512), (1, 96, 1000), (33, 24, 2000)])
def test_gradients_of_few_rows(act, R, K, N):
    """The data gradient's sum runs over N."""
    x, W, b, dy = problem(act, R, K, N, R + K + N)
    say(f"gradients {act} {R} {K} {N}")
    y, saved = ops.resonator_linear_fwd(x, W, b, act="silu", save=True)
    g = ops.resonator_linear_bwd(x, W, dy, pre=saved, act="silu", want_db=True)
    r = O.linear_bwd(host(x), host(W), host(dy), host(b), "silu")
    # (bf16: dy act'(pre) is rounded before both products too)
    for k in ("dx", "dW"):
        assert rel_err(host(g[k]), r[k]) <= 2 * TOL[act], k
    assert rel_err(host(g["db"]), r["db"]) <= 1e-4


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_not_finite(act):
    """A row that is not finite stays alone, also beside rows that are read again past the end."""
    x, W, b, res = problem(act, 5, 200, 72, 1)
    x[4, 3] = float("nan")
    x[1, 7] = float("inf")
    say(f"not finite {act}")
    y = ops.resonator_linear_fwd(x, W, b, residual=res)
    ok = torch.isfinite(y).all(1).tolist()
    assert ok == [True, False, True, True, False]


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_over_the_residual_and_on_another_stream(act):
    x, W, b, res = problem(act, 33, 256, 264, 3)
    say(f"in place, other stream {act}")
    want = ops.resonator_linear_fwd(x, W, b, act="relu", residual=res)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = res.clone()
        got = ops.resonator_linear_fwd(x, W, b, act="relu", residual=y, out=y)
    torch.cuda.current_stream().wait_stream(s)
    assert got.data_ptr() == y.data_ptr() and torch.equal(y, want)
