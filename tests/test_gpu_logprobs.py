"""Token log probabilities on the GPU against their float64 oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import select_oracle as O
from paper_2607_05583_amd import ops

from gpu_util import say
from select_util import DT, HALF, gpu, host, rounded, within

pytestmark = pytest.mark.gpu
ACTS = ["bf16", "f32"]
INF = float("inf")


def rows_of(dt, R, V, seed, wide=2.5, masked=0.0):
    r = np.random.default_rng(seed)
    x = rounded(wide * r.standard_normal((R, V)), dt)
    x[r.random((R, V)) < masked] = -INF
    tok = r.integers(0, V, R)
    tok[r.random(R) < 0.2] = -1
    return x, tok


def check(x, tok, dt, scale=1.0, top=0, pad=0, seed=0):
    R, V = x.shape
    t = gpu(x, dt)
    if pad:
        t = torch.cat([t, torch.full((R, pad), INF, device="cuda", dtype=t.dtype)], 1)[:, :V]
    tk = torch.tensor(tok, device="cuda")
    say(f"logprobs {dt} {R} x {V}, top {top}, scale {scale}, pad {pad}")
    o = ops.resonator_token_logprobs_fwd(t, tk, top=top, entropy=True, scale=scale)
    lp, ent, every = O.logprobs(x, tok, scale)
    # z - max is off by 2^-23 of its size, log S by a few roundings of sums of up to V / 64 terms in a row, each relative to
    # S >= 1; the entropy is a sum of p (z - max) of the same kind, at most as large as log V plus the spread
    most = np.where(np.isfinite(x).any(1), np.where(np.isfinite(x), x, -INF).max(1), 0)
    spread = np.where(np.isfinite(every), -every, 0).max(1) if V else 0
    e = 2.0 ** -23 * (V / 64 + 40)
    bound = lambda v: e + 2.0 ** -22 * np.abs(v)  # noqa: E731
    fine = np.isfinite(lp)
    got = host(o.logp)
    assert np.array_equal(fine, np.isfinite(got)) and np.array_equal(got[~fine], lp[~fine])
    within(got[fine], lp[fine], bound(lp[fine]), "logp")
    within(o.entropy, ent, e * (1 + np.log(V)) + 2.0 ** -22 * ent, "entropy")
    if top:
        ids = O.top(x, top)
        assert np.array_equal(o.top_ids.cpu().numpy(), ids)
        ref, got = np.take_along_axis(every, ids, 1), host(o.top_logp)
        # 1.6 times bf16's lowest value (-3.39e38) is -5.4e38, and float32 ends at -3.4028e38: it rounds to -inf
        ref = np.where(ref < -3.4029e38, -INF, ref)
        fine = np.isfinite(ref)
        assert np.array_equal(got[~fine], ref[~fine])
        within(got[fine], ref[fine], bound(ref[fine]), "top")
    r = np.random.default_rng(seed + 1)
    dl, de = np.float32(r.standard_normal(R)).astype(float), np.float32(r.standard_normal(R)).astype(float)
    for a, b in ((dl, None), (None, de), (dl, de)):
        g = ops.resonator_token_logprobs_bwd(t, tk, o, None if a is None else gpu(a), None if b is None else gpu(b), scale=scale)
        ref = O.logprobs_bwd(x, tok, a, b, scale)
        p = np.exp(every)
        # p is off by its exponent's error, and so is what it multiplies
        off = e + 2.0 ** -21 * (1 + np.where(p > 0, -every, 0))
        size = (0 if a is None else np.abs(a)[:, None]) + (0 if b is None else np.abs(b)[:, None] * (1 + np.where(p > 0, -every, 0) + ent[:, None]))
        hot = np.zeros_like(x)
        ok = tok >= 0
        hot[np.nonzero(ok)[0], tok[ok]] = 1
        if a is not None:
            hot *= np.abs(a)[:, None] * 2.0 ** -23
        within(g, ref, HALF[dt] * np.abs(ref) + scale * (off * p * size + (hot if a is not None else 0)), "gradient")
    return t, tk, o


# vectors that end inside, one work-group of 256 and of 512 threads, several passes of its loop
@pytest.mark.parametrize("dt", ACTS)
@pytest.mark.parametrize("R,V,top", [(1, 1, 1), (3, 2, 2), (5, 63, 7), (4, 257, 64), (7, 1000, 20), (2, 8192, 1), (3, 8193, 20), (2, 32768, 64),
                                     (2, 50305, 8), (1, 131073, 20)])
def test_sizes(R, V, top, dt):
    x, tok = rows_of(dt, R, V, R + V)
    check(x, tok, dt, top=top, pad=V % 3)


@pytest.mark.parametrize("dt", ACTS)
@pytest.mark.parametrize("scale", [0.3, 1.7])
def test_scales(scale, dt):
    x, tok = rows_of(dt, 6, 3001, 5)
    check(x, tok, dt, scale=scale, top=9)


@pytest.mark.parametrize("dt", ACTS)
@pytest.mark.parametrize("V", [40, 9001])
def test_masked_tokens(V, dt):
    """Forbidden tokens: most, all but one, all."""
    x, tok = rows_of(dt, 6, V, 7, masked=0.97)
    x[0] = -INF
    x[1] = -INF
    x[1, V // 2] = -3.0
    x[2, :] = -INF
    x[2, [V - 1, 3]] = 2.0  # equal
    tok[:3] = [1, V // 2, 0]
    check(x, tok, dt, top=12)


@pytest.mark.parametrize("dt", ACTS)
@pytest.mark.parametrize("scale", [1.0, 1.6])
def test_masks_of_the_lowest_value(scale, dt):
    """Tokens at the type's lowest value count for nothing beside others and are equals among themselves."""
    x, tok = rows_of(dt, 4, 5000, 8)
    low = float(torch.finfo(DT[dt]).min)
    x[0, 1:] = low
    x[1] = low
    x[2, ::2] = low
    tok[:] = [0, 7, 1, 5]
    t, tk, o = check(x, tok, dt, scale=scale, top=4)
    assert abs(o.logp[0].item()) < 1e-6 and abs(o.logp[1].item() + math.log(5000)) < 1e-5


@pytest.mark.parametrize("dt", ACTS)
@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "two values", "zeros of both signs"])
@pytest.mark.parametrize("V", [700, 20000])
def test_rows_with_more_candidates_than_the_list_takes(V, kind, dt):
    x = {"equal": np.full((2, V), 1.5), "rising": np.linspace(-20, 20, V)[None].repeat(2, 0), "falling": np.linspace(20, -20, V)[None].repeat(2, 0),
         "two values": np.where(np.arange(V) % 3 == 1, 2.0, 1.0)[None].repeat(2, 0),
         "zeros of both signs": np.where(np.arange(V) % 2 == 1, 0.0, -0.0)[None].repeat(2, 0)}[kind]
    check(rounded(x, dt), np.array([0, V - 1]), dt, top=33)


@pytest.mark.parametrize("dt", ACTS)
@pytest.mark.parametrize("V", [100, 30000])
def test_nan_and_infinity(V, dt):
    x, tok = rows_of(dt, 4, V, 9)
    tok[:] = [1, 2, 3, 4]
    t = gpu(x, dt)
    t[1, V - 1], t[2, 0] = float("nan"), INF
    say(f"logprobs {dt} NaN {V}")
    o = ops.resonator_token_logprobs_fwd(t, torch.tensor(tok, device="cuda"), top=3, entropy=True)
    assert torch.isnan(o.logp).tolist() == [False, True, True, False] == torch.isnan(o.entropy).tolist()
    assert o.top_ids[1, 0] == V - 1 and o.top_ids[2, 0] == 0 and torch.isnan(o.top_logp[1:3, 0]).all()
    assert ((o.top_ids >= 0) & (o.top_ids < V)).all()


@pytest.mark.parametrize("dt", ACTS)
def test_tokens_that_are_ignored_or_no_tokens(dt):
    x, _ = rows_of(dt, 4, 300, 10)
    t, tk = gpu(x, dt), torch.tensor([-1, -100, 300, 2 ** 40], device="cuda")
    o = ops.resonator_token_logprobs_fwd(t, tk)
    assert o.logp[:2].tolist() == [0, 0] and torch.isnan(o.logp[2:]).all()
    g = ops.resonator_token_logprobs_bwd(t, tk, o, torch.ones(4, device="cuda"))
    assert not g[:2].any() and torch.isnan(g[2:]).all()


@pytest.mark.parametrize("dt", ACTS)
def test_gradient_in_the_logits_place_and_in_wider_rows(dt):
    x, tok = rows_of(dt, 5, 4099, 11)
    t, tk, o = check(x, tok, dt, pad=5)
    dl = torch.ones(5, device="cuda")
    g = ops.resonator_token_logprobs_bwd(t, tk, o, dl)
    wide = torch.full((5, 4110), 7.0, device="cuda", dtype=DT[dt])
    ops.resonator_token_logprobs_bwd(t, tk, o, dl, out=wide[:, 3:4102])
    assert torch.equal(wide[:, 3:4102], g) and (wide[:, :3] == 7).all() and (wide[:, 4102:] == 7).all()
    into = t.clone()
    assert ops.resonator_token_logprobs_bwd(into, tk, o, dl, out=into) is into and torch.equal(into, g)


@pytest.mark.parametrize("dt", ACTS)
def test_autograd_and_leading_dimensions(dt):
    x, tok = rows_of(dt, 6, 900, 12)
    t = gpu(x, dt).view(2, 3, 900).requires_grad_()
    tk = torch.tensor(tok, device="cuda").view(2, 3)
    lp, ent = ops.resonator_token_logprobs(t, tk, entropy=True, scale=0.8)
    assert lp.shape == ent.shape == (2, 3)
    (-lp.sum() * 0.5 + ent.sum()).backward()
    o = ops.resonator_token_logprobs_fwd(t.detach(), tk, entropy=True, scale=0.8)
    half = torch.full((2, 3), -0.5, device="cuda")
    assert torch.equal(t.grad, ops.resonator_token_logprobs_bwd(t.detach(), tk, o, half, -2 * half, scale=0.8))
    with torch.no_grad():
        assert not ops.resonator_token_logprobs(t, tk).requires_grad


def test_no_rows_and_refusals():
    t, tk = torch.zeros(0, 10, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda")
    o = ops.resonator_token_logprobs_fwd(t, tk, top=2, entropy=True)
    assert o.logp.shape == (0,) and o.top_ids.shape == (0, 2) and ops.resonator_token_logprobs_bwd(t, tk, o).shape == (0, 10)
    t, tk = torch.zeros(3, 10, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    f = ops.resonator_token_logprobs_fwd
    for bad in [(t, tk[:2]), (t, tk.int()), (t.half(), tk), (t.t(), torch.zeros(10, dtype=torch.int64, device="cuda")), (t.cpu(), tk)]:
        with pytest.raises((ValueError, TypeError)):
            f(*bad)
    for kw in (dict(top=11), dict(top=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=INF)):
        with pytest.raises(Exception):
            f(t, tk, **kw)
    with pytest.raises(ValueError):
        f(torch.zeros(3, 100, device="cuda"), tk, top=65)
    o = f(t, tk)
    with pytest.raises(TypeError):
        ops.resonator_token_logprobs_bwd(t, tk, o, dentropy=torch.ones(3, device="cuda"))
    with pytest.raises(Exception, match="overlap"):  # neither the logits' place nor apart from it
        both = torch.zeros(41, device="cuda")
        ops.resonator_token_logprobs_bwd(both[:30].view(3, 10), tk, o, out=both[11:].view(3, 10))


def test_graph_replays():
    x, tok = rows_of("bf16", 64, 5000, 13)
    t, tk = gpu(x, "bf16"), torch.tensor(tok, device="cuda")
    dl = torch.ones(64, device="cuda")

    def step():
        o = ops.resonator_token_logprobs_fwd(t, tk, top=5, entropy=True)
        return [*o, ops.resonator_token_logprobs_bwd(t, tk, o, dl, dl)]

    eager = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for _ in range(3):
        for v in captured:
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(eager, captured))
        assert all(torch.equal(p, q) for p, q in zip(eager, step()))
