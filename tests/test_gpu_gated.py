"""GPU parity of the gated scan against the float64 oracle on identical inputs.

Tolerances (largest error over max(|value|, rms) of a tensor): 1e-4 for float32
results and 2e-2 where the result is rounded to bfloat16, as for the mixing.  A
float32 step multiplies the state by an a rounded to 2^-24 and adds with 2^-24, so a
state that remembers n steps is off by at most 2^-23 n relative (n below 400 here:
5e-5).
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


def problem(act, B, L, D, seed=0, fused=False, h0=False, lengths=None, pad=0, gamma_lo=1e-2):
    """Inputs on the GPU; behind a row's length they hold NaN and infinities."""
    r = np.random.default_rng(seed)
    p = torch.from_numpy(r.normal(scale=1.5, size=(B, L, 3 * D + pad)).astype(np.float32)).to(DT[act])
    dy = torch.from_numpy(r.normal(size=(B, L, D)).astype(np.float32)).to(DT[act])
    q = dict(gamma=torch.from_numpy(np.exp(r.uniform(np.log(gamma_lo), np.log(8.0), D)).astype(np.float32)).cuda(),
             dh=torch.from_numpy(r.normal(size=(B, D)).astype(np.float32)).cuda())
    if h0:
        q["h0"] = torch.from_numpy(r.normal(size=(B, D)).astype(np.float32)).cuda()
    if lengths is not None:
        for b, n in enumerate(lengths):
            p[b, max(0, n):] = float("nan")
            dy[b, max(0, n):] = float("inf")
        q["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    p, q["dy"] = p.cuda(), dy.cuda()
    q["xri"] = [p[..., k * D + pad:(k + 1) * D + pad] for k in range(3)]
    if not fused:
        q["xri"] = [v.contiguous() for v in q["xri"]]
    return q


def oracle(q, grads=True):
    x, r, i = (np.nan_to_num(host(v)) for v in q["xri"])
    n = None if "lengths" not in q else q["lengths"].cpu().numpy()
    h0 = None if "h0" not in q else host(q["h0"])
    y, h, hs = O.gated_scan_fwd(x, r, i, host(q["gamma"]), h0, n)
    if not grads:
        return y, h
    dy = host(q["dy"])
    dy = np.where(np.isfinite(dy), dy, 0.0)
    return y, h, O.gated_scan_bwd(x, r, i, host(q["gamma"]), dy, h0, n, host(q["dh"]))


SHAPES = [
    # act, B, L, D, fused, h0, lengths, pad
    ("f32", 1, 1, 1, False, False, None, 0),
    ("bf16", 2, 1, 64, True, True, None, 0),
    ("f32", 2, 127, 64, False, True, None, 0),
    ("f32", 1, 129, 66, True, False, None, 0),
    ("bf16", 3, 300, 128, True, True, [300, 0, 129], 0),
    ("bf16", 2, 515, 65, True, False, None, 0),
    ("bf16", 1, 700, 200, True, True, None, 1),
    ("f32", 5, 257, 20, True, True, [257, 1, 0, 128, 256], 0),
    ("f32", 2, 1200, 36, False, False, [1100, 1200], 0),
    ("bf16", 1, 4100, 64, False, False, None, 0),
]


@pytest.mark.parametrize("act,B,L,D,fused,h0,lengths,pad", SHAPES)
def test_scan_parity(act, B, L, D, fused, h0, lengths, pad):
    say(f"gated scan {act} B={B} L={L} D={D} fused={fused} h0={h0} lengths={lengths} pad={pad}")
    q = problem(act, B, L, D, seed=L + D, fused=fused, h0=h0, lengths=lengths, pad=pad)
    y, h, carry = ops.resonator_gated_scan_fwd(*q["xri"], q["gamma"], h0=q.get("h0"), lengths=q.get("lengths"),
                                               return_state=True, save=True)
    dp = torch.full((B, L, 3 * D + pad), 7.0, dtype=DT[act], device="cuda")
    out = [dp[..., k * D + pad:(k + 1) * D + pad] for k in range(3)]
    g = ops.resonator_gated_scan_bwd(*q["xri"], q["gamma"], q["dy"], h0=q.get("h0"), lengths=q.get("lengths"),
                                     dh_out=q["dh"], carry=carry, want_dh0=True, out=out)
    torch.cuda.synchronize()
    yr, hr, gr = oracle(q)
    assert rel_err(host(y), yr) <= TOL[act]
    assert rel_err(host(h), hr) <= TOL["f32"]
    for k in ("dx", "dr", "di"):
        assert rel_err(host(g[k]), gr[k]) <= TOL[act], k
    for k in ("dgamma", "dh0"):
        assert rel_err(host(g[k]), gr[k]) <= TOL["f32"], k
    if pad:
        assert torch.all(dp[..., :pad] == 7.0)
    if lengths is not None:
        for b, n in enumerate(lengths):
            assert torch.all(y[b, n:] == 0) and all(torch.all(g[k][b, n:] == 0) for k in ("dx", "dr", "di"))


def test_scan_without_saved_states_and_without_optional_arguments():
    q = problem("bf16", 2, 333, 72, seed=5)
    y, carry = ops.resonator_gated_scan_fwd(*q["xri"], q["gamma"], save=True)
    g = ops.resonator_gated_scan_bwd(*q["xri"], q["gamma"], q["dy"], carry=carry)
    again = ops.resonator_gated_scan_bwd(*q["xri"], q["gamma"], q["dy"])
    assert set(g) == {"dx", "dr", "di", "dgamma"}
    assert all(torch.equal(g[k], again[k]) for k in g)
    assert torch.equal(y, ops.resonator_gated_scan_fwd(*q["xri"], q["gamma"]))


def test_scan_is_reproducible_and_its_workspace_reusable():
    ws = ops.gated_scan_workspace(torch.bfloat16, 2, 5000, 128, "cuda")
    want = {}
    for turn in range(3):
        for act, B, L, D in (("bf16", 2, 5000, 128), ("f32", 1, 900, 40), ("bf16", 1, 33, 256)):
            q = problem(act, B, L, D, seed=L)
            y, h, carry = ops.resonator_gated_scan_fwd(*q["xri"], q["gamma"], return_state=True, save=True, ws=ws)
            g = ops.resonator_gated_scan_bwd(*q["xri"], q["gamma"], q["dy"], carry=carry, want_dh0=True, ws=ws)
            got = [y, h, carry] + [g[k] for k in sorted(g)]
            if turn == 0:
                want[L] = got
            assert all(torch.equal(a, b) for a, b in zip(want[L], got)), (turn, L)


def test_scan_is_causal_and_splits():
    q = problem("f32", 2, 1500, 64, seed=9, h0=True)
    y, h = ops.resonator_gated_scan_fwd(*q["xri"], q["gamma"], h0=q["h0"], return_state=True)
    cut = [v.clone() for v in q["xri"]]
    for v in cut:
        v[:, 700:] = 3.0
    assert torch.equal(ops.resonator_gated_scan_fwd(*cut, q["gamma"], h0=q["h0"])[:, :700], y[:, :700])
    state = q["h0"].clone()
    parts = []
    for lo, hi in ((0, 700), (700, 701), (701, 1500)):
        yp, state = ops.resonator_gated_scan_fwd(*[v[:, lo:hi] for v in q["xri"]], q["gamma"], h0=state,
                                                 return_state=True, h_out=state)
        parts.append(yp)
    assert rel_err(host(torch.cat(parts, 1)), host(y)) <= 1e-5 and rel_err(host(state), host(h)) <= 1e-5


@pytest.mark.parametrize("act,B,D,fused", [("bf16", 64, 256, True), ("f32", 3, 33, True), ("f32", 1, 1, False)])
def test_steps_continue_a_prompt(act, B, D, fused):
    say(f"gated steps {act} B={B} D={D}")
    q = problem(act, B, 24, D, seed=D, fused=fused)
    _, h = ops.resonator_gated_scan_fwd(*[v[:, :16] for v in q["xri"]], q["gamma"], return_state=True)
    ys = [ops.resonator_gated_scan_step(*[v[:, t] for v in q["xri"]], q["gamma"], h) for t in range(16, 23)]
    h2 = torch.empty_like(h)
    keep = h.clone()
    ys.append(ops.resonator_gated_scan_step(*[v[:, 23] for v in q["xri"]], q["gamma"], h, h_out=h2))
    assert torch.equal(keep, h)
    yr, hr = oracle(q, grads=False)
    assert rel_err(host(torch.stack(ys, 1)), yr[:, 16:]) <= TOL[act] and rel_err(host(h2), hr) <= TOL["f32"]


def test_closed_gates_extreme_logits_and_zero_damping():
    """Logits far out, a damping of zero and of the underflow's size: finite results and the limits of the formulas."""
    q = problem("f32", 1, 130, 8, seed=3, h0=True)
    x, r, i = q["xri"]
    r[0, :, 0], r[0, :, 1], i[0, :, 2] = -200.0, 200.0, -200.0
    r[0, :, 3], r[0, :, 4] = -80.0, float("-inf")
    q["gamma"][5], q["gamma"][6] = 0.0, 1e-38
    q["gamma"][1] = 200.0
    y, h, carry = ops.resonator_gated_scan_fwd(x, r, i, q["gamma"], h0=q["h0"], return_state=True, save=True)
    g = ops.resonator_gated_scan_bwd(x, r, i, q["gamma"], q["dy"], carry=carry, want_dh0=True)
    assert all(torch.isfinite(v).all() for v in (y, h, *g.values()))
    yr, hr, gr = O.gated_scan_fwd(*(host(v) for v in (x, r, i)), host(q["gamma"]), host(q["h0"]))[:2] + (
        O.gated_scan_bwd(*(host(v) for v in (x, r, i)), host(q["gamma"]), host(q["dy"]), host(q["h0"])),)
    assert rel_err(host(y), yr) <= 1e-4
    keep = [0, 1, 2, 3, 4, 5, 7]  # (below 1e-36 the drive's weight, at most 1e-18, is taken as zero)
    for k in ("dx", "dr", "di", "dh0"):
        assert rel_err(host(g[k])[..., keep], gr[k][..., keep]) <= 1e-4, k
    assert rel_err(host(g["dgamma"])[[1, 2, 5, 7]], gr["dgamma"][[1, 2, 5, 7]]) <= 1e-4


def test_empty_sequences():
    x = torch.empty((3, 0, 40), device="cuda")
    gamma = torch.ones(40, device="cuda")
    h0 = torch.randn(3, 40, device="cuda")
    y, h, carry = ops.resonator_gated_scan_fwd(x, x, x, gamma, h0=h0, return_state=True, save=True)
    assert y.shape == (3, 0, 40) and torch.equal(h, h0) and carry.shape == (3, 0, 40)
    g = ops.resonator_gated_scan_bwd(x, x, x, gamma, x, dh_out=h0, carry=carry, want_dh0=True)
    assert torch.equal(g["dh0"], h0) and torch.all(g["dgamma"] == 0)


def test_time_major_and_broadcast_inputs():
    q = problem("f32", 3, 140, 24, seed=8)
    want = ops.resonator_gated_scan_fwd(*q["xri"], q["gamma"])
    tm = [v.transpose(0, 1).contiguous().transpose(0, 1) for v in q["xri"]]
    assert not tm[0].is_contiguous() and torch.equal(ops.resonator_gated_scan_fwd(*tm, q["gamma"]), want)
    one = q["xri"][1][:1, :1].expand(3, 140, 24)  # one logit for all rows and steps
    y = ops.resonator_gated_scan_fwd(q["xri"][0], one, q["xri"][2], q["gamma"])
    assert torch.equal(y, ops.resonator_gated_scan_fwd(q["xri"][0], one.contiguous(), q["xri"][2], q["gamma"]))


def test_autograd_matches_the_direct_calls():
    q = problem("f32", 2, 260, 16, seed=12, h0=True)
    leaves = [v.clone().requires_grad_() for v in (*q["xri"], q["gamma"], q["h0"])]
    y, h = ops.resonator_gated_scan(*leaves[:4], h0=leaves[4])
    ((y * q["dy"]).sum() + (h * q["dh"]).sum()).backward()
    g = ops.resonator_gated_scan_bwd(*q["xri"], q["gamma"], q["dy"], h0=q["h0"], dh_out=q["dh"], want_dh0=True)
    for leaf, k in zip(leaves, ("dx", "dr", "di", "dgamma", "dh0")):
        assert torch.equal(leaf.grad, g[k]), k
    leaves[0].grad = None
    y, h = ops.resonator_gated_scan(*leaves[:4], h0=leaves[4])
    h.sum().backward()  # only the state has a gradient
    g = ops.resonator_gated_scan_bwd(*q["xri"], q["gamma"], torch.zeros_like(q["dy"]), h0=q["h0"],
                                     dh_out=torch.ones_like(q["dh"]))
    assert torch.equal(leaves[0].grad, g["dx"])


def test_scan_on_another_stream_and_in_a_graph():
    q = problem("bf16", 2, 900, 64, seed=21)
    ws = ops.gated_scan_workspace(torch.bfloat16, 2, 900, 64, "cuda")
    want = ops.resonator_gated_scan_fwd(*q["xri"], q["gamma"], ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        assert torch.equal(ops.resonator_gated_scan_fwd(*q["xri"], q["gamma"], ws=ws), want)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            y, carry = ops.resonator_gated_scan_fwd(*q["xri"], q["gamma"], save=True, ws=ws)
            g = ops.resonator_gated_scan_bwd(*q["xri"], q["gamma"], q["dy"], carry=carry, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    eager = None
    for _ in range(3):
        y.zero_()
        g["dx"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        now = ops.resonator_gated_scan_bwd(*q["xri"], q["gamma"], q["dy"], ws=ws)
        assert torch.equal(g["dx"], now["dx"]) and torch.equal(g["dgamma"], now["dgamma"])


def test_scan_refusals():
    q = problem("f32", 2, 40, 16)
    x, r, i = q["xri"]
    fwd = ops.resonator_gated_scan_fwd
    bad = [
        (lambda: fwd(x, r[:, :39], i, q["gamma"]), ValueError),
        (lambda: fwd(x, r.bfloat16(), i, q["gamma"]), ValueError),
        (lambda: fwd(x.double(), r.double(), i.double(), q["gamma"]), TypeError),
        (lambda: fwd(x.cpu(), r, i, q["gamma"]), ValueError),
        (lambda: fwd(x, r, i, q["gamma"][:15]), ValueError),
        (lambda: fwd(x, r, i, None), TypeError),
        (lambda: fwd(x.transpose(1, 2).contiguous().transpose(1, 2), r, i, q["gamma"]), ValueError),
        (lambda: fwd(x, r, i, q["gamma"], h0=torch.zeros(2, 15, device="cuda")), ValueError),
        (lambda: fwd(x, r, i, q["gamma"], lengths=torch.zeros(2, device="cuda", dtype=torch.int64)), ValueError),
        (lambda: fwd(x, r, i, q["gamma"], ws=torch.zeros(16, device="cuda", dtype=torch.uint8)), Exception),
        (lambda: fwd(x, r, i, q["gamma"], out=x), Exception),
        (lambda: ops.resonator_gated_scan_bwd(x, r, i, q["gamma"], q["dy"][:1]), ValueError),
        (lambda: ops.resonator_gated_scan_bwd(x, r, i, q["gamma"], q["dy"], out=(x, r, i)), Exception),
        (lambda: ops.resonator_gated_scan_bwd(x, r, i, q["gamma"], q["dy"], carry=torch.zeros(2, 2, 16, device="cuda")),
         ValueError),
        (lambda: ops.resonator_gated_scan_step(x[:, 0], r[:, 0], i[:, 0], q["gamma"], None), TypeError),
    ]
    dp = torch.empty(2, 40, 16, device="cuda")
    bad.append((lambda: ops.resonator_gated_scan_bwd(x, r, i, q["gamma"], q["dy"],
                                                     out=(dp, dp, torch.empty_like(dp))), Exception))
    for k, (call, kind) in enumerate(bad):
        with pytest.raises(kind):
            call()
            pytest.fail(f"case {k} was taken")
