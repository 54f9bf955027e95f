"""A selective layer: projection, short convolution, selective scan, output projection and MLP together, against the float64
oracles, as training, prefill and decoding call it; and the model of the examples."""
import importlib.util
import os
import sys

import numpy as np
import pytest
import torch

from oracle import layer_oracle as LO
from oracle import select_oracle as SO
from paper_2607_05583_amd import ops

from gpu_util import rel_err, say
from select_util import DT, Scan, gpu, host, rounded

pytestmark = pytest.mark.gpu
# Six operators in a row, each rounding its results (2^-8 or 2^-24 of them) and the backward as many again: a dozen roundings that
# later products mix, and the scan's bf16 weights; float32's 1e-4 is the bound of the other layers' tests.
TOL = {"bf16": 14 * 2.0 ** -8, "f32": 1e-4}


class _Off:
    """Stands in for the native module: takes nothing, so the Python code runs."""

    def __getattr__(self, name):
        return lambda *a: None


@pytest.fixture(params=["native", "python"])
def path(request, monkeypatch):
    monkeypatch.setattr(ops, "_NATIVE", ops._native() if request.param == "native" else _Off())
    return request.param


def problem(act, B, L, d, H, P, G, N, K, f, seed=0):
    r = np.random.default_rng(seed)
    C = H * P + 2 * G * N
    w = lambda k, n: rounded(r.standard_normal((k, n)) / k ** 0.5, act)  # noqa: E731
    v = lambda *s, by=1.0: np.float32(by * r.standard_normal(s)).astype(float)  # noqa: E731
    p = ops.SelectiveLayerParams(w(d, C + H), v(C + H, by=0.1), v(C, K, by=0.5), v(C, by=0.1), np.float32(np.exp(r.uniform(-2, 1, H))).astype(float),
                                 v(H) - 1, v(H), w(H * P, d), v(d, by=0.1), w(d, f), v(f, by=0.1), w(f, d), v(d, by=0.1))
    q = dict(p=p, sizes=(B, L, d, H, P, G, N, K), x=rounded(r.standard_normal((B, L, d)), act), dout=rounded(r.standard_normal((B, L, d)), act),
             state=(rounded(r.standard_normal((B, K - 1, C)), act), v(B, H, P, N)), dstate=(rounded(r.standard_normal((B, K - 1, C)), act), v(B, H, P, N)))
    weights = {"Wp", "Wo", "W1", "W2"}
    q["gp"] = ops.SelectiveLayerParams(*(gpu(t, act if n in weights else None) for n, t in zip(p._fields, p)))
    q["gx"], q["gdout"] = gpu(q["x"], act), gpu(q["dout"], act)
    q["gstate"], q["gdstate"] = (ops.SelectiveState(gpu(a, act), gpu(b)) for a, b in (q["state"], q["dstate"]))
    return q


def oracle(q, lengths=None):
    """(out, last inputs, last state, gradients as a dict) in float64."""
    p, (B, L, d, H, P, G, N, K) = q["p"], q["sizes"]
    C = H * P + 2 * G * N
    u = q["x"] @ p.Wp + p.bp
    v, last = SO.conv_fwd(u[..., :C], p.w, p.wb, "silu", q["state"][0], lengths)
    cut = lambda t: (t[..., :H * P].reshape(B, L, H, P), t[..., H * P:H * P + G * N].reshape(B, L, G, N), t[..., H * P + G * N:].reshape(B, L, G, N))  # noqa: E731
    x, b, c = cut(v)
    more = dict(bias=p.dt_bias, skip=p.skip, h0=q["state"][1], lengths=lengths)
    y, hs = SO.scan_fwd(x, u[..., C:], b, c, p.gamma, **more)
    yf = y.reshape(B, L, H * P)
    z = q["x"] + yf @ p.Wo + p.bo
    pre = z @ p.W1 + p.b1
    m = LO.act_value(pre, "gelu_tanh")
    out = z + m @ p.W2 + p.b2
    two = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
    do = q["dout"]
    dpre = (do @ p.W2.T) * LO.act_slope(pre, "gelu_tanh")
    dz = do + dpre @ p.W1.T
    g = SO.scan_bwd(x, u[..., C:], b, c, p.gamma, (dz @ p.Wo.T).reshape(y.shape), dh=q["dstate"][1], **more)
    dv = np.concatenate([g["dx"].reshape(B, L, -1), g["db"].reshape(B, L, -1), g["dc"].reshape(B, L, -1)], -1)
    dxc, dw, dwb, dfirst = SO.conv_bwd(u[..., :C], p.w, dv, p.wb, "silu", q["state"][0], lengths, q["dstate"][0])
    du = np.concatenate([dxc, g["ddt"]], -1)
    dp = ops.SelectiveLayerParams(two(q["x"]).T @ two(du), two(du).sum(0), dw, dwb, g["dgamma"], g["ddt_bias"], g["dskip"], two(yf).T @ two(dz),
                                  two(dz).sum(0), two(z).T @ two(dpre), two(dpre).sum(0), two(m).T @ two(do), two(do).sum(0))
    return out, last, hs[-1], dict(dx=dz + du @ p.Wp.T, dp=dp, dfirst=dfirst, dh0=g["dh0"])


SIZES = [(2, 70, 32, 4, 16, 2, 16, 4, 64), (1, 200, 48, 3, 24, 1, 10, 3, 40)]


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("sizes", SIZES)
def test_forward_and_backward(path, sizes, act):
    say(f"selective layer {path} {act} {sizes}")
    q = problem(act, *sizes, seed=1)
    G = sizes[5]
    out, last, h, g = oracle(q)
    got, s, saved = ops.resonator_selective_layer_fwd(q["gx"], q["gp"], G, state=q["gstate"], return_state=True, save=True)
    assert rel_err(host(got), out) <= TOL[act] and rel_err(host(s.conv), last) <= TOL[act] and rel_err(host(s.h), h) <= TOL[act]
    d = ops.resonator_selective_layer_bwd(q["gx"], q["gp"], q["gdout"], saved, G, state=q["gstate"], dstate=q["gdstate"], want_dstate=True)
    assert rel_err(host(d["dx"]), g["dx"]) <= TOL[act]
    for name, a, b in zip(q["p"]._fields, d["dp"], g["dp"]):
        assert a.dtype == getattr(q["gp"], name).dtype and rel_err(host(a), b) <= TOL[act], name
    assert rel_err(host(d["dstate"].conv), g["dfirst"]) <= TOL[act] and rel_err(host(d["dstate"].h), g["dh0"]) <= TOL[act]
    leaves = [t.clone().requires_grad_() for t in (q["gx"], *q["gstate"], *q["gp"])]
    o, st = ops.resonator_selective_layer(leaves[0], ops.SelectiveLayerParams(*leaves[3:]), G, state=ops.SelectiveState(*leaves[1:3]))
    grads = torch.autograd.grad((o, *st), leaves, (q["gdout"], *q["gdstate"]))
    for a, b in zip(grads, (d["dx"], *d["dstate"], *d["dp"])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_prefill_of_unequal_rows_then_tokens(path, act):
    """Rows of 0, 3 and 40 steps, then five tokens each, are the whole rows."""
    say(f"selective layer tokens {path} {act}")
    q = problem(act, 3, 45, 32, 4, 16, 1, 16, 4, 64, seed=2)
    lengths = torch.tensor([0, 3, 40], dtype=torch.int32, device="cuda")
    x, p = q["gx"], q["gp"]
    whole, end = ops.resonator_selective_layer_fwd(x, p, lengths=lengths + 5, return_state=True)
    pad = x.clone()
    for r, n in enumerate(lengths.tolist()):
        pad[r, n:] = 3.0
    _, s = ops.resonator_selective_layer_fwd(pad, p, lengths=lengths, return_state=True)
    for k in range(5):
        t = torch.stack([x[r, n + k] for r, n in enumerate(lengths.tolist())])
        y = ops.resonator_selective_layer_step(t, p, s)
        want = torch.stack([whole[r, n + k] for r, n in enumerate(lengths.tolist())])
        assert rel_err(host(y), host(want)) <= TOL[act]
    assert rel_err(host(s.conv), host(end.conv)) <= TOL[act] and rel_err(host(s.h), host(end.h)) <= TOL[act]


def test_written_tensors_count_as_changed(path):
    say(f"selective versions {path}")
    s = Scan("f32", 2, 20, 2, 4, 1, 4, seed=1)
    a, m = s.tensors(), s.more()
    h, y = m["h0"], torch.empty_like(a[0])
    was = [t._version for t in (h, y, a[0])]
    ops.resonator_selective_scan_fwd(*a, **m, out=y, h_out=h)
    assert [t._version for t in (h, y, a[0])] == [was[0] + 1, was[1] + 1, was[2]]
    tok = [t[:, 0].contiguous() for t in a[:4]]
    v = h._version
    ops.resonator_selective_scan_step(*tok, a[4], h)
    assert h._version == v + 1
    x, w = torch.randn(2, 9, 6, device="cuda"), torch.randn(6, 4, device="cuda")
    st, o = torch.randn(2, 3, 6, device="cuda"), torch.empty(2, 9, 6, device="cuda")
    v = st._version, o._version
    ops.resonator_short_conv_fwd(x, w, state=st, state_out=st, out=o)
    assert (st._version, o._version) == (v[0] + 1, v[1] + 1)
    ops.resonator_short_conv_step(x[:, 0], w, st)
    assert st._version == v[0] + 2
    z, t = torch.randn(3, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    r = ops.resonator_token_logprobs_fwd(z, t)
    v = z._version
    ops.resonator_token_logprobs_bwd(z, t, r, torch.ones(3, device="cuda"), out=z)
    assert z._version == v + 1
    leaf = torch.randn(3, 8, device="cuda", requires_grad=True)
    lp = ops.resonator_token_logprobs(leaf * 1.0, t)
    lp.sum().backward()
    assert leaf.grad.any()


def test_both_paths_are_one(monkeypatch):
    say("selective paths")
    q = problem("bf16", 2, 70, 32, 4, 16, 2, 16, 4, 64, seed=3)
    tok = torch.arange(140, device="cuda").view(2, 70) % 32
    tok[0, :3] = -1

    def run():
        o, s, saved = ops.resonator_selective_layer_fwd(q["gx"], q["gp"], 2, state=q["gstate"], return_state=True, save=True)
        d = ops.resonator_selective_layer_bwd(q["gx"], q["gp"], q["gdout"], saved, 2, state=q["gstate"], want_dstate=True)
        y = ops.resonator_selective_layer_step(q["gx"][:, 0].contiguous(), q["gp"], s, 2)
        r = ops.resonator_token_logprobs_fwd(o, tok, top=5, entropy=True, scale=0.7)
        dz = ops.resonator_token_logprobs_bwd(o, tok, r, torch.ones(2, 70, device="cuda"), torch.ones(2, 70, device="cuda"), scale=0.7)
        return [o, *s, *d["dp"], *d["dstate"], d["dx"], y, *r, dz]

    native = run()
    monkeypatch.setattr(ops, "_NATIVE", _Off())
    assert all(torch.equal(a, b) for a, b in zip(native, run()))


def example():
    d = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")
    sys.path.insert(0, d)
    try:
        spec = importlib.util.spec_from_file_location("selective_lm", os.path.join(d, "selective_lm.py"))
        m = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(m)
    finally:
        sys.path.remove(d)
    return m


@pytest.mark.parametrize("dtype,bits", [("bf16", 8), ("f32", 32)])
def test_model_trains_and_decodes(dtype, bits):
    """The example's steps run, every parameter has a finite gradient that is not zero, and decoding token by token goes on where a
    longer prompt's logits are."""
    E = example()
    say(f"selective model {dtype} {bits}")
    m = E.SelectiveLM(32, 64, 2, DT[dtype])
    losses = E.base.train(m, 3, B=4, L=40, bits=bits)
    assert len(losses) == 3 and all(np.isfinite(losses))
    t = E.base.sequences(4, 41, 32, 4, torch.Generator().manual_seed(3))
    loss = -ops.resonator_token_logprobs(m.logits(t[:, :-1]), t[:, 1:].contiguous()).mean()
    loss.backward()
    for group in m.groups:
        for p in group:
            assert torch.isfinite(p.grad).all() and p.grad.any()
    logits, _ = m.prefill(t)
    part, states = m.prefill(t[:, :30].contiguous())
    layers = m.damped()
    for k in range(30, 41):
        step = m.step(t[:, k], states, layers)
        assert rel_err(host(step), host(logits[:, k])) <= 2 * TOL[dtype]
    assert E.base.generate(m, t[:, :30].contiguous(), 5).shape == (4, 5)


def test_token_graph():
    """A model's token step, captured once: every replay is the eager step, with other work in between; two graphs share nothing."""
    E = example()
    say("selective token graph")
    m = E.SelectiveLM(32, 64, 2, torch.bfloat16)
    layers = m.damped()
    r = np.random.default_rng(0)
    tokens = torch.from_numpy(r.integers(0, 32, (6, 4))).cuda()
    _, s0 = m.prefill(tokens[:4].t().contiguous())
    copy = lambda ss: [ops.SelectiveState(s.conv.clone(), s.h.clone()) for s in ss]  # noqa: E731
    t = torch.zeros(4, dtype=torch.long, device="cuda")
    m.step(t, copy(s0), layers)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        states, side, graph = copy(s0), torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            out = m.step(t, states, layers)
        torch.cuda.synchronize()
        for h, s in zip(states, s0):
            h.conv.copy_(s.conv)
            h.h.copy_(s.h)
        graphs.append((graph, out, states))
    eager = copy(s0)
    for k in range(6):
        t.copy_(tokens[k])
        want = m.step(tokens[k], eager, layers)
        for graph, out, states in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for graph, out, states in graphs:
            assert torch.equal(out, want), k
            assert all(torch.equal(a.conv, b.conv) and torch.equal(a.h, b.h) for a, b in zip(states, eager)), k
