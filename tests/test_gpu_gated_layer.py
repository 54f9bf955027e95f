"""The gated recurrent layer (projection, gated scan, output projection, MLP) forward, backward and for single tokens, and
a small model that trains and decodes with it.

Tolerances (largest error over max(|value|, rms)): the layer in float32 is four products of K <= 256 random terms and
a scan, each off by about 2^-24 sqrt(K) of its result's size, 1e-6, and a gradient passes through seven of them with slopes
of order one: 2e-4 holds a factor of twenty.  In bfloat16 about ten results on a gradient's way are rounded, each to
2^-9 of its size; ten independent ones at five standard deviations are 5 sqrt(10) 2^-9 / sqrt(3) = 1.8e-2, with a factor
of three for the slopes 6e-2.
"""
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle as O
from gpu_util import host, rel_err, say

pytestmark = pytest.mark.gpu

ops = None
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TOL = {"f32": 2e-4, "bf16": 6e-2}


def setup_module(module):
    global ops
    from paper_2607_05583_amd import ops as _ops
    ops = _ops


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_lm.py")
    spec = importlib.util.spec_from_file_location("gated_lm", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def problem(act, B, L, d, f, seed):
    r = np.random.default_rng(seed)

    def t(*s, scale=1.0):
        return torch.from_numpy((r.normal(size=s) * scale).astype(np.float32)).cuda()

    def w(k, n):
        return t(k, n, scale=k ** -0.5).to(DT[act])

    gamma = torch.from_numpy(r.uniform(0.05, 2.0, d).astype(np.float32)).cuda()
    p = ops.GatedLayerParams(w(d, 3 * d), t(3 * d), gamma, w(d, d), t(d), w(d, f), t(f), w(f, d), t(d))
    return dict(p=p, x=t(B, L, d).to(DT[act]), dout=t(B, L, d).to(DT[act]), h0=t(B, d), dh=t(B, d),
                lengths=torch.from_numpy(r.integers(0, L + 1, B).astype(np.int32)).cuda())


def plain(q, act, lengths):
    """(out, h, gradients) in 64 bits"""
    p = ops.GatedLayerParams(*(host(t) for t in q["p"]))
    x, h0, dout, dh = (host(q[k]) for k in ("x", "h0", "dout", "dh"))
    n = None if lengths is None else lengths.cpu().numpy()
    B, L, d = x.shape
    flat = lambda t: t.reshape(B * L, -1)  # noqa: E731
    u = O.linear_fwd(flat(x), p.Wp, p.bp)[0].reshape(B, L, 3 * d)
    parts = [u[..., k * d:(k + 1) * d] for k in range(3)]
    y, h = O.gated_scan_fwd(*parts, p.gamma, h0, n)[:2]
    z = O.linear_fwd(flat(y), p.Wo, p.bo, residual=flat(x))[0]
    m = O.linear_fwd(z, p.W1, p.b1, act)[0]
    out = O.linear_fwd(m, p.W2, p.b2, residual=z)[0]
    g2 = O.linear_bwd(m, p.W2, flat(dout), p.b2)
    g1 = O.linear_bwd(z, p.W1, g2["dx"], p.b1, act, residual=flat(dout))
    go = O.linear_bwd(flat(y), p.Wo, g1["dx"], p.bo)
    gs = O.gated_scan_bwd(*parts, p.gamma, go["dx"].reshape(B, L, d), h0, n, dh)
    gp = O.linear_bwd(flat(x), p.Wp, flat(np.concatenate([gs["dx"], gs["dr"], gs["di"]], -1)), p.bp, residual=g1["dx"])
    dp = ops.GatedLayerParams(gp["dW"], gp["db"], gs["dgamma"], go["dW"], go["db"], g1["dW"], g1["db"], g2["dW"], g2["db"])
    return out.reshape(B, L, d), h, gp["dx"].reshape(B, L, d), gs["dh0"], dp


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("fn", ["gelu_tanh", "relu"])
@pytest.mark.parametrize("B,L,d,f,ragged", [(2, 37, 24, 96, False), (3, 130, 40, 160, True), (1, 1, 8, 32, False),
                                            (5, 9, 7, 13, True), (1, 300, 64, 256, False)])
def test_layer(act, fn, B, L, d, f, ragged):
    q = problem(act, B, L, d, f, 100 * B + L)
    n = q["lengths"] if ragged else None
    say(f"layer {act} {fn} {B} {L} {d} {f} {ragged}")
    out, h, saved = ops.resonator_gated_layer_fwd(q["x"], q["p"], h0=q["h0"], lengths=n, act=fn, return_state=True, save=True)
    g = ops.resonator_gated_layer_bwd(q["x"], q["p"], q["dout"], saved, lengths=n, dh=q["dh"], act=fn, want_dh0=True)
    ro, rh, rdx, rdh0, rdp = plain(q, fn, n)
    assert rel_err(host(out), ro) <= TOL[act]
    assert rel_err(host(h), rh) <= TOL[act]
    if fn == "relu" and act == "bf16":
        return  # where pre is nearer to 0 than its rounding, the slope is the other of the two
    assert rel_err(host(g["dx"]), rdx) <= TOL[act]
    assert rel_err(host(g["dh0"]), rdh0) <= TOL[act]
    for name, a, b in zip(rdp._fields, g["dp"], rdp):
        assert rel_err(host(a), b) <= TOL[act], name


def test_layer_against_differences():
    """Along the gradient itself the loss changes by the gradient's length."""
    q = problem("f32", 2, 33, 24, 96, 3)
    say("differences")

    def loss(s, v):
        p = ops.GatedLayerParams(*(t + s * e for t, e in zip(q["p"], v[:9])))
        out, h = ops.resonator_gated_layer_fwd(q["x"] + s * v[9], p, h0=q["h0"] + s * v[10], return_state=True)
        return ((out.double() * q["dout"].double()).sum() + (h.double() * q["dh"].double()).sum()).item()

    saved = ops.resonator_gated_layer_fwd(q["x"], q["p"], h0=q["h0"], save=True)[1]
    g = ops.resonator_gated_layer_bwd(q["x"], q["p"], q["dout"], saved, dh=q["dh"], want_dh0=True)
    v = [*g["dp"], g["dx"], g["dh0"]]
    size = sum((t.double() ** 2).sum() for t in v).sqrt().item()
    v = [(t / size) for t in v]
    # (the third derivative's term is about (2^-6)^2 / 6 of the first; the sums' own rounding less than 1e-3 of it)
    step = 2.0 ** -6
    assert abs((loss(step, v) - loss(-step, v)) / (2 * step) - size) <= 5e-3 * size


def test_layer_autograd():
    """The autograd form is the two entries, bit for bit, and the state's gradient reaches h0."""
    q = problem("f32", 2, 21, 16, 64, 5)
    say("autograd")
    x, h0 = q["x"].clone().requires_grad_(), q["h0"].clone().requires_grad_()
    p = ops.GatedLayerParams(*(t.clone().requires_grad_() for t in q["p"]))
    out, h = ops.resonator_gated_layer(x, p, h0=h0, lengths=q["lengths"], act="silu")
    torch.autograd.backward([out, h], [q["dout"], q["dh"]])
    o2, h2, saved = ops.resonator_gated_layer_fwd(q["x"], q["p"], h0=q["h0"], lengths=q["lengths"], act="silu",
                                                  return_state=True, save=True)
    g = ops.resonator_gated_layer_bwd(q["x"], q["p"], q["dout"], saved, lengths=q["lengths"], dh=q["dh"], act="silu",
                                      want_dh0=True)
    assert torch.equal(out, o2) and torch.equal(h, h2)
    assert torch.equal(x.grad, g["dx"]) and torch.equal(h0.grad, g["dh0"])
    for a, b in zip(p, g["dp"]):
        assert torch.equal(a.grad, b)
    x.grad = None
    out, h = ops.resonator_gated_layer(x, p, h0=h0)
    h.sum().backward()  # the output has no gradient of its own
    assert torch.isfinite(x.grad).all()


@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_prefill_then_tokens(act):
    """Prefill of ragged rows, then single tokens: what one longer prefill of each row gives."""
    B, L, more, d = 3, 70, 6, 32
    q = problem(act, B, L + more, d, 4 * d, 11)
    lengths = torch.tensor([70, 1, 0], dtype=torch.int32, device="cuda")
    say(f"prefill and tokens {act}")
    whole = torch.zeros_like(q["x"])
    for b, n in enumerate(lengths.tolist()):  # (the row's tokens after its prompt follow it)
        whole[b, :n], whole[b, n:n + more] = q["x"][b, :n], q["x"][b, L:]
    all_n = (lengths + more).to(torch.int32)
    ref, href = ops.resonator_gated_layer_fwd(whole, q["p"], h0=q["h0"], lengths=all_n, return_state=True)
    _, h = ops.resonator_gated_layer_fwd(q["x"][:, :L].contiguous(), q["p"], h0=q["h0"], lengths=lengths, return_state=True)
    for k in range(more):
        y = ops.resonator_gated_layer_step(q["x"][:, L + k].contiguous(), q["p"], h)
        want = torch.stack([ref[b, n + k] for b, n in enumerate(lengths.tolist())])
        assert rel_err(host(y), host(want)) <= TOL[act]
    assert rel_err(host(h), host(href)) <= TOL[act]


def test_token_graph():
    """A model's token step, captured once: every replay is the eager step, with other work in between."""
    E = example()
    say("token graph")
    m = E.GatedLM(32, 64, 2, torch.bfloat16)
    layers = m.damped()
    r = np.random.default_rng(0)
    tokens = torch.from_numpy(r.integers(0, 32, (6, 4))).cuda()
    _, s0 = m.prefill(tokens[:4].t().contiguous())
    t, states = torch.zeros(4, dtype=torch.long, device="cuda"), [h.clone() for h in s0]
    m.step(t, [h.clone() for h in s0], layers)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        out = m.step(t, states, layers)
    torch.cuda.synchronize()
    for h, s in zip(states, s0):
        h.copy_(s)
    eager = [h.clone() for h in s0]
    for k in range(6):
        t.copy_(tokens[k])
        graph.replay()
        want = m.step(tokens[k], eager, layers)
        torch.cuda.synchronize()
        assert torch.equal(out, want), k
        for h, s in zip(states, eager):
            assert torch.equal(h, s), k


@pytest.mark.parametrize("dtype,bits", [("bf16", 32), ("bf16", 8), ("f32", 32), ("f32", 8)])
def test_model_learns(dtype, bits):
    """From log(32) = 3.47 the loss falls to what the first tokens of a sequence leave open, and decoding goes on right."""
    E = example()
    say(f"train {dtype} {bits}")
    m = E.GatedLM(32, 64, 2, DT[dtype])
    losses = E.train(m, 150, B=32, L=64, bits=bits)
    assert losses[0] > 2.5 and max(losses[-10:]) < 0.5, (losses[0], losses[-10:])
    t = E.sequences(16, 64, 32, 4, torch.Generator().manual_seed(2))
    assert (E.generate(m, t[:, :32], 32) == t[:, 32:]).float().mean().item() > 0.8


def test_workspace_status():
    """Calls that share a workspace leave its status word at zero."""
    q = problem("bf16", 2, 900, 64, 128, 1)
    say("status")
    ws = ops.gated_scan_workspace(torch.bfloat16, 2, 900, 64, "cuda")
    for _ in range(3):
        out, saved = ops.resonator_gated_layer_fwd(q["x"], q["p"], save=True, ws=ws)
        ops.resonator_gated_layer_bwd(q["x"], q["p"], q["dout"], saved, ws=ws)
    assert ops.resonator_fwd_status(ws) == 0 and torch.isfinite(out).all()


def test_sequences_without_tokens():
    """L = 0: the state passes through, and so does its gradient; the parameters' gradients are zero."""
    q = problem("f32", 2, 1, 16, 32, 2)
    x = q["x"][:, :0].contiguous()
    say("no tokens")
    out, h, saved = ops.resonator_gated_layer_fwd(x, q["p"], h0=q["h0"], return_state=True, save=True)
    g = ops.resonator_gated_layer_bwd(x, q["p"], torch.empty_like(x), saved, dh=q["dh"], want_dh0=True)
    assert out.shape == g["dx"].shape == x.shape
    assert torch.equal(h, q["h0"]) and torch.equal(g["dh0"], q["dh"])
    assert not any(v.any() for v in g["dp"])
