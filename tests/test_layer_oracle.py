"""Pins of the gated recurrent layer's oracle (CPU): closed forms and differences."""
import numpy as np
import pytest

import oracle as O


def _scan_problem(seed, B=2, L=9, D=3):
    r = np.random.default_rng(seed)
    return dict(x=r.normal(size=(B, L, D)), r=r.normal(size=(B, L, D)), i=r.normal(size=(B, L, D)),
                gamma=np.exp(r.uniform(-3, 1, D)), h0=r.normal(size=(B, D)))


def test_scan_of_constant_gates_is_a_geometric_sum():
    B, L, D = 1, 12, 2
    gamma = np.array([0.3, 2.0])
    zero = np.zeros((B, L, D))
    y, h, _ = O.gated_scan_fwd(np.ones((B, L, D)), zero, zero, gamma)
    a = np.exp(-gamma / 2)  # sigmoid(0) = 1/2
    t = np.arange(1, L + 1)[:, None]
    want = np.sqrt(1 - a * a) * 0.5 * (1 - a ** t) / (1 - a)
    assert np.allclose(y[0], want, rtol=1e-13) and np.allclose(h[0], want[-1], rtol=1e-13)


def test_scan_closed_and_open_gates():
    p = _scan_problem(1)
    y, h, _ = O.gated_scan_fwd(p["x"], np.full_like(p["x"], -800.0), p["i"], p["gamma"], p["h0"])
    assert np.allclose(y, p["h0"][:, None], rtol=1e-12)  # a closed gate keeps the state
    y, _, _ = O.gated_scan_fwd(p["x"], np.full_like(p["x"], 800.0), np.full_like(p["x"], 800.0),
                               np.full(3, 60.0), p["h0"])
    assert np.allclose(y, p["x"], rtol=1e-12)  # full damping forgets all but the drive


def test_scan_lengths_and_split():
    p = _scan_problem(2)
    n = np.array([4, 0])
    y, h, _ = O.gated_scan_fwd(p["x"], p["r"], p["i"], p["gamma"], p["h0"], n)
    y4, h4, _ = O.gated_scan_fwd(p["x"][:, :4], p["r"][:, :4], p["i"][:, :4], p["gamma"], p["h0"])
    assert np.array_equal(y[0, :4], y4[0]) and np.all(y[0, 4:] == 0) and np.array_equal(h[0], h4[0])
    assert np.all(y[1] == 0) and np.array_equal(h[1], p["h0"][1])
    rest, hr, _ = O.gated_scan_fwd(p["x"][:, 4:], p["r"][:, 4:], p["i"][:, 4:], p["gamma"], h4)
    full, hf, _ = O.gated_scan_fwd(p["x"], p["r"], p["i"], p["gamma"], p["h0"])
    assert np.array_equal(full[:, 4:], rest) and np.array_equal(hf, hr)


@pytest.mark.parametrize("lengths", [None, [9, 5], [0, 9]])
def test_scan_backward_against_differences(lengths):
    p = _scan_problem(3)
    n = None if lengths is None else np.array(lengths)
    r = np.random.default_rng(4)
    dy, dh = r.normal(size=p["x"].shape), r.normal(size=p["h0"].shape)

    def loss(**q):
        y, h, _ = O.gated_scan_fwd(q["x"], q["r"], q["i"], q["gamma"], q["h0"], n)
        return np.sum(dy * y) + np.sum(dh * h)

    g = O.gated_scan_bwd(p["x"], p["r"], p["i"], p["gamma"], dy, p["h0"], n, dh)
    for name in p:
        got, eps = g["d" + name], 1e-6
        for k in np.ndindex(p[name].shape):
            hi, lo = dict(p), dict(p)
            hi[name], lo[name] = p[name].copy(), p[name].copy()
            hi[name][k] += eps
            lo[name][k] -= eps
            num = (loss(**hi) - loss(**lo)) / (2 * eps)
            assert abs(num - got[k]) <= 2e-8 * max(1.0, abs(num)), (name, k)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu_tanh"])
def test_linear_backward_against_differences(act):
    r = np.random.default_rng(7)
    p = dict(x=r.normal(size=(4, 3)), W=r.normal(size=(3, 5)), b=r.normal(size=5))
    dy, res = r.normal(size=(4, 5)), r.normal(size=(4, 3))
    g = O.linear_bwd(p["x"], p["W"], dy, p["b"], act)
    assert np.array_equal(O.linear_bwd(p["x"], p["W"], dy, p["b"], act, res)["dx"], g["dx"] + res)
    for name in p:
        for k in np.ndindex(p[name].shape):
            v = []
            for e in (1e-6, -1e-6):
                q = {n: a.copy() for n, a in p.items()}
                q[name][k] += e
                v.append(np.sum(dy * O.linear_fwd(q["x"], q["W"], q["b"], act)[0]))
            assert abs((v[0] - v[1]) / 2e-6 - g["d" + name][k]) <= 1e-7 * max(1.0, abs(g["d" + name][k]))


def test_activations_closed_forms():
    assert O.act_value(np.array([0.0]), "gelu_tanh")[0] == 0.0 and O.act_slope(np.array([0.0]), "gelu_tanh")[0] == 0.5
    assert abs(O.act_value(np.array([40.0]), "silu")[0] - 40.0) < 1e-14
    assert np.array_equal(O.act_value(np.array([-2.0, 3.0]), "relu"), [0.0, 3.0])


def test_adamw_first_step_and_decay():
    p, g = np.array([1.0, -2.0, 0.5]), np.array([0.3, -4.0, 0.0])
    z = np.zeros(3)
    q, m, v = O.adamw(p, g, z, z, 1, 0.1, (0.9, 0.99), 0.0 + 1e-300, 0.5)
    # the first step moves by lr against the gradient's sign, after the decay
    assert np.allclose(q, p * (1 - 0.05) - 0.1 * np.sign(g), rtol=1e-13)
    assert np.allclose(m, 0.1 * g) and np.allclose(v, 0.01 * g * g)


def test_adamw_codes():
    r = np.random.default_rng(5)
    v = np.concatenate([r.normal(size=256), np.zeros(256), 1e-35 * r.normal(size=256)])
    place, scale = O.adamw_encode(v, False)
    back = O.adamw_decode(np.rint(place), scale, False)
    big = np.abs(v[:256]).max()
    # half a code of the square-root grid: |sqrt(value) - sqrt(kept)| <= sqrt(big) / 254
    assert np.all(np.abs(np.sqrt(np.abs(v[:256])) - np.sqrt(np.abs(back[:256]))) <= np.sqrt(big) / 254 * (1 + 1e-12))
    assert np.all(back[256:] == 0)
    w = v[:256] ** 2
    place, scale = O.adamw_encode(w, True)
    assert np.all(np.rint(place)[w > 0] >= 1) and np.rint(place).max() == 255
