"""Pins of the selective layer's oracle: closed forms, differences, planted mistakes."""
import numpy as np
import pytest

from oracle import select_oracle as O


def numeric(f, v, h=1e-6):
    g = np.zeros_like(v)
    for i in np.ndindex(v.shape):
        keep = v[i]
        v[i] = keep + h
        up = f()
        v[i] = keep - h
        g[i] = (up - f()) / (2 * h)
        v[i] = keep
    return g


@pytest.mark.parametrize("act", ["none", "silu", "gelu_tanh"])
def test_conv_gradients_are_differences(act):
    r = np.random.default_rng(1)
    B, L, D, K, lengths = 2, 5, 3, 3, np.array([5, 1])
    x, w, b, s = r.standard_normal((B, L, D)), r.standard_normal((D, K)), r.standard_normal(D), r.standard_normal((B, K - 1, D))
    dy, dl = r.standard_normal((B, L, D)), r.standard_normal((B, K - 1, D))

    def loss():
        y, last = O.conv_fwd(x, w, b, act, s, lengths)
        return (dy * y).sum() + (dl * last).sum()

    for got, v in zip(O.conv_bwd(x, w, dy, b, act, s, lengths, dl), (x, w, b, s)):
        np.testing.assert_allclose(got, numeric(loss, v), atol=1e-7)


def test_conv_is_numpys_convolution_and_goes_on_from_its_state():
    r = np.random.default_rng(2)
    x, w = r.standard_normal((1, 9, 2)), r.standard_normal((2, 4))
    y, _ = O.conv_fwd(x, w, act="none")
    for d in range(2):
        np.testing.assert_allclose(y[0, :, d], np.convolve(x[0, :, d], w[d])[:9], atol=1e-14)
    a, s = O.conv_fwd(x[:, :2], w, act="none")
    b, _ = O.conv_fwd(x[:, 2:], w, act="none", state=s)
    np.testing.assert_allclose(np.concatenate([a, b], 1), y, atol=1e-14)


def test_scan_gradients_are_differences():
    r = np.random.default_rng(3)
    B, L, H, P, G, N, lengths = 2, 4, 4, 2, 2, 3, np.array([4, 2])
    t = dict(x=r.standard_normal((B, L, H, P)), dt=r.standard_normal((B, L, H)), b=r.standard_normal((B, L, G, N)),
             c=r.standard_normal((B, L, G, N)), gamma=r.uniform(0.1, 2, H))
    bias, skip, h0 = r.standard_normal(H), r.standard_normal(H), r.standard_normal((B, H, P, N))
    dy, dh = r.standard_normal((B, L, H, P)), r.standard_normal((B, H, P, N))

    def loss():
        y, hs = O.scan_fwd(*t.values(), bias, skip, h0, lengths)
        return (dy * y).sum() + (dh * hs[-1]).sum()

    g = O.scan_bwd(*t.values(), dy, bias, skip, h0, lengths, dh)
    for name, v in dict(t, ddt_bias=bias, dskip=skip, dh0=h0).items():
        np.testing.assert_allclose(g[name if name in g else "d" + name], numeric(loss, v), atol=2e-7, err_msg=name)


def test_scan_closed_forms():
    # one state, steps of softplus(0) = ln 2 and gamma 1: a = 1/2; constant ones give a geometric sum
    L = 6
    one = np.ones((1, L, 1, 1))
    y, hs = O.scan_fwd(one, np.zeros((1, L, 1)), one, one, np.ones(1))
    np.testing.assert_allclose(y[0, :, 0, 0], np.log(2) * 2 * (1 - 0.5 ** np.arange(1, L + 1)), rtol=1e-14)
    # without damping the state is a sum of outer products, as a linear attention's
    r = np.random.default_rng(4)
    x, b, c = r.standard_normal((1, L, 2, 3)), r.standard_normal((1, L, 1, 5)), r.standard_normal((1, L, 1, 5))
    y, _ = O.scan_fwd(x, np.full((1, L, 2), np.log(np.e - 1)), b, c, np.zeros(2))  # steps of 1
    w = np.tril(c[0, :, 0] @ b[0, :, 0].T)
    np.testing.assert_allclose(y[0], np.einsum("ts,shp->thp", w, x[0]), atol=1e-12)


def test_scan_in_two_calls():
    r = np.random.default_rng(5)
    x, dt, b, c, g = (r.standard_normal((2, 7, 2, 3)), r.standard_normal((2, 7, 2)), r.standard_normal((2, 7, 1, 4)),
                      r.standard_normal((2, 7, 1, 4)), r.uniform(0.1, 2, 2))
    y, hs = O.scan_fwd(x, dt, b, c, g)
    y0, h0 = O.scan_fwd(x[:, :3], dt[:, :3], b[:, :3], c[:, :3], g)
    y1, h1 = O.scan_fwd(x[:, 3:], dt[:, 3:], b[:, 3:], c[:, 3:], g, h0=h0[-1])
    np.testing.assert_allclose(np.concatenate([y0, y1], 1), y, atol=1e-14)
    np.testing.assert_allclose(h1[-1], hs[-1], atol=1e-14)


def test_logprobs_gradient_is_differences():
    r = np.random.default_rng(6)
    x, tok = r.standard_normal((4, 7)), np.array([2, -1, 6, 0])
    x[3, 4] = -np.inf
    dl, de = r.standard_normal(4), r.standard_normal(4)

    def loss():
        a, b, _ = O.logprobs(x, tok, 0.7)
        return (dl * a + de * b).sum()

    keep = np.isfinite(x)
    got, want = O.logprobs_bwd(x, tok, dl, de, 0.7), np.zeros_like(x)
    for i in np.argwhere(keep):
        i = tuple(i)
        v = x[i]
        x[i] = v + 1e-6
        up = loss()
        x[i] = v - 1e-6
        want[i] = (up - loss()) / 2e-6
        x[i] = v
    np.testing.assert_allclose(got, want, atol=1e-8)
    np.testing.assert_allclose(got[[0, 2, 3]].sum(1), 0, atol=1e-14)  # shifting a row's logits changes nothing


def test_logprobs_closed_forms():
    lp, ent, every = O.logprobs(np.zeros((1, 8)), np.array([3]))
    assert np.isclose(lp[0], -np.log(8)) and np.isclose(ent[0], np.log(8)) and np.isclose(np.exp(every).sum(), 1)
    x = np.full((2, 4), -np.inf)
    x[0, 2] = 5.0
    lp, ent, _ = O.logprobs(x, np.array([2, 1]))
    assert lp[0] == 0 and lp[1] == -np.inf and not ent.any()
    assert not O.logprobs_bwd(x, np.array([2, 1]), np.ones(2), np.ones(2)).any()
    assert O.top(np.array([[1.0, 3.0, 3.0, -np.inf]]), 4).tolist() == [[1, 2, 0, 3]]


def test_planted_mistakes_are_seen():
    r = np.random.default_rng(7)
    x, dt, b, c, g = (r.standard_normal((1, 5, 2, 2)), r.standard_normal((1, 5, 2)), r.standard_normal((1, 5, 1, 3)),
                      r.standard_normal((1, 5, 1, 3)), r.uniform(0.5, 2, 2))
    y, hs = O.scan_fwd(x, dt, b, c, g)
    D = np.logaddexp(0, dt)
    late = np.einsum("bthpn,btn->bthp", hs[:-1].swapaxes(0, 1), c[:, :, 0])       # the state before the step is read
    undamped, _ = O.scan_fwd(x, dt, b, c, 0 * g)
    unscaled, _ = O.scan_fwd(x / D[..., None], dt, b, c, g)                       # the write without its step
    swapped, _ = O.scan_fwd(x, dt, c, b, g)
    for wrong in (late, undamped, unscaled, swapped):
        assert np.abs(wrong - y).max() > 1e-2
    dy = r.standard_normal(y.shape)
    right = O.scan_bwd(x, dt, b, c, g, dy)
    assert np.abs(O.scan_bwd(x, dt, b, c, g, dy[:, ::-1])["db"] - right["db"]).max() > 1e-2
