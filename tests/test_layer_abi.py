"""Argument checks of the gated recurrent layer's C entry points that need no GPU: each bad argument is refused with its
status before any HIP call is made."""
import ctypes

import pytest

from paper_2607_05583_amd import _lib as L

BASE = 0x7F0000000000  # addresses that are never read: every call here is refused


def at(k, off=0):
    return ctypes.c_void_p(BASE + (k << 36) + off)


def rows(k, sb, st, off=0):
    return L.Rows(BASE + (k << 36) + off, sb, st)


def err():
    return L.lib().resonator_last_error().decode()


B, T, D = 2, 300, 64


def scan_fwd(**kw):
    a = dict(x=rows(1, T * D, D), r=rows(2, T * D, D), i=rows(3, T * D, D), dt=L.RES_F32, y=at(4), B=B, T=T, D=D, gamma=at(5),
             h0=None, lengths=None, h_out=None, carry=None, ws=at(6), wsb=1 << 30)
    a.update(kw)
    return L.lib().resonator_gated_scan_fwd(a["x"], a["r"], a["i"], a["dt"], a["y"], a["B"], a["T"], a["D"], a["gamma"], a["h0"],
                                            a["lengths"], a["h_out"], a["carry"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("bad,code", [
    (dict(dt=7), L.RES_ERR_INVALID_ARG), (dict(B=0), L.RES_ERR_INVALID_ARG), (dict(D=0), L.RES_ERR_INVALID_ARG),
    (dict(T=-1), L.RES_ERR_INVALID_ARG), (dict(T=1 << 31), L.RES_ERR_UNSUPPORTED), (dict(B=1 << 30), L.RES_ERR_UNSUPPORTED),
    (dict(x=L.Rows(None, T * D, D)), L.RES_ERR_INVALID_ARG), (dict(r=rows(2, T * D, D, 2)), L.RES_ERR_MISALIGNED),
    (dict(i=rows(3, -1, D)), L.RES_ERR_UNSUPPORTED), (dict(x=rows(1, T * D, 1 << 22)), L.RES_ERR_UNSUPPORTED),
    (dict(gamma=None), L.RES_ERR_INVALID_ARG), (dict(y=None), L.RES_ERR_INVALID_ARG), (dict(y=at(4, 2)), L.RES_ERR_MISALIGNED),
    (dict(lengths=at(7, 1)), L.RES_ERR_MISALIGNED), (dict(ws=None), L.RES_ERR_WORKSPACE), (dict(wsb=255), L.RES_ERR_WORKSPACE),
    (dict(ws=at(6, 16)), L.RES_ERR_MISALIGNED), (dict(y=at(1)), L.RES_ERR_INVALID_ARG), (dict(h_out=at(4)), L.RES_ERR_INVALID_ARG),
    (dict(h0=at(8), h_out=at(8, 4)), L.RES_ERR_INVALID_ARG), (dict(carry=at(5)), L.RES_ERR_INVALID_ARG),
])
def test_scan_forward(bad, code):
    assert scan_fwd(**bad) == code, err()


def test_scan_forward_workspace_is_the_size_that_is_asked_for():
    need = L.lib().resonator_gated_scan_workspace_bytes(L.RES_F32, B, T, D)
    assert need >= 256
    assert scan_fwd(wsb=need - 1) == L.RES_ERR_WORKSPACE
    assert L.lib().resonator_gated_scan_workspace_bytes(9, B, T, D) == 0
    assert L.lib().resonator_gated_scan_workspace_bytes(L.RES_F32, 0, T, D) == 0


def scan_bwd(**kw):
    # the gradients are the columns of one tensor [B, T, 3 D]
    a = dict(x=rows(1, T * D, D), r=rows(2, T * D, D), i=rows(3, T * D, D), dy=rows(4, T * D, D), dt=L.RES_F32,
             dx=rows(5, 3 * T * D, 3 * D), dr=rows(5, 3 * T * D, 3 * D, 4 * D), di=rows(5, 3 * T * D, 3 * D, 8 * D), gamma=at(6),
             carry=at(7), lengths=None, dh_out=None, dgamma=at(8), dh0=None, ws=at(9), wsb=1 << 30)
    a.update(kw)
    return L.lib().resonator_gated_scan_bwd(a["x"], a["r"], a["i"], a["dy"], a["dt"], a["dx"], a["dr"], a["di"], B, T, D, a["gamma"],
                                            a["carry"], a["lengths"], a["dh_out"], a["dgamma"], a["dh0"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("bad,code", [
    (dict(dy=L.Rows(None, 0, 0)), L.RES_ERR_INVALID_ARG), (dict(carry=None), L.RES_ERR_INVALID_ARG),
    (dict(dgamma=None), L.RES_ERR_INVALID_ARG), (dict(dgamma=at(8, 2)), L.RES_ERR_MISALIGNED),
    (dict(dx=rows(5, 3 * T * D, 3 * D, 4)), L.RES_ERR_INVALID_ARG),       # meets dr's first column
    (dict(dx=rows(1, T * D, D)), L.RES_ERR_INVALID_ARG),                  # over x
    (dict(dx=rows(10, T * D, D - 1)), L.RES_ERR_INVALID_ARG),             # rows that meet each other
    (dict(dh0=at(8)), L.RES_ERR_INVALID_ARG), (dict(ws=at(9, 8)), L.RES_ERR_MISALIGNED), (dict(wsb=0), L.RES_ERR_WORKSPACE),
])
def test_scan_backward(bad, code):
    assert scan_bwd(**bad) == code, err()


def test_scan_step():
    f = L.lib().resonator_gated_scan_step
    x, r, i = rows(1, D, 0), rows(2, D, 0), rows(3, D, 0)
    assert f(x, r, i, L.RES_BF16, None, B, D, at(5), at(6), at(6), None) == L.RES_ERR_INVALID_ARG
    assert f(x, r, i, L.RES_BF16, at(4), B, D, at(5), None, at(6), None) == L.RES_ERR_INVALID_ARG
    assert f(x, r, i, L.RES_BF16, at(4), B, D, at(5), at(6), at(6, 4), None) == L.RES_ERR_INVALID_ARG and "overlap" in err()
    assert f(x, r, i, L.RES_BF16, at(1), B, D, at(5), at(6), at(6), None) == L.RES_ERR_INVALID_ARG and "overlap" in err()
    assert f(x, r, i, L.RES_BF16, at(4, 1), B, D, at(5), at(6), at(6), None) == L.RES_ERR_MISALIGNED


R, K, N = 40, 72, 48


def lin_fwd(**kw):
    a = dict(x=at(1), ldx=K, W=at(2), dt=L.RES_F32, bias=at(3), act=0, res=None, y=at(4), pre=None, R=R, K=K, N=N, ws=None, wsb=0)
    a.update(kw)
    return L.lib().resonator_linear_fwd(a["x"], a["ldx"], a["W"], a["dt"], a["bias"], a["act"], a["res"], a["y"], a["pre"], a["R"],
                                        a["K"], a["N"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("bad,code", [
    (dict(dt=5), L.RES_ERR_INVALID_ARG), (dict(act=4), L.RES_ERR_INVALID_ARG), (dict(act=-1), L.RES_ERR_INVALID_ARG),
    (dict(K=0), L.RES_ERR_INVALID_ARG), (dict(N=0), L.RES_ERR_INVALID_ARG), (dict(R=-1), L.RES_ERR_INVALID_ARG),
    (dict(K=1 << 21, ldx=1 << 21), L.RES_ERR_UNSUPPORTED), (dict(W=None), L.RES_ERR_INVALID_ARG), (dict(x=None), L.RES_ERR_INVALID_ARG),
    (dict(y=None), L.RES_ERR_INVALID_ARG), (dict(ldx=K - 1), L.RES_ERR_INVALID_ARG), (dict(x=at(1, 2)), L.RES_ERR_MISALIGNED),
    (dict(bias=at(3, 2)), L.RES_ERR_MISALIGNED), (dict(y=at(1)), L.RES_ERR_INVALID_ARG), (dict(res=at(4, 4)), L.RES_ERR_INVALID_ARG),
    (dict(pre=at(4)), L.RES_ERR_INVALID_ARG), (dict(x=at(1, 4)), L.RES_ERR_WORKSPACE), (dict(ldx=K + 1), L.RES_ERR_WORKSPACE),
    (dict(x=at(1, 4), ws=at(5, 64), wsb=1 << 30), L.RES_ERR_MISALIGNED), (dict(x=at(1, 4), ws=at(2), wsb=1 << 30), L.RES_ERR_INVALID_ARG),
])
def test_linear_forward(bad, code):
    assert lin_fwd(**bad) == code, err()


def test_linear_without_rows_or_workspace():
    assert lin_fwd(R=0, x=None, y=None) == L.RES_OK  # nothing to do, nothing launched
    size = L.lib().resonator_linear_workspace_bytes
    assert size(0, L.RES_F32, 0, R, K, N, 0) == 0
    assert size(0, L.RES_F32, 0, R, K, N, 1) >= (R * K + K * N) * 4
    assert size(1, L.RES_BF16, 2, R, K, N, 0) > 0
    assert size(0, 7, 0, R, K, N, 0) == 0 and size(0, L.RES_F32, 9, R, K, N, 0) == 0


def lin_bwd(**kw):
    a = dict(x=at(1), ldx=K, W=at(2), dt=L.RES_F32, bias=at(3), dy=at(4), pre=at(5), act=2, res=None, dx=at(6), dW=at(7), db=at(8),
             ws=at(9), wsb=1 << 30)
    a.update(kw)
    return L.lib().resonator_linear_bwd(a["x"], a["ldx"], a["W"], a["dt"], a["bias"], a["dy"], a["pre"], a["act"], a["res"], a["dx"],
                                        a["dW"], a["db"], R, K, N, a["ws"], a["wsb"], None)


@pytest.mark.parametrize("bad,code", [
    (dict(dx=None, dW=None, db=None), L.RES_ERR_INVALID_ARG), (dict(dy=None), L.RES_ERR_INVALID_ARG),
    (dict(x=None), L.RES_ERR_INVALID_ARG), (dict(W=None), L.RES_ERR_INVALID_ARG), (dict(ldx=0), L.RES_ERR_INVALID_ARG),
    (dict(dx=None, dW=None, x=None, pre=None), L.RES_ERR_INVALID_ARG),  # pre has to be computed again, from x
    (dict(db=at(8, 2)), L.RES_ERR_MISALIGNED), (dict(dx=at(1)), L.RES_ERR_INVALID_ARG), (dict(dW=at(6)), L.RES_ERR_INVALID_ARG),
    (dict(res=at(6, 4)), L.RES_ERR_INVALID_ARG), (dict(ws=None), L.RES_ERR_WORKSPACE), (dict(ws=at(9, 4)), L.RES_ERR_MISALIGNED),
    (dict(ws=at(5)), L.RES_ERR_INVALID_ARG),
])
def test_linear_backward(bad, code):
    assert lin_bwd(**bad) == code, err()


def adamw(tensors=None, state=None, out=None, p_dt=L.RES_F32, lr=0.1, b1=0.9, b2=0.99, eps=1e-8, wd=0.0, step=1, scale=None):
    t = [(1, 2, 1, 100, 0)] if tensors is None else tensors
    table = (L.AdamWTensor * len(t))()
    for k, (p, g, o, n, s) in enumerate(t):
        addr = lambda v: None if v is None else BASE + (v << 36) if v < 1000 else v  # noqa: E731
        table[k] = L.AdamWTensor(addr(p), addr(g), addr(o), n, s)
    make = lambda s: L.AdamWState(*s)  # noqa: E731
    a = (32, at(10).value, at(11).value, None, None, None) if state is None else state
    b = a if out is None else out
    return L.lib().resonator_adamw_step(table, len(t), p_dt, L.RES_F32, ctypes.byref(make(a)), ctypes.byref(make(b)), lr, b1, b2, eps,
                                        wd, step, scale, None)


M, V = BASE + (10 << 36), BASE + (11 << 36)


@pytest.mark.parametrize("bad,code", [
    (dict(p_dt=6), L.RES_ERR_INVALID_ARG), (dict(lr=-0.1), L.RES_ERR_INVALID_ARG), (dict(lr=float("nan")), L.RES_ERR_INVALID_ARG),
    (dict(b1=1.0), L.RES_ERR_INVALID_ARG), (dict(b2=-0.1), L.RES_ERR_INVALID_ARG), (dict(eps=-1.0), L.RES_ERR_INVALID_ARG),
    (dict(wd=-1.0), L.RES_ERR_INVALID_ARG), (dict(step=0), L.RES_ERR_INVALID_ARG),
    (dict(tensors=[(1, 2, 1, -1, 0)]), L.RES_ERR_INVALID_ARG), (dict(tensors=[(1, 2, 1, 9, 128)]), L.RES_ERR_INVALID_ARG),
    (dict(tensors=[(None, 2, 1, 9, 0)]), L.RES_ERR_INVALID_ARG), (dict(tensors=[(1, 2, 2, 9, 0)]), L.RES_ERR_INVALID_ARG),
    (dict(tensors=[(1, 2, BASE + (1 << 36) + 4, 9, 0)]), L.RES_ERR_INVALID_ARG),
    (dict(tensors=[(1, BASE + (2 << 36) + 2, 1, 9, 0)]), L.RES_ERR_MISALIGNED),
    (dict(state=(16, M, V, None, None, None)), L.RES_ERR_INVALID_ARG), (dict(state=(8, M, V, None, None, None)), L.RES_ERR_INVALID_ARG),
    (dict(state=(32, M, None, None, None, None)), L.RES_ERR_INVALID_ARG),
    (dict(state=(32, M + 4, V, None, None, None)), L.RES_ERR_MISALIGNED),
    (dict(out=(8, M, V, M, V, None)), L.RES_ERR_INVALID_ARG),             # two kinds of state
    (dict(state=(32, M, V, None, None, M)), L.RES_ERR_INVALID_ARG),       # float32 parameters have no copy
    (dict(scale=at(3, 2)), L.RES_ERR_MISALIGNED),
])
def test_adamw(bad, code):
    assert adamw(**bad) == code, err()


def test_adamw_of_nothing_and_values():
    assert adamw(tensors=[(None, None, None, 0, 0)]) == L.RES_OK
    f = L.lib().resonator_adamw_values
    s8 = L.AdamWState(8, M, V, M + (1 << 30), V + (1 << 30), None)
    assert f(ctypes.byref(L.AdamWState(32, M, V, None, None, None)), 256, at(1), at(2), None) == L.RES_ERR_INVALID_ARG
    assert f(ctypes.byref(s8), 255, at(1), at(2), None) == L.RES_ERR_INVALID_ARG
    assert f(ctypes.byref(s8), 256, None, at(2), None) == L.RES_ERR_INVALID_ARG
    assert f(ctypes.byref(s8), 256, at(1, 4), at(2), None) == L.RES_ERR_MISALIGNED
    assert f(ctypes.byref(s8), 256, at(1), at(1, 256), None) == L.RES_ERR_INVALID_ARG
    assert f(ctypes.byref(s8), 0, None, None, None) == L.RES_OK
