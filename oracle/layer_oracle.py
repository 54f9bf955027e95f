"""Float64 oracle of the gated recurrent layer: the gated scan, the linear product
with its epilogue and the AdamW step, straight from their definitions (NumPy).

Gated scan, per channel:
    s = gamma sigmoid(r_t), a = exp(-s), beta = sqrt(1 - a^2), q = sigmoid(i_t)
    h_t = a h_{t-1} + beta q x_t,  y_t = h_t  for t < lengths[b]; behind it y = 0, h stays.
"""
from __future__ import annotations

import numpy as np


def _sigmoid(v):
    return np.where(v >= 0, 1.0 / (1.0 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1.0 + np.exp(-np.abs(v))))


def gated_scan_fwd(x, r, i, gamma, h0=None, lengths=None):
    """(y [B, L, D], h [B, D], states [L + 1, B, D])"""
    B, L, D = x.shape
    end = np.full(B, L) if lengths is None else np.clip(lengths, 0, L)
    h = np.zeros((B, D)) if h0 is None else np.array(h0, dtype=np.float64)
    y, hs = np.zeros((B, L, D)), np.zeros((L + 1, B, D))
    hs[0] = h
    for t in range(L):
        for b in range(B):
            if t < end[b]:
                s = gamma * _sigmoid(r[b, t])
                h[b] = np.exp(-s) * h[b] + np.sqrt(-np.expm1(-2 * s)) * _sigmoid(i[b, t]) * x[b, t]
                y[b, t] = h[b]
        hs[t + 1] = h
    return y, h.copy(), hs


def gated_scan_bwd(x, r, i, gamma, dy, h0=None, lengths=None, dh=None):
    """dict of the gradients of sum(dy y) + sum(dh h_last)"""
    B, L, D = x.shape
    end = np.full(B, L) if lengths is None else np.clip(lengths, 0, L)
    hs = gated_scan_fwd(x, r, i, gamma, h0, lengths)[2]
    dx, dr, di, dg = np.zeros((B, L, D)), np.zeros((B, L, D)), np.zeros((B, L, D)), np.zeros(D)
    g = np.zeros((B, D)) if dh is None else np.array(dh, dtype=np.float64)
    for t in range(L - 1, -1, -1):
        for b in range(B):
            if t >= end[b]:
                continue
            sr, q = _sigmoid(r[b, t]), _sigmoid(i[b, t])
            s = gamma * sr
            a, beta = np.exp(-s), np.sqrt(-np.expm1(-2 * s))
            inv = np.divide(1.0, beta, out=np.zeros(D), where=beta > 0)
            gt = g[b] + dy[b, t]
            w = gt * (a * a * inv * q * x[b, t] - a * hs[t, b])
            dx[b, t] = gt * beta * q
            di[b, t] = gt * beta * q * (1 - q) * x[b, t]
            dr[b, t] = w * s * (1 - sr)
            dg += w * sr
            g[b] = a * gt
    return dict(dx=dx, dr=dr, di=di, dgamma=dg, dh0=g)


# ---------------------------------------------------------------------------
# linear product: y = act(x W + b) + residual
# ---------------------------------------------------------------------------
def act_value(v, act):
    if act == "relu":
        return np.maximum(v, 0.0)
    if act == "silu":
        return v * _sigmoid(v)
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (v + 0.044715 * v ** 3)))
    return v


def act_slope(v, act):
    if act == "relu":
        return (v > 0).astype(np.float64)
    if act == "silu":
        q = _sigmoid(v)
        return q * (1.0 + v * (1.0 - q))
    if act == "gelu_tanh":
        c = np.sqrt(2.0 / np.pi)
        th = np.tanh(c * (v + 0.044715 * v ** 3))
        return 0.5 * (1.0 + th) + 0.5 * v * (1.0 - th * th) * c * (1.0 + 3 * 0.044715 * v * v)
    return np.ones_like(v)


def linear_fwd(x, W, b=None, act="none", residual=None):
    """(y, pre)"""
    pre = x @ W + (0.0 if b is None else b)
    return act_value(pre, act) + (0.0 if residual is None else residual), pre


def linear_bwd(x, W, dy, b=None, act="none", residual=None, pre=None):
    """dict dx (plus residual), dW, db; pre is computed unless given"""
    pre = linear_fwd(x, W, b)[1] if pre is None else pre
    d = dy * act_slope(pre, act)
    return dict(dx=d @ W.T + (0.0 if residual is None else residual), dW=x.T @ d, db=d.sum(0))


# ---------------------------------------------------------------------------
# AdamW and its states in 8 bits (blocks of 256 elements with one scale)
# ---------------------------------------------------------------------------
def adamw(p, g, m, v, step, lr, betas, eps, weight_decay, scale=1.0):
    """(p, m, v) after one step"""
    g = g * scale
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    up = m / (1 - betas[0] ** step) / (np.sqrt(v / (1 - betas[1] ** step)) + eps)
    return p - lr * weight_decay * p - lr * up, m, v


def adamw_encode(v, positive):
    """(place of every value on its block's grid before rounding, scales): codes are the places rounded"""
    top, root = (255, 4) if positive else (127, 2)
    b = v.reshape(-1, 256)
    scale = np.abs(b).max(1)
    share = np.divide(np.abs(b), scale[:, None], out=np.zeros_like(b), where=scale[:, None] >= 1e-30)
    place = top * share ** (1.0 / root)
    if positive:
        place = np.where((place > 0) & (place < 1), 1.0, place)
    return (place * np.sign(b)).reshape(-1), scale


def adamw_decode(code, scale, positive):
    top, root = (255, 4) if positive else (127, 2)
    c = code.astype(np.float64).reshape(-1, 256) / top
    return (np.sign(c) * np.abs(c) ** root * scale[:, None]).reshape(-1)
