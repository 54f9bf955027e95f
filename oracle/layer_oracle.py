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
