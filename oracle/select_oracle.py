"""Float64 NumPy oracle of the selective layer's operators and of the token probabilities: the definitions, one step after the
other.  Shares no code with the GPU path."""
from __future__ import annotations

import numpy as np

from .layer_oracle import act_slope as _slope, act_value as _act


def conv_fwd(x, w, bias=None, act="silu", state=None, lengths=None):
    """(y [B, L, D], the K - 1 inputs before each row's end)."""
    B, L, D = x.shape
    K = w.shape[1]
    y, last = np.zeros((B, L, D)), np.zeros((B, K - 1, D))
    for r in range(B):
        n = L if lengths is None else int(np.clip(lengths[r], 0, L))
        u = np.concatenate([np.zeros((K - 1, D)) if state is None else state[r], x[r, :n]])
        last[r] = u[n:]
        for t in range(n):
            pre = sum(w[:, k] * u[t + K - 1 - k] for k in range(K))
            y[r, t] = _act(pre if bias is None else pre + bias, act)
    return y, last


def conv_bwd(x, w, dy, bias=None, act="silu", state=None, lengths=None, dlast=None):
    """(dx, dw, dbias, dstate) of sum(dy y) + sum(dlast last)."""
    B, L, D = x.shape
    K = w.shape[1]
    dx, dw, db, ds = np.zeros((B, L, D)), np.zeros((D, K)), np.zeros(D), np.zeros((B, K - 1, D))
    for r in range(B):
        n = L if lengths is None else int(np.clip(lengths[r], 0, L))
        u = np.concatenate([np.zeros((K - 1, D)) if state is None else state[r], x[r, :n]])
        du = np.zeros_like(u)
        if dlast is not None:
            du[n:] += dlast[r]
        for t in range(n):
            pre = sum(w[:, k] * u[t + K - 1 - k] for k in range(K))
            d = dy[r, t] * _slope(pre if bias is None else pre + bias, act)
            db += d
            for k in range(K):
                dw[:, k] += d * u[t + K - 1 - k]
                du[t + K - 1 - k] += d * w[:, k]
        ds[r], dx[r, :n] = du[:K - 1], du[K - 1:]
    return dx, dw, db, ds


def _steps(dt, bias, lengths):
    v = dt + (0.0 if bias is None else bias)
    inside = np.ones(dt.shape[:2], bool)
    if lengths is not None:
        inside = np.arange(dt.shape[1])[None, :] < np.asarray(lengths)[:, None]
    D = np.where(inside[..., None], np.logaddexp(0.0, np.where(inside[..., None], v, 0.0)), 0.0)
    with np.errstate(over="ignore"):
        slope = np.where(inside[..., None], 1.0 / (1.0 + np.exp(-np.where(inside[..., None], v, 0.0))), 0.0)
    return D, slope, inside


def _inside(inside, *ts):
    return [np.where(inside.reshape(inside.shape + (1,) * (t.ndim - 2)), t, 0.0) for t in ts]


def scan_fwd(x, dt, b, c, gamma, bias=None, skip=None, h0=None, lengths=None):
    """(y [B, L, H, P], states [L + 1, B, H, P, N]): the state before each step, and behind the last."""
    B, L, H, P = x.shape
    G, N = b.shape[2:]
    D, _, inside = _steps(dt, bias, lengths)
    x, b, c = _inside(inside, x, b, c)
    hs = np.zeros((L + 1, B, H, P, N))
    if h0 is not None:
        hs[0] = h0
    y = np.zeros((B, L, H, P))
    for t in range(L):
        bt, ct = (np.repeat(v[:, t], H // G, axis=1) for v in (b, c))
        a = np.exp(-gamma * D[:, t])
        hs[t + 1] = a[..., None, None] * hs[t] + (D[:, t, :, None] * x[:, t])[..., None] * bt[:, :, None, :]
        y[:, t] = np.einsum("bhpn,bhn->bhp", hs[t + 1], ct) + (0.0 if skip is None else skip[:, None] * x[:, t])
    return _inside(inside, y)[0], hs


def scan_bwd(x, dt, b, c, gamma, dy, bias=None, skip=None, h0=None, lengths=None, dh=None):
    """dict: dx, ddt, db, dc, dgamma, ddt_bias, dskip, dh0 of sum(dy y) + sum(dh last state), and gs [L, B, H, P, N]: the
    gradient of the state behind each step from later ones."""
    B, L, H, P = x.shape
    G, N = b.shape[2:]
    D, slope, inside = _steps(dt, bias, lengths)
    _, hs = scan_fwd(x, dt, b, c, gamma, bias, skip, h0, lengths)
    x, b, c, dy = _inside(inside, x, b, c, dy)
    g = np.zeros((B, H, P, N)) if dh is None else np.array(dh, float)
    out = dict(dx=np.zeros(x.shape), ddt=np.zeros(D.shape), db=np.zeros(b.shape), dc=np.zeros(c.shape), dgamma=np.zeros(H),
               dskip=np.einsum("blhp,blhp->h", dy, x), gs=np.zeros((L, B, H, P, N)))
    for t in range(L - 1, -1, -1):
        bt, ct = (np.repeat(v[:, t], H // G, axis=1) for v in (b, c))
        out["gs"][t] = g
        out["dc"][:, t] = np.einsum("bhpn,bhp->bhn", hs[t + 1], dy[:, t]).reshape(B, G, H // G, N).sum(2)
        g = g + dy[:, t, ..., None] * ct[:, :, None, :]
        du = np.einsum("bhpn,bhn->bhp", g, bt)
        out["db"][:, t] = (D[:, t, :, None] * np.einsum("bhpn,bhp->bhn", g, x[:, t])).reshape(B, G, H // G, N).sum(2)
        out["dx"][:, t] = D[:, t, :, None] * du + (0.0 if skip is None else skip[:, None] * dy[:, t])
        a = np.exp(-gamma * D[:, t])
        dl = a * np.einsum("bhpn,bhpn->bh", g, hs[t])
        out["ddt"][:, t] = slope[:, t] * (np.einsum("bhp,bhp->bh", du, x[:, t]) - gamma * dl)
        out["dgamma"] -= (D[:, t] * dl).sum(0)
        g = a[..., None, None] * g
    for k in ("db", "dc"):
        out[k] = _inside(inside, out[k])[0]
    out["ddt_bias"], out["dh0"] = out["ddt"].sum((0, 1)), g
    return out


def logprobs(x, tokens, scale=1.0):
    """(logp [R], entropy [R], all log probabilities [R, V]): a row of -inf alone has log probabilities of -inf, entropy 0."""
    R, V = x.shape
    lp = np.full((R, V), -np.inf)
    logp, ent = np.zeros(R), np.zeros(R)
    for r in range(R):
        m = x[r].max()
        if m > -np.inf:
            e = np.exp(scale * (x[r] - m))
            with np.errstate(divide="ignore"):
                lp[r] = scale * (x[r] - m) - np.log(e.sum())
            p = e / e.sum()
            ent[r] = -(p[p > 0] * lp[r][p > 0]).sum()
        if tokens[r] >= 0:
            logp[r] = lp[r, tokens[r]] if tokens[r] < V else np.nan
    return logp, ent, lp


def logprobs_bwd(x, tokens, dlogp=None, dent=None, scale=1.0):
    """The logits' gradient [R, V]."""
    R, V = x.shape
    _, ent, lp = logprobs(x, np.where(tokens < V, tokens, 0), scale)
    out = np.zeros((R, V))
    for r in range(R):
        if not np.any(lp[r] > -np.inf):
            continue
        p = np.exp(lp[r])
        if dlogp is not None and tokens[r] >= 0:
            out[r] -= dlogp[r] * p
            if tokens[r] < V:
                out[r, tokens[r]] += dlogp[r]
            elif dlogp[r] != 0:
                out[r] = np.nan
        if dent is not None:
            out[r][p > 0] -= dent[r] * p[p > 0] * (lp[r][p > 0] + ent[r])
    return out * scale


def top(x, k):
    """The places of each row's k largest values, largest first, equal ones by the lowest place."""
    return np.argsort(-x, axis=-1, kind="stable")[:, :k]
