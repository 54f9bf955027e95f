"""Performance cases of a selective layer's operators and of a language model's token probabilities.

Three operators make, train and serve a sequence mixer whose state is written and
read by the data, and score the tokens that a model over it predicts:

  short conv      y_t = act(sum_{k<K} w[k] x_{t-k} + bias), per channel; forward, backward and
                  one token from the inputs before it
  selective scan  D_t = softplus(dt_t + dt_bias), a_t = exp(-gamma D_t), per head a state [P, N]:
                  h_t = a_t h_{t-1} + D_t x_t b_t^T, y_t = h_t c_t + skip x_t; the heads of a group
                  share b and c; forward, backward and one token from a carried state
  token logprobs  with z = scale logits: z[token] - log sum exp z, the entropy of softmax(z), the
                  likeliest tokens with their log probabilities, and the logits' gradient

``listed()`` names the cases, ``draw(rng)`` gives one more of the same ranges,
``prepare`` / ``run`` are one pass, ``work`` what the pass cannot do without and
``exact`` the results in float64.  Where ``own`` is false ``run`` computes the
operators in elementary torch operations in float32, rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_ES = {"bf16": 2, "f32": 4}


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # A training step's convolution over the drive, b and c columns of a fused projection (eight heads of 64, one
        # group of 64 states) at the training benchmark's batch and length.
        dict(name="conv_train", kind="conv_train", act="bf16", B=8, L=8192, D=640, K=4, fn="silu", pad=8, state=False, ragged=False),
        # A float32 step over rows of unequal length, one of them empty, that continue earlier ones.
        dict(name="conv_train_ragged", kind="conv_train", act="f32", B=5, L=2001, D=203, K=3, fn="none", pad=0, state=True, ragged=True),
        # One token for each sequence of a decoding batch: latency counts.
        dict(name="conv_token", kind="conv_step", act="bf16", B=64, D=640, K=4, fn="silu", pad=8),
        # A selective layer of a training step at the training benchmark's batch and length.
        dict(name="selective_train", kind="selective_train", act="bf16", B=8, L=8192, H=8, P=64, G=1, N=64, fused=True, h0=False, ragged=False),
        # Prefill of a long context at the headline's batch and length, with wide states, for decoding from them.
        dict(name="selective_prefill", kind="selective_fwd", act="bf16", B=4, L=32768, H=8, P=64, G=1, N=128, fused=True, h0=False, ragged=False),
        # A float32 training step of odd sizes over rows of unequal length that continue a state.
        dict(name="selective_train_ragged", kind="selective_train", act="f32", B=5, L=2001, H=6, P=40, G=2, N=24, fused=False, h0=True, ragged=True),
        # One user's prompt in a wide model: few chains, a short time axis.
        dict(name="selective_prompt", kind="selective_fwd", act="bf16", B=1, L=777, H=32, P=64, G=2, N=128, fused=True, h0=False, ragged=False),
        # One token for each sequence of a decoding batch.
        dict(name="selective_token", kind="selective_step", act="bf16", B=64, H=8, P=64, G=1, N=64, fused=True),
        # The loss of a training step with its gradient: a word-piece vocabulary, some positions ignored.
        dict(name="logprobs_train", kind="logprobs_train", act="bf16", R=8192, V=50304, scale=1.0, entropy=False, masked=False, ignored=True, pad=0),
        # Scoring given continuations with a large vocabulary: log probabilities, entropy and twenty alternatives.
        dict(name="logprobs_score", kind="logprobs_fwd", act="bf16", R=2048, V=128000, top=20, scale=1.0, entropy=True, masked=False, ignored=False, pad=0),
        # What a server answers with for a decoding batch's tokens, at a temperature.
        dict(name="logprobs_token", kind="logprobs_fwd", act="bf16", R=64, V=50304, top=8, scale=0.8, entropy=True, masked=False, ignored=False, pad=0),
        # A float32 policy step (entropy in the loss) over an odd vocabulary whose forbidden tokens are masked.
        dict(name="logprobs_train_f32", kind="logprobs_train", act="f32", R=777, V=11573, scale=0.7, entropy=True, masked=True, ignored=True, pad=5),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], uniform in the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width of [lo, hi]: a multiple of 64, a multiple of 8, or any."""
    w, step = _log_int(rng, lo, hi), rng.choice((64, 64, 8, 1))
    return max(lo, w // step * step)


def draw(rng):
    kind = rng.choice(("conv_train", "conv_train", "conv_step", "selective_fwd", "selective_fwd", "selective_train",
                       "selective_train", "selective_step", "logprobs_fwd", "logprobs_fwd", "logprobs_train"))
    act = rng.choice(("bf16", "bf16", "f32"))
    yes = lambda p: rng.random() < p  # noqa: E731
    if kind.startswith("conv"):
        c = dict(kind=kind, act=act, D=_width(rng, 16, 4096), K=rng.choice((2, 3, 4, 4, 4, 7)),
                 fn=rng.choice(("silu", "silu", "none", "gelu_tanh")), pad=rng.choice((0, 0, 8, 3)))
        if kind == "conv_step":
            return dict(c, B=_log_int(rng, 1, 256))
        B = _log_int(rng, 1, 16)
        L = _log_int(rng, 1, max(1, min(32768, (1 << 24) // (B * c["D"]))))
        return dict(c, B=B, L=L, state=yes(0.4), ragged=yes(0.4))
    if kind.startswith("selective"):
        P, N, G = rng.choice((64, 64, 32, 128, 40)), rng.choice((64, 64, 128, 16, 24)), rng.choice((1, 1, 2))
        H = G * _log_int(rng, 1, 16)
        c = dict(kind=kind, act=act, H=H, P=P, G=G, N=N, fused=yes(0.6))
        if kind == "selective_step":
            return dict(c, B=_log_int(rng, 1, 128))
        B = _log_int(rng, 1, 8)
        L = _log_int(rng, 1, max(1, min(32768, (1 << (30 if act == "bf16" else 28)) // (B * H * P * N))))
        return dict(c, B=B, L=L, h0=yes(0.4), ragged=yes(0.4))
    V = _width(rng, 32, 131072)
    R = _log_int(rng, 1, max(1, min(32768, (1 << 26) // V)))
    c = dict(kind=kind, act=act, R=R, V=V, scale=rng.choice((1.0, 1.0, 0.7, 1.6)), entropy=yes(0.5), masked=yes(0.3),
             ignored=yes(0.4), pad=rng.choice((0, 0, 8, 3)))
    return dict(c, top=rng.choice((0, 1, 5, 20))) if kind == "logprobs_fwd" else c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, dt = case["kind"], _DT[case["act"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    def uniform(lo, hi, *shape):
        return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32) * (hi - lo) + lo

    def lengths(B, L):  # from none to all
        n = torch.randint(0, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        n[0] = L
        if B > 1:
            n[1] = 0
        return n, torch.arange(L, device="cuda")[None, :] >= n[:, None]

    t = {}
    if kind.startswith("conv"):
        B, D, K = case["B"], case["D"], case["K"]
        lead = (B,) if kind == "conv_step" else (B, case["L"])
        x = normal(*lead, D + case["pad"]).to(dt)
        if case.get("ragged"):  # what lies behind a row's end is not defined
            t["lengths"], behind = lengths(B, case["L"])
            x[behind] = float("nan")
        t["x"] = x[..., :D]
        t["w"], t["bias"] = uniform(-1, 1, D, K) / math.sqrt(K), 0.1 * normal(D)
        if kind == "conv_step" or case["state"]:
            t["state"] = normal(B, K - 1, D).to(dt)
        if kind == "conv_train":
            t["dy"], t["dstate"] = normal(*lead, D).to(dt), normal(B, K - 1, D).to(dt)
    elif kind.startswith("selective"):
        B, H, P, G, N = (case[k] for k in "BHPGN")
        lead = (B,) if kind == "selective_step" else (B, case["L"])
        p = normal(*lead, H * P + 2 * G * N + H)
        # the drive and what writes and reads the state are a convolution's outputs, the last columns the steps' logits
        u = p[..., :-H]
        u.copy_(u / (1 + torch.exp(-u)) * 1.5)
        p = p.to(dt)
        if case.get("ragged"):
            t["lengths"], behind = lengths(B, case["L"])
            p[behind] = float("nan")
        x, b, c, d = p.split((H * P, G * N, G * N, H), dim=-1)
        if not case["fused"]:
            x, b, c, d = (v.contiguous() for v in (x, b, c, d))
        t["x"], t["dt"] = x.unflatten(-1, (H, P)), d
        t["b"], t["c"] = b.unflatten(-1, (G, N)), c.unflatten(-1, (G, N))
        # steps of 1e-3 to 0.1 before the data move them, dampings of 1 to 16
        t["dt_bias"] = torch.log(torch.expm1(torch.exp(uniform(math.log(1e-3), math.log(0.1), H))))
        t["gamma"], t["skip"] = uniform(1.0, 16.0, H), 1.0 + 0.1 * normal(H)
        if kind == "selective_step" or case["h0"]:
            t["h"] = 0.3 * normal(B, H, P, N)
        if kind == "selective_train":
            t["dy"], t["dh"] = normal(*lead, H, P).to(dt), 0.1 * normal(B, H, P, N)
    else:
        R, V = case["R"], case["V"]
        x = normal(R, V + case["pad"])
        x = x.mul_(2.5).to(dt)
        tok = torch.randint(0, V, (R,), generator=g, device="cuda")
        if case["masked"]:  # forbidden tokens; in one row all but the given one
            x[:, :V].masked_fill_(torch.rand((R, V), generator=g, device="cuda") < 0.3, -math.inf)
            x[0, :V] = -math.inf
            x[torch.arange(R, device="cuda"), tok] = 1.0
        x[torch.arange(R, device="cuda"), tok] += uniform(0, 8, R).to(dt)  # a trained model's tokens are likely ones
        if case["ignored"]:
            tok = torch.where(torch.rand((R,), generator=g, device="cuda") < 0.1, -1, tok)
        t["logits"], t["tokens"] = x[:, :V], tok
        if kind == "logprobs_train":
            t["dlogp"] = -uniform(0.5, 1.5, R) / R
            if case["entropy"]:
                t["dent"] = 0.1 * normal(R) / R
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    st = {"case": dict(case), **t}
    kind = case["kind"]
    if kind == "conv_step":
        st["state_new"] = torch.empty_like(t["state"])
    if kind == "selective_step":
        st["h_new"] = torch.empty_like(t["h"])
    if kind == "selective_train":  # the fused projection's gradient, or one for each input
        B, L, H, P, G, N = (case[k] for k in "BLHPGN")
        cols = (H * P, G * N, G * N, H)
        dt = _DT[case["act"]]
        if case["fused"]:
            st["dp"] = torch.empty((B, L, sum(cols)), device="cuda", dtype=dt)
            dx, db, dc, dd = st["dp"].split(cols, dim=-1)
        else:
            dx, db, dc, dd = (torch.empty((B, L, n), device="cuda", dtype=dt) for n in cols)
        st["out"] = dx.unflatten(-1, (H, P)), dd, db.unflatten(-1, (G, N)), dc.unflatten(-1, (G, N))
    if own and kind in ("selective_fwd", "selective_train"):  # the workspace that a training or serving loop keeps
        from paper_2607_05583_amd import ops

        st["ws"] = ops.selective_scan_workspace(_DT[case["act"]], *(case[k] for k in "BLHPGN"), "cuda",
                                                backward=kind == "selective_train")
    return st


# ---------------------------------------------------------------------------
# plain forms: elementary operations in float32
# ---------------------------------------------------------------------------
def _act(v, fn):
    if fn == "silu":
        return v / (1.0 + torch.exp(-v))
    if fn == "gelu_tanh":
        return v / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    return v


def _leaves(*ts):
    return [None if v is None else v.detach().float().requires_grad_() for v in ts]


def _plain_conv(st):
    case, dt = st["case"], _DT[st["case"]["act"]]
    B, D, K, fn = case["B"], case["D"], case["K"], case["fn"]
    if case["kind"] == "conv_step":
        seen = torch.cat([st["state"], st["x"][:, None]], dim=1)
        y = (seen.flip(1).float() * st["w"].t()).sum(1) + st["bias"]
        return _act(y, fn).to(dt), seen[:, 1:].contiguous()
    L, n = case["L"], st.get("lengths")
    valid = None if n is None else (torch.arange(L, device="cuda")[None, :] < n[:, None])[..., None]
    x, w, bias, state = _leaves(st["x"] if valid is None else torch.where(valid, st["x"], 0), st["w"], st["bias"], st.get("state"))
    first = torch.zeros((B, K - 1, D), device="cuda") if state is None else state
    seen = torch.cat([first, x], dim=1)
    pre = bias
    for k in range(K):
        pre = pre + seen[:, K - 1 - k:K - 1 - k + L] * w[:, k]
    y = _act(pre, fn)
    if valid is not None:
        y = torch.where(valid, y, 0.0)
    if n is None:
        last = seen[:, L:]
    else:  # the K - 1 inputs before each row's end
        at = n[:, None].long() + torch.arange(K - 1, device="cuda")[None, :]
        last = seen.gather(1, at[..., None].expand(B, K - 1, D))
    loss = (y * st["dy"].float()).sum() + (last * st["dstate"].float()).sum()
    wrt = [x, w, bias] + ([state] if state is not None else [])
    dx, dw, db, *ds = torch.autograd.grad(loss, wrt)
    return (y.detach().to(dt), last.detach().to(dt), dx.to(dt), dw, db, *(v.to(dt) for v in ds))


_Q = 64  # steps of a chunk: within it the steps act on each other by products, across it by the state


def _plain_selective(x, d, b, c, gamma, dt_bias, skip, h0, valid):
    """(y, last state) in float32 from float32 inputs, differentiable."""
    B, L, H, P = x.shape
    G, N = b.shape[2:]
    n = -(-L // _Q)
    pad = n * _Q - L
    v = d + dt_bias
    step = torch.where(v > 0, v, 0.0) + torch.log1p(torch.exp(-v.abs()))
    if valid is not None:
        step = torch.where(valid[..., None], step, 0.0)

    def chunks(u):  # [B, L, heads, ...] to [B, chunk, head, step, ...]
        u = torch.cat([u, u.new_zeros((B, pad, *u.shape[2:]))], dim=1) if pad else u
        return u.reshape(B, n, _Q, *u.shape[2:]).transpose(2, 3)

    X, S, Bc, Cc = chunks(x), chunks(step), chunks(b), chunks(c)
    s = torch.cumsum(S.double() * gamma.double()[:, None], dim=-1)
    low = torch.ones((_Q, _Q), device=x.device, dtype=torch.bool).tril()
    E = torch.exp(-torch.where(low, s[..., :, None] - s[..., None, :], 1e4).float())
    each = H // G
    Bh, Ch = Bc.repeat_interleave(each, 2), Cc.repeat_interleave(each, 2)
    M = torch.matmul(Cc, Bc.transpose(-1, -2).contiguous()).repeat_interleave(each, 2) * E * S[..., None, :]
    Y = torch.matmul(M, X)
    total = s[..., -1:]
    W = X * (torch.exp(-(total - s)).float() * S)[..., None]
    add = torch.matmul(W.transpose(-1, -2).contiguous(), Bh)
    keep = torch.exp(-total).float()[..., None]
    h, before = h0, []
    for k in range(n):
        before.append(h)
        h = keep[:, k] * h + add[:, k]
    if n:
        before = torch.stack(before, dim=1)
        Y = Y + torch.matmul(Ch, before.transpose(-1, -2).contiguous()) * torch.exp(-s).float()[..., None]
    y = Y.transpose(2, 3).reshape(B, n * _Q, H, P)[:, :L] + skip[:, None] * x
    if valid is not None:
        y = torch.where(valid[..., None, None], y, 0.0)
    return y, h


def _plain_scan(st):
    case, dt = st["case"], _DT[st["case"]["act"]]
    B, H, P, G, N = (case[k] for k in "BHPGN")
    if case["kind"] == "selective_step":
        x, d, b, c = (st[k].float() for k in ("x", "dt", "b", "c"))
        b, c = (v.repeat_interleave(H // G, 1)[:, :, None, :] for v in (b, c))
        v = d + st["dt_bias"]
        step = torch.where(v > 0, v, 0.0) + torch.log1p(torch.exp(-v.abs()))
        h = torch.exp(-step * st["gamma"])[..., None, None] * st["h"] + (step[..., None] * x)[..., None] * b
        return ((h * c).sum(-1) + st["skip"][:, None] * x).to(dt), h
    L, n = case["L"], st.get("lengths")
    valid = None if n is None else torch.arange(L, device="cuda")[None, :] < n[:, None]
    data = [st["x"], st["dt"], st["b"], st["c"]]
    if valid is not None:
        data = [torch.where(valid.view(B, L, *[1] * (v.dim() - 2)), v, 0) for v in data]
    h0 = st["h"] if case["h0"] else torch.zeros((B, H, P, N), device="cuda")
    if case["kind"] == "selective_fwd":
        y, h = _plain_selective(*(v.float() for v in data), st["gamma"], st["dt_bias"], st["skip"], h0, valid)
        return y.to(dt), h
    wrt = _leaves(*data, st["gamma"], st["dt_bias"], st["skip"], h0)
    y, h = _plain_selective(*wrt, valid)
    loss = (y * st["dy"].float()).sum() + (h * st["dh"]).sum()
    dx, dd, db, dc, *params = torch.autograd.grad(loss, wrt)
    return (y.detach().to(dt), h.detach(), dx.to(dt), dd.to(dt), db.to(dt), dc.to(dt), *params)


def _plain_logprobs(st):
    case, dt = st["case"], _DT[st["case"]["act"]]
    z, tok = st["logits"].float() * case["scale"], st["tokens"]
    most = z.amax(-1, keepdim=True)
    off = z - most
    e = torch.exp(off)
    total = e.sum(-1, keepdim=True)
    logp_all = off - torch.log(total)
    given = tok >= 0
    at = torch.where(given, tok, 0)[:, None]
    logp = torch.where(given, logp_all.gather(-1, at)[:, 0], 0.0)
    p = e / total
    out = [logp]
    if case["entropy"]:
        ent = -(torch.where(p > 0, p * logp_all, 0.0)).sum(-1)
        out.append(ent)
    if case["kind"] == "logprobs_fwd":
        if case["top"]:
            place = torch.arange(case["V"], device="cuda")[None, :]
            x = st["logits"].float()  # (the scale is positive; its product may round two values to one)
            taken, ids, vals = torch.zeros_like(x, dtype=torch.bool), [], []
            for _ in range(case["top"]):  # the lowest place of the largest value left
                m = torch.where(taken, -math.inf, x).amax(-1, keepdim=True)
                i = torch.where((x == m) & ~taken, place, case["V"]).amin(-1, keepdim=True)
                ids.append(i)
                vals.append(logp_all.gather(-1, i))
                taken.scatter_(-1, i, True)
            out += [torch.cat(ids, -1), torch.cat(vals, -1)]
        return tuple(out)
    dlogp = torch.where(given, st["dlogp"], 0.0)[:, None]
    dz = -p * dlogp
    dz.scatter_add_(-1, at, dlogp)
    if case["entropy"]:
        dz -= torch.where(p > 0, p * (logp_all + ent[:, None]), 0.0) * st["dent"][:, None]
    return (*out, (dz * case["scale"]).to(dt))


def run(st):
    case, kind = st["case"], st["case"]["kind"]
    if not own:
        return (_plain_conv if kind.startswith("conv") else _plain_scan if kind.startswith("selective") else _plain_logprobs)(st)
    from paper_2607_05583_amd import ops

    if kind == "conv_step":
        y = ops.resonator_short_conv_step(st["x"], st["w"], st["state"], st["bias"], act=case["fn"], state_out=st["state_new"])
        return y, st["state_new"]
    if kind == "conv_train":
        y, last = ops.resonator_short_conv_fwd(st["x"], st["w"], st["bias"], act=case["fn"], state=st.get("state"),
                                               lengths=st.get("lengths"), return_state=True)
        d = ops.resonator_short_conv_bwd(st["x"], st["w"], st["dy"], st["bias"], act=case["fn"], state=st.get("state"),
                                         lengths=st.get("lengths"), dstate_out=st["dstate"], want_dstate=case["state"])
        return (y, last, d["dx"], d["dw"], d["dbias"]) + ((d["dstate"],) if case["state"] else ())
    data = [st.get(k) for k in ("x", "dt", "b", "c", "gamma")]
    if kind == "selective_step":
        y = ops.resonator_selective_scan_step(*data, st["h"], dt_bias=st["dt_bias"], skip=st["skip"], h_out=st["h_new"])
        return y, st["h_new"]
    if kind.startswith("selective"):
        more = dict(dt_bias=st["dt_bias"], skip=st["skip"], h0=st.get("h"), lengths=st.get("lengths"), ws=st["ws"])
        if kind == "selective_fwd":
            return ops.resonator_selective_scan_fwd(*data, return_state=True, **more)
        y, h, carry = ops.resonator_selective_scan_fwd(*data, return_state=True, save=True, **more)
        d = ops.resonator_selective_scan_bwd(*data, st["dy"], dh_out=st["dh"], carry=carry, want_dh0=True, out=st["out"], **more)
        return (y, h) + tuple(d[k] for k in ("dx", "ddt", "db", "dc", "dgamma", "ddt_bias", "dskip", "dh0"))
    r = ops.resonator_token_logprobs_fwd(st["logits"], st["tokens"], top=case.get("top", 0), entropy=case["entropy"], scale=case["scale"])
    out = (r.logp,) + ((r.entropy,) if case["entropy"] else ())
    if kind == "logprobs_fwd":
        return out + ((r.top_ids, r.top_logp) if case["top"] else ())
    return out + (ops.resonator_token_logprobs_bwd(st["logits"], st["tokens"], r, st["dlogp"], st.get("dent"), scale=case["scale"]),)


# ---------------------------------------------------------------------------
# what a pass cannot do without: each input read once and each output written
# once (what the forward keeps for the backward is neither); a transcendental
# counts as one operation.  The scan counts its definition's operations: per
# state element and step two for the decay and the write, two for the read,
# and twice as many and the gradients' sums in the backward.
# ---------------------------------------------------------------------------
def work(case):
    kind, e = case["kind"], _ES[case["act"]]
    if kind.startswith("conv"):
        B, D, K = case["B"], case["D"], case["K"]
        n, state, w = B * D * case.get("L", 1), B * (K - 1) * D * e, 4 * D * (K + 1)
        if kind == "conv_step":
            return {"bytes": 2 * n * e + 2 * state + w, "flops": n * (2 * K + 4)}
        return {"bytes": 4 * n * e + (4 if case["state"] else 2) * state + 2 * w, "flops": n * (8 * K + 12)}
    if kind.startswith("selective"):
        B, H, P, G, N = (case[k] for k in "BHPGN")
        t = B * case.get("L", 1)
        x, bc, d, state = t * H * P * e, t * 2 * G * N * e, t * H * e, 4 * B * H * P * N
        if kind == "selective_train":  # x, dy, dh in; y, h and the gradients out
            return {"bytes": 4 * x + 2 * bc + 2 * d + (4 if case["h0"] else 3) * state + 24 * H, "flops": 17 * t * H * P * N}
        had = 2 if kind == "selective_step" or case["h0"] else 1
        return {"bytes": 2 * x + bc + d + had * state + 12 * H, "flops": 5 * t * H * P * N}
    R, V = case["R"], case["V"]
    if kind == "logprobs_train":
        return {"bytes": 2 * R * V * e + R * (20 if case["entropy"] else 16), "flops": R * V * (12 if case["entropy"] else 8)}
    return {"bytes": R * V * e + R * (16 + 12 * case["top"]), "flops": R * V * (6 if case["entropy"] else 4)}


# ---------------------------------------------------------------------------
# float64 results, from the definitions: one step after the other
# ---------------------------------------------------------------------------
def _slope(fn, v):
    """The activation and its derivative."""
    if fn == "none":
        return v, torch.ones_like(v)
    if fn == "silu":
        q = torch.sigmoid(v)
        return v * q, q + v * q * (1 - q)
    c = math.sqrt(2 / math.pi)
    th = torch.tanh(c * (v + 0.044715 * v ** 3))
    return 0.5 * v * (1 + th), 0.5 * (1 + th) + 0.5 * v * (1 - th * th) * c * (1 + 3 * 0.044715 * v * v)


def _exact_conv(case, t):
    B, D, K, fn = case["B"], case["D"], case["K"], case["fn"]
    w, bias = t["w"].double(), t["bias"].double()
    if case["kind"] == "conv_step":
        pre = bias + w[:, 0] * t["x"].double()
        for k in range(1, K):
            pre = pre + w[:, k] * t["state"][:, K - 1 - k].double()
        return _slope(fn, pre)[0], torch.cat([t["state"][:, 1:], t["x"][:, None]], 1).double()
    L = case["L"]
    out = [torch.zeros((B, L, D), device="cuda", dtype=torch.float64), torch.zeros((B, K - 1, D), device="cuda", dtype=torch.float64)]
    dx, dstate = torch.zeros_like(out[0]), torch.zeros_like(out[1])
    dw, db = torch.zeros_like(w), torch.zeros_like(bias)
    for r in range(B):  # each row by itself: its earlier inputs, then its own, then nothing
        n = int(t["lengths"][r]) if case["ragged"] else L
        first = t["state"][r].double() if case["state"] else torch.zeros((K - 1, D), device="cuda", dtype=torch.float64)
        u = torch.cat([first, t["x"][r, :n].double()])
        pre = bias + sum(w[:, k] * u[K - 1 - k:K - 1 - k + n] for k in range(K))
        y, s = _slope(fn, pre)
        out[0][r, :n], out[1][r] = y, u[n:]
        d = t["dy"][r, :n].double() * s
        du = torch.zeros_like(u)
        du[n:] += t["dstate"][r].double()
        for k in range(K):
            du[K - 1 - k:K - 1 - k + n] += w[:, k] * d
            dw[:, k] += (d * u[K - 1 - k:K - 1 - k + n]).sum(0)
        db += d.sum(0)
        dstate[r], dx[r, :n] = du[:K - 1], du[K - 1:]
    return (*out, dx, dw, db) + ((dstate,) if case["state"] else ())


def _exact_scan(case, t):
    B, H, P, G, N = (case[k] for k in "BHPGN")
    one = case["kind"] == "selective_step"
    L = 1 if one else case["L"]
    f = lambda v: (v[:, None] if one else v).double()  # noqa: E731
    x, d, b, c = f(t["x"]), f(t["dt"]), f(t["b"]), f(t["c"])
    gamma, skip = t["gamma"].double(), t["skip"].double()
    each = H // G
    end = t["lengths"].long() if case.get("ragged") else torch.full((B,), L, device="cuda")
    inside = torch.arange(L, device="cuda")[None, :] < end[:, None]
    x, d, b, c = (torch.where(inside.view(B, L, *[1] * (v.dim() - 2)), v, 0.0) for v in (x, d, b, c))
    v = d + t["dt_bias"].double()
    step = torch.where(inside[..., None], torch.logaddexp(v, torch.zeros_like(v)), 0.0)
    a = torch.exp(-gamma * step)
    train = case["kind"] == "selective_train"
    h = t["h"].double() if "h" in t else torch.zeros((B, H, P, N), device="cuda", dtype=torch.float64)
    hs = torch.zeros((L + 1, B, H, P, N) if train else (1,), device="cuda", dtype=torch.float64)
    y = torch.zeros((B, L, H, P), device="cuda", dtype=torch.float64)
    if train:
        hs[0] = h
    for k in range(L):
        bk, ck = b[:, k].repeat_interleave(each, 1), c[:, k].repeat_interleave(each, 1)
        h = a[:, k, :, None, None] * h + (step[:, k, :, None] * x[:, k])[..., None] * bk[:, :, None, :]
        y[:, k] = (h * ck[:, :, None, :]).sum(-1)
        if train:
            hs[k + 1] = h
    y = torch.where(inside[..., None, None], y + skip[:, None] * x, 0.0)
    if one:
        return y[:, 0], h
    if not train:
        return y, h
    dy = torch.where(inside[..., None, None], t["dy"].double(), 0.0)
    g = t["dh"].double()
    dx, dstep, db, dc = torch.zeros_like(x), torch.zeros_like(step), torch.zeros_like(b), torch.zeros_like(c)
    dgamma = torch.zeros_like(gamma)
    for k in range(L - 1, -1, -1):
        bk, ck = b[:, k].repeat_interleave(each, 1), c[:, k].repeat_interleave(each, 1)
        dc[:, k] = (hs[k + 1] * dy[:, k, ..., None]).sum(2).view(B, G, each, N).sum(2)
        g = g + dy[:, k, ..., None] * ck[:, :, None, :]
        gb = (g * bk[:, :, None, :]).sum(-1)
        db[:, k] = (step[:, k, :, None] * (g * x[:, k, ..., None]).sum(2)).view(B, G, each, N).sum(2)
        dx[:, k] = step[:, k, :, None] * gb
        dlog = a[:, k] * (g * hs[k]).sum((-1, -2))
        dstep[:, k] = (gb * x[:, k]).sum(-1) - gamma * dlog
        dgamma -= (step[:, k] * dlog).sum(0)
        g = a[:, k, :, None, None] * g
    dx = torch.where(inside[..., None, None], dx + skip[:, None] * dy, 0.0)
    dd = torch.where(inside[..., None], dstep * torch.sigmoid(v), 0.0)
    db, dc = (torch.where(inside[..., None, None], u, 0.0) for u in (db, dc))
    return y, h, dx, dd, db, dc, dgamma, dd.sum((0, 1)), (dy * x).sum((0, 1, 3)), g


def _exact_logprobs(case, t):
    out = {"logp": [], "ent": [], "ids": [], "top": [], "dz": []}
    V, most = case["V"], max(1, (1 << 26) // case["V"])
    for r in range(0, case["R"], most):  # some rows at a time
        z = t["logits"][r:r + most].double() * case["scale"]
        tok = t["tokens"][r:r + most]
        logp = z - torch.logsumexp(z, -1, keepdim=True)
        given = tok >= 0
        hot = torch.zeros_like(z)
        hot[given.nonzero()[:, 0], tok[given]] = 1.0
        p = torch.exp(logp)
        out["logp"].append(torch.where(hot > 0, logp, 0.0).sum(-1))
        info = torch.where(p > 0, logp, 0.0)
        ent = -(p * info).sum(-1, keepdim=True)
        out["ent"].append(ent[:, 0])
        if case["kind"] == "logprobs_fwd" and case["top"]:  # equal values in the order of their places
            i = torch.sort(t["logits"][r:r + most].double(), dim=-1, descending=True, stable=True)[1]
            out["ids"].append(i[:, :case["top"]])
            out["top"].append(logp.gather(-1, i[:, :case["top"]]))
        if case["kind"] == "logprobs_train":
            dz = t["dlogp"][r:r + most, None].double() * given[:, None] * (hot - p)
            if case["entropy"]:
                dz = dz - t["dent"][r:r + most, None].double() * p * (info + ent)
            out["dz"].append(dz.mul_(case["scale"]).to(torch.float32) if case["act"] == "bf16" else dz * case["scale"])
    names = ["logp"] + (["ent"] if case["entropy"] else []) + ["ids", "top", "dz"]
    return tuple(torch.cat(out[k]) for k in names if out[k])


def exact(case, seed):
    t = _inputs(case, seed)
    kind = case["kind"]
    return (_exact_conv if kind.startswith("conv") else _exact_scan if kind.startswith("selective") else _exact_logprobs)(case, t)
