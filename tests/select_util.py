"""Inputs and error bounds of the tests of the selective layer's operators.

Bounds are counted in roundings.  A rounding to bf16 is off by at most HALF["bf16"] = 2^-8 of the value, one to float32 by
2^-24.  Where an operator's terms cancel, the error is of the size of the sum of their absolute values, which is the same
operator on absolute values.
"""
import numpy as np
import torch

from oracle import select_oracle as O

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
TINY = 1e-30  # results that small may be flushed


def gpu(a, act=None):
    """A float64 array as a tensor of the activations' type (or float32)."""
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda", DT[act] if act else torch.float32)


def rounded(a, act):
    """What the activations' type holds of an array, in float64."""
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DT[act]).double().numpy()


def host(t):
    return t.detach().double().cpu().numpy()


def within(got, ref, bound, name):
    got = host(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    off = np.abs(got - ref) - (bound + TINY)
    assert np.all(np.isfinite(got)) and (off.size == 0 or off.max() <= 0), (
        name, float(np.nanmax(np.abs(got - ref) / (bound + TINY))), int(np.argmax(off)) if off.size else None)


class Scan:
    """Inputs of a selective scan, its exact results, and how far off an implementation in `act` may be."""

    def __init__(self, act, B, L, H, P, G, N, seed=0, h0=True, lengths=None, dt_at=-2.0, dt_width=1.0, bias=True, skip=True):
        r = np.random.default_rng(seed)
        self.act, self.sizes, self.lengths = act, (B, L, H, P, G, N), lengths
        n = lambda *s: r.standard_normal(s)  # noqa: E731
        self.x, self.b, self.c = rounded(n(B, L, H, P), act), rounded(n(B, L, G, N), act), rounded(n(B, L, G, N), act)
        self.dt, self.dy = rounded(dt_at + dt_width * n(B, L, H), act), rounded(n(B, L, H, P), act)
        f = lambda v: np.float32(v).astype(np.float64)  # noqa: E731
        self.gamma, self.bias, self.skip = f(np.exp(r.uniform(-3, 2, H))), f(n(H)) if bias else None, f(n(H)) if skip else None
        self.h0, self.dh = f(n(B, H, P, N)) if h0 else None, f(n(B, H, P, N)) if h0 else None
        data = self.x, self.dt, self.b, self.c, self.gamma
        more = dict(h0=self.h0, lengths=lengths)
        self.y, hs = O.scan_fwd(*data, self.bias, self.skip, **more)
        self.h = hs[-1]
        self.grads = O.scan_bwd(*data, self.dy, self.bias, self.skip, dh=self.dh, **more)
        self._bounds()

    def _bounds(self):
        B, L, H, P, G, N = self.sizes
        a = lambda v: None if v is None else np.abs(v)  # noqa: E731
        data = a(self.x), self.dt, a(self.b), a(self.c), self.gamma
        more = dict(h0=a(self.h0), lengths=self.lengths)
        y0, hs = O.scan_fwd(*data, self.bias, None, **more)
        y, _ = O.scan_fwd(*data, self.bias, a(self.skip), **more)
        g = O.scan_bwd(*data, a(self.dy), self.bias, a(self.skip), dh=a(self.dh), **more)
        g0 = O.scan_bwd(*data, a(self.dy), self.bias, None, dh=a(self.dh), **more)
        D, slope, inside = O._steps(self.dt, self.bias, self.lengths)
        x, dy = O._inside(inside, a(self.x), a(self.dy))
        # the decays' exponents are sums over a chunk's 64 steps (up to 512 each, base 2), each sum off by 2^-24 of itself
        ld = np.minimum(D * self.gamma * np.log2(np.e), 512.0)
        pad = np.zeros((B, -L % 64, H))
        most = np.concatenate([ld, pad], 1).reshape(B, -1, 64, H).sum(2).max() if L else 0.0
        # at most some thousand float32 roundings in a row: sums over 64 steps, 128 states or rows, over chunks, twice nested
        e = 2.0 ** -24 * (1024 + 4 * most)
        one = e + (2.0 ** -8 + 4 * 2.0 ** -16 if self.act == "bf16" else 0.0)  # and a weight of one bf16 part, states of two
        half = HALF[self.act]
        dl = np.zeros((B, L, H))
        if L:
            ry, cu = (dy * y0).sum(-1), (x * g0["dx"]).sum(-1)
            for t in range(L):
                end = min(L, t // 64 * 64 + 64)
                dl[:, t] = (ry[:, t:end] + cu[:, t:end]).sum(1) + np.einsum("bhpn,bhpn->bh", g["gs"][end - 1], hs[end])
        du_x = np.where(D > 0, (x * g0["dx"]).sum(-1) / np.where(D > 0, D, 1), 0)
        ddt = slope * (du_x + self.gamma * dl)
        self.bound = dict(
            y=half * np.abs(self.y) + one * y, h=e * hs[-1], dx=half * np.abs(self.grads["dx"]) + one * g["dx"],
            db=half * np.abs(self.grads["db"]) + one * g["db"], dc=half * np.abs(self.grads["dc"]) + one * g["dc"],
            ddt=half * np.abs(self.grads["ddt"]) + e * ddt, dgamma=e * (D * dl).sum((0, 1)), ddt_bias=e * ddt.sum((0, 1)),
            dskip=e * (x * dy).sum((0, 1, 3)), dh0=e * g["dh0"])

    def tensors(self, fused=False):
        """x, dt, b, c, gamma on the GPU; behind the rows' ends NaN; `fused`: columns of one tensor."""
        B, L, H, P, G, N = self.sizes
        x, dt, b, c = (gpu(v, self.act) for v in (self.x, self.dt, self.b, self.c))
        if self.lengths is not None:
            for r, n in enumerate(self.lengths):
                for v in (x, dt, b, c):
                    v[r, max(0, n):] = float("nan")
        if fused:
            u = torch.cat([x.flatten(2), b.flatten(2), c.flatten(2), dt, dt[..., :1]], dim=-1)
            x, b, c, dt, _ = u.split((H * P, G * N, G * N, H, 1), dim=-1)
            x, b, c = x.unflatten(-1, (H, P)), b.unflatten(-1, (G, N)), c.unflatten(-1, (G, N))
        return x, dt, b, c, gpu(self.gamma)

    def more(self):
        o = lambda v: None if v is None else gpu(v)  # noqa: E731
        n = None if self.lengths is None else torch.tensor(self.lengths, dtype=torch.int32, device="cuda")
        return dict(dt_bias=o(self.bias), skip=o(self.skip), h0=o(self.h0), lengths=n)
