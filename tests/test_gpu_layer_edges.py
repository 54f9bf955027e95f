"""The gated recurrent layer's operators at their edges: offsets that 32 bits do not hold, codes of 8-bit states at the points
where their rounding turns, unaligned tensors, many tensors, other streams and graphs."""
import numpy as np
import pytest
import torch

from gpu_util import host, rel_err, say

pytestmark = pytest.mark.gpu

ops = None


def setup_module(module):
    global ops
    from paper_2607_05583_amd import ops as _ops
    ops = _ops


def far(shape, stride, dtype, seed):
    """A tensor whose rows lie far apart in a buffer of their own, and the same values close together."""
    n = sum((s - 1) * st for s, st in zip(shape, stride)) + 1
    t = torch.empty(n, dtype=dtype, device="cuda").as_strided(shape, stride)
    near = torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()
    t.copy_(near)
    return t, near


def test_scan_rows_beyond_32_bits():
    """A batch row that begins 2^32 bytes behind the first (and 2^31 elements): forward, backward and single tokens."""
    B, L, D = 2, 200, 72
    say("scan beyond 32 bits")
    ins = [far((B, L, D), ((1 << 31) + 8, 2 * D, 1), torch.bfloat16, k) for k in range(4)]
    gamma = torch.linspace(0.1, 1.5, D, device="cuda")
    x, r, i, dy = (t[0] for t in ins)
    cx, cr, ci, cdy = (t[1] for t in ins)
    y, carry = ops.resonator_gated_scan_fwd(x, r, i, gamma, save=True)
    y2, carry2 = ops.resonator_gated_scan_fwd(cx, cr, ci, gamma, save=True)
    assert torch.equal(y, y2) and torch.equal(carry, carry2)
    g2 = ops.resonator_gated_scan_bwd(cx, cr, ci, gamma, cdy, carry=carry2)
    out = (far((B, L, D), ((1 << 31) + 8, 2 * D, 1), torch.bfloat16, 9)[0], torch.empty_like(cx), torch.empty_like(cx))
    g = ops.resonator_gated_scan_bwd(x, r, i, gamma, dy, carry=carry, out=out)
    for k in ("dx", "dr", "di", "dgamma"):
        assert torch.equal(g[k], g2[k]), k
    h, h2 = torch.ones(B, D, device="cuda"), torch.ones(B, D, device="cuda")
    assert torch.equal(ops.resonator_gated_scan_step(x[:, 0], r[:, 0], i[:, 0], gamma, h),
                       ops.resonator_gated_scan_step(cx[:, 0], cr[:, 0], ci[:, 0], gamma, h2)) and torch.equal(h, h2)


def test_linear_outputs_beyond_32_bits():
    """More than 2^31 outputs: the last rows are what they are on their own."""
    R, K, N = (1 << 21) + 67, 64, 1024
    say("linear beyond 32 bits")
    gen = torch.Generator().manual_seed(1)
    base = torch.randn(1024, K, generator=gen).bfloat16().cuda()
    x = base.repeat(-(-R // 1024), 1)[:R].contiguous()
    W, b = (torch.randn(K, N, generator=gen) / 8).bfloat16().cuda(), torch.randn(N, generator=gen).cuda()
    y = ops.resonator_linear_fwd(x, W, b, act="silu")
    want = torch.nn.functional.silu(base.float() @ W.float() + b)
    for at in (0, (1 << 20) + 512, R - 100):
        got = y[at:at + 100].float()
        ref = want.repeat(2, 1)[at % 1024:at % 1024 + 100]
        assert rel_err(host(got), host(ref)) <= 2.0 ** -7, at  # (one rounding to bfloat16 and the float32 product's)


def test_adamw_beyond_32_bits():
    """A tensor of more than 2^31 elements: its last blocks are stepped as they are on their own."""
    n, tail = (1 << 31) + 256 * 5 + 77, 256 * 9 + 77
    say("adamw beyond 32 bits")
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator().manual_seed(2)
    p[n - tail:], g[n - tail:] = torch.randn(tail, generator=gen).bfloat16().cuda(), torch.randn(tail, generator=gen).bfloat16().cuda()
    ps, gs = p[n - tail:].clone(), g[n - tail:].clone()
    st, ss = ops.adamw_state([p], bits=8, master=False), ops.adamw_state([ps], bits=8, master=False)
    ops.resonator_adamw_step([p], [g], st, step=1, lr=0.1)
    ops.resonator_adamw_step([ps], [gs], ss, step=1, lr=0.1)
    at = n - tail  # (a multiple of a block)
    assert at % 256 == 0 and torch.equal(p[at:], ps) and not p[:at].any()
    for k in ("exp_avg", "exp_avg_sq"):
        assert torch.equal(st[k][at:at + tail], ss[k][:tail]), k
    assert torch.equal(st["scale_avg"][at // 256:], ss["scale_avg"])


@pytest.mark.parametrize("scale", [1.0, 0.37, 3.1e-7])
def test_codes_where_their_rounding_turns(scale):
    """With betas of 0 the new states are g and g^2.  Values within a few units in the last place of the points between two
    codes get the codes of correctly rounded operations, bit for bit."""
    f32 = np.float32
    m = [(k + 0.5) / 127 for k in range(127)]
    v = [((k + 0.5) / 255) ** 2 for k in range(255)]
    g = []
    for point in (np.array(m) ** 2, np.array(v)):
        base = (point * scale).astype(f32)
        for ulps in range(-4, 5):
            g.append((base.view(np.int32) + ulps).view(f32))
    g = np.concatenate(g)
    g = g[(g > 0) & (g < scale)]
    blocks = []
    for k in range(0, g.size, 255):  # each block of 256 with the largest value in it
        part = g[k:k + 255]
        blocks.append(np.concatenate([part, np.zeros(255 - part.size, f32), [f32(scale)]]))
    g = np.concatenate(blocks).astype(f32)
    g[::2] *= -1
    say(f"codes {scale} {g.size}")
    p = torch.zeros(g.size, device="cuda")
    st = ops.adamw_state([p], bits=8)
    ops.resonator_adamw_step([p], [torch.from_numpy(g).cuda()], st, step=1, lr=0.1, betas=(0.0, 0.0))
    gb = g.reshape(-1, 256)
    sm = np.abs(gb).max(1)
    sq = gb * gb
    sv = sq.max(1)
    assert np.array_equal(st["scale_avg"].cpu().numpy(), sm) and np.array_equal(st["scale_sq"].cpu().numpy(), sv)
    one = f32(1)
    cm = np.rint(np.sqrt(np.abs(gb) * (one / sm)[:, None]) * f32(127)) * np.sign(gb)
    cv = np.rint(np.sqrt(np.sqrt(sq * (one / sv)[:, None])) * f32(255))
    cv = np.where((sq > 0) & (cv < 1), one, cv)
    assert cm.dtype == f32 and cv.dtype == f32
    assert np.array_equal(st["exp_avg"].cpu().numpy(), cm.astype(np.int8).reshape(-1))
    assert np.array_equal(st["exp_avg_sq"].cpu().numpy(), cv.astype(np.uint8).reshape(-1))


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_adamw_of_many_unaligned_tensors(bits, dtype):
    """150 tensors (three launches) one behind the other at any element, some empty: what aligned copies of them give."""
    r = np.random.default_rng(4)
    sizes = [int(v) for v in r.integers(0, 700, 150)]
    say(f"many tensors {bits} {dtype}")
    flat, fg = (torch.from_numpy(r.normal(size=sum(sizes) + 1).astype(np.float32)).to(dtype).cuda() for _ in range(2))
    at = np.cumsum([1] + sizes)
    p, g = ([f[a:a + n] for a, n in zip(at, sizes)] for f in (flat, fg))
    p2, g2 = [t.clone() for t in p], [t.clone() for t in g]
    first = flat[0].clone()
    st, st2 = ops.adamw_state(p, bits=bits), ops.adamw_state(p2, bits=bits)
    for step in (1, 2):
        ops.resonator_adamw_step(p, g, st, step=step, lr=0.01)
        ops.resonator_adamw_step(p2, g2, st2, step=step, lr=0.01)
    assert torch.equal(flat[0], first)
    for a, b in zip(p, p2):
        assert torch.equal(a, b)
    for k in st:
        assert torch.equal(st[k], st2[k]), k


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_on_another_stream_and_in_a_graph(bits):
    """The step is the captured one's every time (what depends on its number is fixed at the capture)."""
    r = np.random.default_rng(5)
    t = lambda n: torch.from_numpy(r.normal(size=n).astype(np.float32)).cuda()  # noqa: E731
    p, g, scale = [t(1000), t(77)], [t(1000), t(77)], torch.ones(1, device="cuda")
    say(f"adamw graph {bits}")
    ref_p, st = [v.clone() for v in p], ops.adamw_state(p, bits=bits)
    ref = ops.adamw_state(p, bits=bits)
    ops.resonator_adamw_step([v.clone() for v in p], g, ops.adamw_state(p, bits=bits), step=3, lr=0.01, grad_scale=scale)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        ops.resonator_adamw_step(p, g, st, step=3, lr=0.01, grad_scale=scale)
    for k in range(4):
        for v in g:
            v.copy_(t(v.numel()))
        scale.fill_(1.0 + k)
        graph.replay()
        ops.resonator_adamw_step(ref_p, g, ref, step=3, lr=0.01, grad_scale=scale)
        torch.cuda.synchronize()
        for a, b in zip(p, ref_p):
            assert torch.equal(a, b), k
        for name in st:
            assert torch.equal(st[name], ref[name]), (k, name)


@pytest.mark.parametrize("act", [torch.float32, torch.bfloat16])
def test_linear_in_a_graph(act):
    """Forward and backward (a cut sum, packed operands, computed gradients of the bias) captured once and replayed."""
    r = np.random.default_rng(6)
    t = lambda *s: torch.from_numpy(r.normal(size=s).astype(np.float32)).cuda()  # noqa: E731
    R, K, N = 700, 203, 96
    x, W, b, dy = t(R, K).to(act), (t(K, N) / 14).to(act), t(N), t(R, N).to(act)
    say(f"linear graph {act}")

    def both():
        y, saved = ops.resonator_linear_fwd(x, W, b, act="gelu_tanh", save=True)
        g = ops.resonator_linear_bwd(x, W, dy, pre=saved, act="gelu_tanh", want_db=True)
        return [y, g["dx"], g["dW"], g["db"]]

    both()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        out = both()
    for k in range(4):
        x.copy_(t(R, K))
        dy.copy_(t(R, N))
        graph.replay()
        want = both()
        torch.cuda.synchronize()
        for a, c in zip(out, want):
            assert torch.equal(a, c), k
