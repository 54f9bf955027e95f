"""More work than one launch takes (2^32 threads): the scan's tiles, the token step's elements, AdamW's chunks and the values of
its codes, the linear product's copies of operands and the sums of dy.  Each is compared with small calls on the same rows or
elements, or on those around the place where a launch ends, or with its definition.

The memory that a case needs is what the operator's own buffers take; a card that has not got it free skips the case.
"""
import gc

import pytest
import torch

from gpu_util import say

pytestmark = pytest.mark.gpu

ops = None


def setup_module(module):
    global ops
    from paper_2607_05583_amd import ops as _ops
    ops = _ops


@pytest.fixture
def room():
    """room(gigabytes): skips where the card has not got them free; what a case used is handed back after it."""
    def ask(gb):
        gc.collect()
        torch.cuda.empty_cache()
        free = torch.cuda.mem_get_info()[0] / 2 ** 30
        if free < gb:
            pytest.skip(f"{gb} GiB are needed, {free:.0f} are free")
    yield ask
    gc.collect()
    torch.cuda.empty_cache()


def normal(*shape, seed, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


@pytest.mark.parametrize("B,L", [((1 << 23) + 5, 1), ((1 << 22) + 3, 300)])
def test_scan_of_many_tiles(room, B, L):
    """2^23 chains of one step (one work-group of 512 threads each in the backward), 2^22 of two and three tiles."""
    room(70)
    say(f"scan of many tiles {B} {L}")
    x, r, i, dy = (normal(B, L, 1, seed=k) for k in range(4))
    gamma, h0, dh = torch.full((1,), 0.5, device="cuda"), normal(B, 1, seed=5, dtype=torch.float32), normal(B, 1, seed=6, dtype=torch.float32)
    lengths = torch.randint(0, L + 1, (B,), device="cuda", dtype=torch.int32)
    y, h, carry = ops.resonator_gated_scan_fwd(x, r, i, gamma, h0=h0, lengths=lengths, return_state=True, save=True)
    g = ops.resonator_gated_scan_bwd(x, r, i, gamma, dy, lengths=lengths, dh_out=dh, carry=carry, want_dh0=True)
    dgamma, off = 0.0, 0.0
    parts = 4
    cut = [B * k // parts for k in range(parts + 1)]
    for lo, hi in zip(cut, cut[1:]):  # (every row: each quarter is one launch)
        s = slice(lo, hi)
        a = [v[s] for v in (x, r, i)]
        y2, h2, c2 = ops.resonator_gated_scan_fwd(*a, gamma, h0=h0[s], lengths=lengths[s], return_state=True, save=True)
        assert torch.equal(y[s], y2) and torch.equal(h[s], h2) and torch.equal(carry[s], c2)
        g2 = ops.resonator_gated_scan_bwd(*a, gamma, dy[s], lengths=lengths[s], dh_out=dh[s], carry=c2, want_dh0=True)
        for k in ("dx", "dr", "di", "dh0"):
            assert torch.equal(g[k][s], g2[k]), k
        dgamma += g2["dgamma"].double()
        # (the same float32 sums of tiles added in float64: what is left is each result's rounding, 2^-24 of its size)
        off += 2.0 ** -24 * g2["dgamma"].abs().item()
    assert (g["dgamma"].double() - dgamma).abs().item() <= off + 2.0 ** -24 * dgamma.abs().item()


def test_token_step_of_many_elements(room):
    B, D = (1 << 21) + 3, 2048
    room(90)
    say(f"token step of many elements {B} {D}")
    x, r, i = (normal(B, D, seed=k) for k in range(3))
    gamma, h = torch.linspace(0.1, 1.0, D, device="cuda"), normal(B, D, seed=3, dtype=torch.float32)
    for s in (slice(0, 7), slice((1 << 21) - 5, B)):
        old = h[s].clone()
        want = ops.resonator_gated_scan_step(x[s], r[s], i[s], gamma, old)
        if s.start == 0:
            first = want, old
    y = ops.resonator_gated_scan_step(x, r, i, gamma, h)
    assert torch.equal(y[:7], first[0]) and torch.equal(h[:7], first[1])
    assert torch.equal(y[s], want) and torch.equal(h[s], old)


def test_adamw_of_many_elements(room):
    """2^34 elements are 2^24 chunks: around that place, the step and the values of its codes are a small tensor's."""
    n = (1 << 34) + 256 * 7 + 11
    room(185)
    say(f"adamw of many elements {n}")
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    at = (1 << 34) - 4096  # (a chunk's start, with the place where a launch ends behind it)
    p[at:], g[at:] = normal(n - at, seed=1), normal(n - at, seed=2)
    ps, gs = p[at:].clone(), g[at:].clone()
    st, ss = ops.adamw_state([p], bits=8, master=False), ops.adamw_state([ps], bits=8, master=False)
    ops.resonator_adamw_step([p], [g], st, step=1, lr=0.1)
    ops.resonator_adamw_step([ps], [gs], ss, step=1, lr=0.1)
    assert torch.equal(p[at:], ps) and not p[:1 << 20].any()
    for k in ("exp_avg", "exp_avg_sq"):
        assert torch.equal(st[k][at:], ss[k]), k
    for k in ("scale_avg", "scale_sq"):
        assert torch.equal(st[k][at // 256:], ss[k]), k
    del p, g
    torch.cuda.empty_cache()
    m, v = ops.resonator_adamw_values(st)
    m2, v2 = ops.resonator_adamw_values(ss)
    assert torch.equal(m[at:], m2) and torch.equal(v[at:], v2)


def test_linear_copy_of_many_elements(room):
    """An operand of 2^35 elements whose rows are not whole pieces is copied in more than one launch."""
    R, K, N = (1 << 15) + 9, (1 << 20) - 3, 8
    room(140)
    say(f"linear copy of many elements {R} {K}")
    x = torch.zeros(R, K, dtype=torch.bfloat16, device="cuda")
    rows = [0, 1, (1 << 15) - 1, 1 << 15, R - 1]
    for k, row in enumerate(rows):
        x[row] = normal(K, seed=k)
    W = normal(K, N, seed=9)
    y = ops.resonator_linear_fwd(x, W)
    xs = x[rows].double()
    want = xs @ W.double()
    # (2^-8 of the result for its rounding; K random terms in float32 add 2^-24 sqrt(K) / 2.4 of its size, 2.5e-5)
    assert (y[rows].double() - want).abs().max() <= 2.0 ** -8 * want.abs().max()
    rest = torch.ones(R, dtype=torch.bool, device="cuda")
    rest[rows] = False
    assert not y[rest].any()


def test_linear_column_sums_of_many_elements(room):
    """db of more rows than a launch takes (a work-group for 64 rows); whole numbers, whose sums are exact."""
    R, N = (1 << 30) + 64 * 3 + 5, 9
    room(90)
    say(f"linear column sums of many elements {R} {N}")
    dy = torch.zeros(R, N, dtype=torch.bfloat16, device="cuda")
    at = (1 << 30) - 64  # (where a launch ends)
    dy[at - 100:at + 100] = torch.randint(-3, 4, (200, N), device="cuda").bfloat16()
    dy[R - 70:] = 1.0
    want = dy[at - 100:at + 100].double().sum(0) + 70
    x, W = torch.zeros(R, 1, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, N, dtype=torch.bfloat16, device="cuda")
    g = ops.resonator_linear_bwd(x, W, dy, want_dx=False, want_dw=False, want_db=True)
    assert torch.equal(g["db"].double(), want)


def test_linear_zeros_of_many_elements(room):
    """The weight gradient of no rows: 2^32 and some zeros, one a thread."""
    K, N = (1 << 20) - 1, 4100
    room(40)
    say(f"linear zeros of many elements {K} {N}")
    W = torch.empty(K, N, dtype=torch.bfloat16, device="cuda")
    x, dy = torch.empty(0, K, dtype=torch.bfloat16, device="cuda"), torch.empty(0, N, dtype=torch.bfloat16, device="cuda")
    junk = torch.full((K, N), 3.0, dtype=torch.bfloat16, device="cuda")
    del junk  # (what the allocator hands out again)
    g = ops.resonator_linear_bwd(x, W, dy, want_dx=False)
    assert not g["dW"].any()
