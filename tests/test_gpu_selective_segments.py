"""The selective scan where its segments have several chunks of 64 steps: enough rows for the chip leave few segments, or one.
Its calls over more work than one launch takes (2^32 threads), and over rows of more than 2^31 elements, with those of the other
operators beside it.  A card that has not got the memory free skips a large case."""
import gc

import numpy as np
import pytest
import torch

from paper_2607_05583_amd import ops

from gpu_util import say
from select_util import Scan, gpu, host, within
from test_gpu_selective import check_backward, check_forward

pytestmark = pytest.mark.gpu
ACTS = ["bf16", "f32"]


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


# segments of 3, 4 (one), 2 and 2 chunks; states of 16, 16, 128 and 16; the last has two row blocks a head
SIZES = [(130, 600, 4, 8, 1, 8), (520, 200, 1, 5, 1, 3), (260, 200, 1, 3, 1, 70), (40, 450, 2, 70, 2, 9)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("sizes", SIZES)
def test_several_chunks_a_segment(sizes, ragged, act):
    B, L = sizes[:2]
    say(f"selective segments {sizes} {ragged} {act}")
    lengths = None
    if ragged:
        r = np.random.default_rng(3)
        lengths = [int(v) for v in r.integers(0, L + 1, B)]
        lengths[:6] = [0, 1, 64, 65, L - 1, L]
    s = Scan(act, *sizes, seed=11, lengths=lengths, dt_at=-4.0)
    carry = check_forward(s)[2]
    check_backward(s, carry=carry)


def test_scan_of_more_rows_than_a_launch_takes(room):
    """A work-group of 256 threads each for 2^24 rows and some: all against the first row's result, which is the others' too."""
    B = (1 << 24) + 5
    room(8)
    say(f"selective scan of {B} rows")
    s = Scan("bf16", 1, 3, 1, 2, 1, 2, seed=5, h0=False)
    x, dt, b, c, gamma = s.tensors()
    wide = [v.expand(B, *v.shape[1:]) for v in (x, dt, b, c)]
    more = {k: v for k, v in s.more().items() if k in ("dt_bias", "skip")}
    y, h = ops.resonator_selective_scan_fwd(*wide, gamma, return_state=True, **more)
    one, h1 = ops.resonator_selective_scan_fwd(x, dt, b, c, gamma, return_state=True, **more)
    assert bool((y == one).all()) and bool((h == h1).all())
    out = ops.resonator_selective_scan_step(*(v[:, 0] for v in wide), gamma, torch.zeros_like(h), **more)
    assert bool((out == one[:, 0]).all())


def test_logprobs_of_more_rows_than_a_launch_takes(room):
    R, V = (1 << 24) + 7, 3
    room(8)
    say(f"logprobs of {R} rows")
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((R, V), generator=g, device="cuda").bfloat16()
    tok = torch.randint(0, V, (R,), generator=g, device="cuda")
    dl = torch.ones(R, device="cuda")
    o = ops.resonator_token_logprobs_fwd(x, tok, entropy=True, top=1)
    d = ops.resonator_token_logprobs_bwd(x, tok, o, dl)
    for k in (slice(0, 64), slice(R // 2, R // 2 + 64), slice((1 << 24) - 32, R)):  # (a row's result is its own)
        p = ops.resonator_token_logprobs_fwd(x[k], tok[k], entropy=True, top=1)
        for a, e in zip(o, p):
            assert torch.equal(a[k], e)
        assert torch.equal(d[k], ops.resonator_token_logprobs_bwd(x[k], tok[k], p, dl[k]))
    every = torch.logsumexp(x.double(), 1)
    # a row's log probability: three roundings of values up to about 10, and of sums of three terms
    off = (o.logp.double() - (x.double().gather(1, tok[:, None])[:, 0] - every)).abs().max()
    assert float(off) < 16 * 2.0 ** -23 * 4
    # its gradient: one rounding of at most 1 to bf16, and what p is off by
    p = torch.softmax(x.float(), 1)
    want = -p
    want.scatter_add_(1, tok[:, None], dl[:, None])
    assert float((d.float() - want).abs().max()) < 2.0 ** -8 + 2.0 ** -18


def test_convolution_of_more_rows_than_a_launch_takes(room):
    """2^32 threads and some, of two channels and one step each."""
    B, D = (1 << 25) + 3, 256
    room(40)
    say(f"short convolution of {B} rows")
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((1, 1, D), generator=g, device="cuda").bfloat16()
    w = torch.randn((D, 2), generator=g, device="cuda")
    wide = x.expand(B, 1, D)
    y = ops.resonator_short_conv_fwd(wide, w)
    one = ops.resonator_short_conv_fwd(x, w)
    for lo in range(0, B, 1 << 22):
        assert bool((y[lo:lo + (1 << 22)] == one).all())


def test_row_of_more_than_2_31_elements(room):
    """A row's last 4096 steps against a call that goes on from the state before them; their gradients, which nothing behind them
    adds to, too."""
    H, P, N, tail = 8, 64, 64, 4096
    L = (1 << 22) + 3 * 64 + 7
    room(60)
    say(f"selective scan of {L} x {H * P}")
    g = torch.Generator(device="cuda").manual_seed(3)
    u = torch.randn((1, L, H * P + 2 * N), generator=g, device="cuda", dtype=torch.bfloat16)
    x, b, c = u.split((H * P, N, N), dim=-1)
    x, b, c = x.unflatten(-1, (H, P)), b.unflatten(-1, (1, N)), c.unflatten(-1, (1, N))
    dt = torch.randn((1, L, H), generator=g, device="cuda", dtype=torch.bfloat16) - 3
    gamma = torch.linspace(0.5, 4, H, device="cuda")
    y, h, carry = ops.resonator_selective_scan_fwd(x, dt, b, c, gamma, return_state=True, save=True)
    dy = torch.randn((1, L, H, P), generator=g, device="cuda", dtype=torch.bfloat16)
    d = ops.resonator_selective_scan_bwd(x, dt, b, c, gamma, dy, carry=carry)
    cut = L - tail
    assert cut * H * P > 2 ** 31 - 2 ** 22
    _, mid = ops.resonator_selective_scan_fwd(x[:, :cut], dt[:, :cut], b[:, :cut], c[:, :cut], gamma, return_state=True)
    end = [v[:, cut:] for v in (x, dt, b, c)]
    y2, h2 = ops.resonator_selective_scan_fwd(*end, gamma, h0=mid, return_state=True)
    d2 = ops.resonator_selective_scan_bwd(*end, gamma, dy[:, cut:].contiguous(), h0=mid)

    def near(a, e, by):
        a, e = host(a), host(e)
        assert np.isfinite(a).all() and np.linalg.norm(a - e) <= by * np.linalg.norm(e), float(np.linalg.norm(a - e) / np.linalg.norm(e))

    # Two results in bf16 that are each off by a rounding (2^-8 at most) and a weight's of each term (2^-8 at most, of terms
    # whose signs are random) differ by 4 times that; float32 ones by the roundings of some thousand terms.
    near(h, h2, 2.0 ** -14)
    near(y[:, cut:], y2, 2.0 ** -6)
    for k in ("dx", "ddt", "db", "dc"):
        near(d[k][:, cut:], d2[k], 2.0 ** -6)
