"""The gated scan on views: the time axis first in memory, with the three inputs and their gradients as columns of one tensor.  What
comes out is, bit for bit, what comes out of the same values batch first and apart."""
import pytest
import torch

from gpu_util import say

pytestmark = pytest.mark.gpu

ops = None
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


class _Off:
    """Stands in for the native module: takes nothing, so the Python code runs."""

    def __getattr__(self, name):
        return lambda *a: None


def setup_module(module):
    global ops
    from paper_2607_05583_amd import ops as _ops
    ops = _ops


@pytest.fixture(params=["native", "python"])
def path(request, monkeypatch):
    monkeypatch.setattr(ops, "_NATIVE", ops._native() if request.param == "native" else _Off())
    return request.param


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,D", [(2, 2, 1), (3, 40, 64), (2, 700, 72), (1, 300, 24), (5, 1, 16), (4, 515, 33)])
def test_time_first(path, act, B, L, D):
    say(f"time first {path} {act} {B} {L} {D}")
    g = torch.Generator(device="cuda").manual_seed(L)
    t = lambda *s: torch.randn(s, generator=g, device="cuda").to(DT[act])  # noqa: E731
    p, dy = t(L, B, 3 * D).transpose(0, 1), t(L, B, D).transpose(0, 1)
    gamma = torch.linspace(0.05, 2.0, D, device="cuda")
    xri = p.split(D, dim=-1)
    y, carry = ops.resonator_gated_scan_fwd(*xri, gamma, save=True)
    dp = torch.empty(L, B, 3 * D, dtype=DT[act], device="cuda").transpose(0, 1)
    got = ops.resonator_gated_scan_bwd(*xri, gamma, dy, carry=carry, out=dp.split(D, dim=-1))
    apart = [v.contiguous() for v in xri]
    y2, carry2 = ops.resonator_gated_scan_fwd(*apart, gamma, save=True)
    want = ops.resonator_gated_scan_bwd(*apart, gamma, dy.contiguous(), carry=carry2)
    assert torch.equal(y, y2) and torch.equal(carry, carry2) and torch.equal(got["dgamma"], want["dgamma"])
    assert torch.equal(dp, torch.cat([want[k] for k in ("dx", "dr", "di")], dim=-1))


@pytest.mark.parametrize("B,L,D,shift", [(3, 40, 64, 63), (3, 40, 64, 1), (2, 2, 4, 3)])
def test_time_first_columns_that_meet_are_refused(path, B, L, D, shift):
    say(f"columns that meet {path} {B} {L} {D} {shift}")
    x = torch.randn(L, B, D, device="cuda").transpose(0, 1)
    gamma = torch.ones(D, device="cuda")
    dp = torch.empty(L, B, 3 * D, device="cuda").transpose(0, 1)
    _, carry = ops.resonator_gated_scan_fwd(x, x, x, gamma, save=True)
    out = dp[..., :D], dp[..., shift:shift + D], dp[..., 2 * D:]
    with pytest.raises(Exception, match="overlap"):
        ops.resonator_gated_scan_bwd(x, x, x, gamma, x, carry=carry, out=out)


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("B,D", [(1400, 512), (700, 1001)])
def test_one_step_of_many_rows_time_first(path, act, B, D):
    """One step, whose distance to a next one (2^21 elements and more) plays no part."""
    say(f"one step time first {path} {act} {B} {D}")
    p = torch.randn(1, B, 3 * D, device="cuda").to(DT[act]).transpose(0, 1)
    assert p.stride(1) > 1 << 21
    gamma, dy = torch.linspace(0.05, 2.0, D, device="cuda"), torch.randn(B, 1, D, device="cuda").to(DT[act])
    xri = p.split(D, dim=-1)
    y, carry = ops.resonator_gated_scan_fwd(*xri, gamma, save=True)
    dp = torch.full((1, B, 3 * D), 7.0, dtype=DT[act], device="cuda").transpose(0, 1)
    got = ops.resonator_gated_scan_bwd(*xri, gamma, dy, carry=carry, out=dp.split(D, dim=-1))
    apart = [v.contiguous() for v in xri]
    y2, carry2 = ops.resonator_gated_scan_fwd(*apart, gamma, save=True)
    want = ops.resonator_gated_scan_bwd(*apart, gamma, dy, carry=carry2)
    assert torch.equal(y, y2) and torch.equal(carry, carry2) and torch.equal(got["dgamma"], want["dgamma"])
    assert torch.equal(dp, torch.cat([want[k] for k in ("dx", "dr", "di")], dim=-1))
