"""Calls of the linear product that are plain for a user and rare for the library: no rows at all with sizes that are not whole
16-byte pieces, rows far apart in memory, and an empty sum."""
import numpy as np
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
@pytest.mark.parametrize("fn", ["none", "silu"])
@pytest.mark.parametrize("K,N", [(7, 5), (7, 8), (8, 5), (203, 1), (1, 96)])
def test_no_rows(path, act, fn, K, N):
    """The gradients of the weights and of the bias are zero, whatever the sizes."""
    say(f"no rows {path} {act} {fn} {K} {N}")
    x, W = torch.empty(0, K, dtype=DT[act], device="cuda"), torch.ones(K, N, dtype=DT[act], device="cuda")
    b = torch.ones(N, device="cuda")
    y, saved = ops.resonator_linear_fwd(x, W, b, act=fn, save=True)
    assert y.shape == (0, N)
    g = ops.resonator_linear_bwd(x, W, y, pre=saved, act=fn, want_db=True)
    assert g["dx"].shape == (0, K) and g["dW"].shape == (K, N) and g["db"].shape == (N,)
    assert not g["dW"].any() and not g["db"].any()


@pytest.mark.parametrize("act,K", [("bf16", 256), ("f32", 256), ("bf16", 250)])
@pytest.mark.parametrize("apart", [(1 << 21) - 8, 1 << 21, (1 << 21) + 8, (1 << 28) + 8])
def test_rows_far_apart(path, act, K, apart):
    """The last token of every long row (`x[:, -1]`), and rows farther apart: what the same rows close together give."""
    say(f"rows far apart {path} {act} {K} {apart}")
    r = np.random.default_rng(K)
    t = lambda *s: torch.from_numpy(r.normal(size=s).astype(np.float32))  # noqa: E731
    near = t(4, K).to(DT[act]).cuda()
    far = torch.empty(3 * apart + K, dtype=DT[act], device="cuda").as_strided((4, K), (apart, 1))
    far.copy_(near)
    W, b, dy = (t(K, 96) / 16).to(DT[act]).cuda(), t(96).cuda(), t(4, 96).to(DT[act]).cuda()
    got, want = [], []
    for x, to in ((far, got), (near, want)):
        y, saved = ops.resonator_linear_fwd(x, W, b, act="gelu_tanh", save=True)
        g = ops.resonator_linear_bwd(x, W, dy, pre=saved, act="gelu_tanh", want_db=True)
        to += [y, g["dx"], g["dW"], g["db"]]
    for a, c in zip(got, want):
        assert torch.equal(a, c)


def test_last_tokens_of_long_rows():
    x = torch.randn(4, 8192, 256, device="cuda").bfloat16()
    W = torch.randn(256, 64, device="cuda").bfloat16()
    say("last tokens")
    assert x[:, -1].stride(0) == 1 << 21
    assert torch.equal(ops.resonator_linear_fwd(x[:, -1], W), ops.resonator_linear_fwd(x[:, -1].contiguous(), W))


def test_empty_sum_is_refused(path):
    x, W = torch.empty(4, 0, device="cuda"), torch.empty(0, 8, device="cuda")
    say(f"empty sum {path}")
    with pytest.raises(ValueError):
        ops.resonator_linear_fwd(x, W)
    with pytest.raises(ValueError):
        ops.resonator_linear_bwd(x, W, torch.empty(4, 8, device="cuda"))
