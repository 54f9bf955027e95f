"""Calls of the linear product that are plain for a user and rare for the library: no rows at all with sizes that are not whole
16-byte pieces."""
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
