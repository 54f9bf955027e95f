"""The AdamW step with eps = 0: second moments below float32's normal range (gradients of about 1e-19) have a root, and the
step is what the definition makes of them.

Tolerance: m and v are taken as float32 operations give them (in their order, in NumPy), so what is left is the update's
square root, quotient and products, 10 x 2^-23 of the update, as for the other steps.
"""
import numpy as np
import pytest
import torch

from gpu_util import host, say

pytestmark = pytest.mark.gpu

LR, BETAS = 3e-3, (0.9, 0.95)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_small_second_moments(bits, dtype):
    from paper_2607_05583_amd import ops
    say(f"small second moments {bits} {dtype}")
    n = 1000
    g = torch.from_numpy((np.logspace(-21, -12, n) * np.where(np.arange(n) % 3 == 0, -1.0, 1.0)).astype(np.float32)).to(dtype).cuda()
    for lo in (0, 1):  # beside others in a lane's four, and with large ones between
        if lo:
            g[1::2] = 1.0
        p = [torch.zeros(n, device="cuda")]
        st = ops.adamw_state(p, bits=bits)
        ops.resonator_adamw_step(p, [g], st, step=1, lr=LR, betas=BETAS, eps=0.0, weight_decay=0.0)
        f32 = np.float32
        gr = host(g).astype(f32)
        m = (gr * f32(1 - BETAS[0])).astype(np.float64)
        v = ((gr * gr) * f32(1 - BETAS[1])).astype(np.float64)
        assert (v > 0).all() and (v < 2.0 ** -126).any()
        up = LR / (1 - BETAS[0]) * m / np.sqrt(v / (1 - BETAS[1]))
        assert np.all(np.abs(host(p[0]) + up) <= 10 * 2.0 ** -23 * np.abs(up))
