"""The example that trains a dense tower between two exchanges: it learns, and its gradients are those of the formulas."""
import os
import sys

import numpy as np
import pytest

from dense_util import drop_factor

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def _example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import dense_tower
    return dense_tower


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_tower_learns(dtype):
    losses = _example().run(steps=12, dtype=dtype, tables=4, batch=1024, dim=16, rate=0.5, report=lambda s: None)
    assert all(np.isfinite(losses)) and losses[-1] < 0.9 * losses[0], losses


def test_gradients_of_a_step():
    """f32 against the same tower in 64 bits: five layers of sums of up to 1024 terms, each off by no more than about
    1024 2^-24 of its terms' magnitudes, which for these random signs are some thirty times the sums: 1e-2 relative in the
    worst case, 1e-4 is asked for in the norm."""
    import torch
    ex = _example()
    rows, features, hidden, step = 300, 64, 48, 5
    t = ex.Tower(rows, features, hidden=hidden, dtype="f32", drop=0.25, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((rows, features), generator=g, device="cuda")
    d = torch.randn((rows, 1), generator=g, device="cuda")
    logit = t.forward(x, step).clone()
    dx = t.backward(x, d)
    w = [v.double().requires_grad_() for v in t.w]
    bias = [v.double().requires_grad_() for v in t.bias]
    xd = x.double().requires_grad_()
    f3 = torch.from_numpy(drop_factor(rows, hidden, 0.25, 3, step)).cuda()
    f4 = torch.from_numpy(drop_factor(rows, hidden, 0.25, 4, step)).cuda()
    h1 = torch.relu(xd @ w[0].t() + bias[0])
    z = h1 @ w[1].t()
    h2 = torch.nn.functional.silu(z[:, :2 * hidden]) * z[:, 2 * hidden:]
    h3 = torch.relu(h2 @ w[2].t() + bias[2]) * f3 + h1
    want = (h3 * f4) @ w[3].t() + bias[3]
    want.backward(d.double())

    def close(a, c):
        assert float((a.double() - c).norm()) <= 1e-4 * float(c.norm())

    close(logit, want.detach())
    close(dx, xd.grad)
    for i in range(4):
        close(t.dw[i], w[i].grad)
        if i != 1:
            close(t.dbias[i], bias[i].grad)
