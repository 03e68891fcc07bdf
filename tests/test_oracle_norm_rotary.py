"""Pins of the head norm's oracle: rows of unit mean square, the rotation's and the weights' places, and the gradient
against automatic differentiation in 64 bits."""

import numpy as np
import pytest
import torch

from oracle import norm_rotary as nr
from oracle.q8 import rotate

FREQ = [1e4 ** (-i / 64) for i in range(64)]
AXES = [i % 3 for i in range(64)]


def _inputs(seed):
    rng = np.random.default_rng(seed)
    return rng.standard_normal((2, 3, 5, 128)) * 3, rng.uniform(0.2, 2, 128), rng.integers(-500, 500, (2, 3, 5)), rng.standard_normal((2, 3, 5, 128))


@pytest.mark.parametrize("adjacent", [False, True])
def test_norm(adjacent):
    x, w, pos, _ = _inputs(1)
    y, size = nr.norm_rotate(x, np.ones(128), 1e-12, pos, FREQ, AXES, adjacent)
    np.testing.assert_allclose((y * y).mean(-1), 1, rtol=1e-10)
    assert np.all(np.abs(y) <= size)
    y, _ = nr.norm_rotate(x, w, 0.5, pos * 0, FREQ, AXES, adjacent)
    np.testing.assert_allclose(y, w * x / np.sqrt((x ** 2).sum(-1, keepdims=True) / 128 + 0.5), rtol=1e-12)
    back = rotate(nr.norm_rotate(x, w, 0.5, pos, FREQ, AXES, adjacent)[0], pos, FREQ, AXES, inverse=True, adjacent=adjacent)
    np.testing.assert_allclose(back, y, atol=1e-12)


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("eps", [1e-6, 2.0])
def test_gradient(adjacent, eps):
    x, w, pos, up = _inputs(2)
    dx, dx_size, dw, dw_size = nr.norm_rotate_grad(x, w, eps, pos, up, FREQ, AXES, adjacent)
    xt, wt = torch.tensor(x, requires_grad=True), torch.tensor(w, requires_grad=True)
    n = xt * torch.rsqrt((xt * xt).mean(-1, keepdim=True) + eps) * wt
    i, j = nr._halves(adjacent)
    angle = torch.tensor(pos[:, AXES, :].transpose(0, 2, 1)[:, None] * np.array(FREQ))
    a, b = n[..., i], n[..., j]
    u = torch.tensor(up)
    loss = (u[..., i] * (a * angle.cos() - b * angle.sin()) + u[..., j] * (b * angle.cos() + a * angle.sin())).sum()
    gx, gw = torch.autograd.grad(loss, (xt, wt))
    np.testing.assert_allclose(dx, gx.numpy(), atol=1e-11)
    np.testing.assert_allclose(dw, gw.numpy(), atol=1e-10)
    assert np.all(np.abs(dx) <= dx_size * (1 + 1e-12)) and np.all(np.abs(dw) <= dw_size)
