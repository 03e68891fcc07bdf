"""Head norms with rotary positions in float64 numpy: the formulas of include/okvq.h's okvq_norm_rotary and of its
gradient, with the absolute sizes from which the tests' tolerances are formed."""

from __future__ import annotations

import numpy as np

from .q8 import D, rotate


def _halves(adjacent):
    return (slice(0, D, 2), slice(1, D, 2)) if adjacent else (slice(0, 64), slice(64, D))


def pair_size(x, adjacent):
    """|a| + |b| of an element's pair (a, b), for both of them."""
    i, j = _halves(adjacent)
    out = np.empty_like(x)
    out[..., i] = out[..., j] = np.abs(x[..., i]) + np.abs(x[..., j])
    return out


def norm_rotate(x, w, eps, pos, inv_freq, axes, adjacent=False):
    """x [B][heads][n][128], w [128], pos [B][3][n] -> (y, size): an element is off by its rounding and a small part of size."""
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    return rotate(n, pos, inv_freq, axes, adjacent=adjacent), pair_size(n, adjacent)


def norm_rotate_grad(x, w, eps, pos, dy, inv_freq, axes, adjacent=False):
    """-> (dx, dx_size, dw, dw_size)"""
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    g = rotate(dy, pos, inv_freq, axes, inverse=True, adjacent=adjacent)
    size = pair_size(dy, adjacent)
    xn = x * r
    mean = (g * w * xn).mean(-1, keepdims=True)
    mean_size = (size * np.abs(w * xn)).mean(-1, keepdims=True)
    dx = r * (w * g - xn * mean)
    return dx, r * (np.abs(w) * size + np.abs(xn) * mean_size), (g * xn).sum((0, 1, 2)), (size * np.abs(xn)).sum((0, 1, 2))
