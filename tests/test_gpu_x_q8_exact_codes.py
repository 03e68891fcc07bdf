"""Scores of queries far from mean zero against blocks of keys with one channel that dwarfs the others and that the queries do
not use: the block's scale is large, its other codes are small, and so are the scores. Every kernel that a window's or a tree's rows can
take has to form them from the codes themselves, inside oracle.q8.attention's bound, which goes with sum |q code| scale: a form that
carried an offset on the codes would be off by 2^-24 of offset scale |sum q| in every token of the block, 0.02 of a log2 unit at a mean
of 20 and a channel of 1000. The values' signs go with the kind of block, so that an error of one kind's scores moves every output."""

import numpy as np
import pytest

from test_gpu_u_q8_cache import _append, _new, _rows
from test_gpu_w_q8_window_tree import _check_tree, _check_window, _masks, _parents, _tree, _window

pytestmark = pytest.mark.gpu
UNUSED = 4  # channels that the queries do not use


def _cache(H, Hq, L, top, fmt, dtype, seed):
    """Odd blocks have a channel of +-top, a different one from block to block; values are +1 in them, -1 in the others."""
    import torch
    c = _new(1, H, Hq, [L], 64, fmt, dtype)
    g = torch.Generator().manual_seed(seed)
    k, v = 0.05 * torch.randn(1, H, L, 128, generator=g), 0.1 * torch.randn(1, H, L, 128, generator=g)
    t = torch.arange(L)
    odd = t // 32 % 2 == 1
    k[:, :, t[odd], (t[odd] // 64) % UNUSED] = top * (1 - 2.0 * (t[odd] % 2))
    v += torch.where(odd, 1.0, -1.0)[:, None]
    dt = torch.float16 if dtype == "fp16" else torch.bfloat16
    _append(c, 0, k.to(dt), v.to(dt), [0], [L])
    return c


def _queries(Hq, n, mean, dtype, seed):
    q = _rows(seed, 1, Hq, n, 128, dtype="fp16").float() + mean
    q[..., :UNUSED] = 0
    return q.to(_rows(0, 1, dtype=dtype).dtype)


SIZES = [(5.0, 100.0), (20.0, 1000.0), (-20.0, 1000.0)]


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16"), ("int8", "bf16"), ("e4m3", "fp16")])
@pytest.mark.parametrize("mean, top", SIZES)
@pytest.mark.parametrize("n", [1, 16])  # the split kernel, the wide one
def test_trees(fmt, dtype, mean, top, n):
    L, Hq = 20000, 16
    c, q = _cache(1, Hq, L, top, fmt, dtype, 181), _queries(Hq, n, mean, dtype, 182)
    kd, vd = _rows(183, 1, 1, n, 128, dtype=dtype, scale=0.05), _rows(184, 1, 1, n, 128, dtype=dtype)
    visible = _masks([_parents(np.random.default_rng(185), n, "any")], n)
    out = _tree(c, [L], q, kd, vd, visible, [n])
    _check_tree(c, out, [L], q, kd, vd, visible, [n], fmt, dtype, f"exact tree {fmt} {dtype} mean {mean} top {top} rows {n}",
                rows=np.array([0, 3, 4, 15]))


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16"), ("int8", "bf16"), ("e4m3", "fp16")])
@pytest.mark.parametrize("mean, top", SIZES)
@pytest.mark.parametrize("H, Hq, L, n, window", [(1, 16, 20000, 1, 15000), (1, 16, 20000, 20, 15000), (4, 28, 3000, 1200, 1500)])
def test_windows(fmt, dtype, mean, top, H, Hq, L, n, window):
    """one token, the wide kernel, the prompt kernel"""
    c, q = _cache(H, Hq, L, top, fmt, dtype, 186), _queries(Hq, n, mean, dtype, 187)
    out = _window(c, [L], q, [n], window, 5)
    _check_window(c, out, [L], q, [n], window, 5, fmt, dtype, f"exact window {fmt} {dtype} mean {mean} top {top} rows {n}",
                  rows=np.array([0, 3, 19, 600, n - 1]))
