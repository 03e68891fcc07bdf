"""Windows and trees over the 8-bit cache at shapes that take each kernel in each role (test_q8_span_shapes.py holds the plan to that):
the prompt kernel's splits, whose records a merge joins, and, for every kernel, pages that no row sees. Tolerances as in
test_gpu_w_q8_window_tree.py."""

import numpy as np
import pytest
import q8_span_shapes as sh

from test_gpu_u_q8_cache import _filled, _rows
from test_gpu_w_q8_window_tree import _check_tree, _check_window, _drafts, _masks, _np, _parents, _tree, _window

pytestmark = pytest.mark.gpu


def _ids(shapes):
    return [s.name.replace(" ", "-") for s in shapes]


def _tree_inputs(s, dtype, seed):
    n = max(s.n)
    q, k, v = _drafts(seed, len(s.lens), s.H, s.Hq, n, dtype)
    visible = _masks([_parents(np.random.default_rng(seed + b), m, "any") for b, m in enumerate(s.n)], n)
    for b, m in enumerate(s.n):
        q[b, :, m:] = k[b, :, m:] = v[b, :, m:] = float("nan")
    return q, k, v, visible


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("s", sh.SPLIT_TREES, ids=_ids(sh.SPLIT_TREES))
def test_split_trees_of_the_prompt_kernel(fmt, dtype, s):
    c = _filled(len(s.lens), s.H, s.Hq, s.lens, 64, fmt, dtype, 191)
    q, k, v, visible = _tree_inputs(s, dtype, 192)
    out = _tree(c, s.lens, q, k, v, visible, s.n, s.window, s.sinks)
    _check_tree(c, out, s.lens, q, k, v, visible, s.n, fmt, dtype, f"split tree {fmt} {dtype} {s.name}", s.window, s.sinks,
                rows=np.array([0, 1, 18, 19, 36, 37, 63, 100, 128, 199, 255]))


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("s", sh.SPLIT_WINDOWS, ids=_ids(sh.SPLIT_WINDOWS))
def test_split_windows_of_the_prompt_kernel(fmt, dtype, s):
    c = _filled(len(s.lens), s.H, s.Hq, s.lens, 64, fmt, dtype, 193)
    q = _rows(194, len(s.lens), s.Hq, max(s.n) + 1, 128, dtype=dtype, scale=1.5)  # a row more than any sequence has
    for b, m in enumerate(s.n):
        q[b, :, m:] = float("nan")
    out = _window(c, s.lens, q, s.n, s.window, s.sinks)
    _check_window(c, out, s.lens, q, s.n, s.window, s.sinks, fmt, dtype, f"split window {fmt} {dtype} {s.name}",
                  rows=np.array([0, 1, 18, 19, 31, 32, 100, 199, 255, 256, 499, 511]))


def _hide(c, s, first_seen):
    """Fill the pages behind the sinks and before the first that some row of the slot sees with NaN scales and codes of 0x7f."""
    hidden = 0
    for b, at in enumerate(first_seen):
        for page in c["block_table"][b, -(-s.sinks // 64):max(at, 0) // 64].tolist():
            hidden += 1
            for f in ("k_scale", "v_scale"):
                c[f][0, page] = float("nan")
            for f in ("k_codes", "v_codes"):
                c[f][0, page] = 0x7f
    assert hidden >= 2


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("s", sh.HIDDEN_WINDOWS, ids=_ids(sh.HIDDEN_WINDOWS))
def test_windows_do_not_read_hidden_pages(fmt, s):
    c = _filled(len(s.lens), s.H, s.Hq, s.lens, 64, fmt, "fp16", 195)
    q = _rows(196, len(s.lens), s.Hq, max(s.n), 128)
    want = _np(_window(c, s.lens, q, s.n, s.window, s.sinks))
    _hide(c, s, [L - m + 1 - s.window for L, m in zip(s.lens, s.n)])
    assert np.isfinite(want).all() and np.array_equal(_np(_window(c, s.lens, q, s.n, s.window, s.sinks)), want)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("s", sh.HIDDEN_TREES, ids=_ids(sh.HIDDEN_TREES))
def test_trees_do_not_read_hidden_pages(fmt, s):
    c = _filled(len(s.lens), s.H, s.Hq, s.lens, 64, fmt, "fp16", 197)
    q, k, v, visible = _tree_inputs(s, "fp16", 198)
    want = _np(_tree(c, s.lens, q, k, v, visible, s.n, s.window, s.sinks))
    _hide(c, s, [L + 1 - s.window for L in s.lens])  # of a row that names one draft
    again = _np(_tree(c, s.lens, q, k, v, visible, s.n, s.window, s.sinks))
    assert np.isfinite(want).all() and np.array_equal(again, want)


def test_whole_attention_of_few_rows_accepts_the_small_workspace():
    """Up to 32 rows of a KV head the windows' calls ask for twice as much."""
    import torch

    import paper_2609_11582_amd as okvq
    small, lens, n = 512 * 16 * 528, [3000, 700], 8
    c = _filled(2, 2, 8, lens, 64, "int8", "fp16", 199)
    assert okvq.okvq_q8_workspace_bytes(c.dims, 3000, n) == 2 * small
    q, n_dev = _rows(200, 2, 8, n, 128).cuda(), torch.tensor([n, 5], dtype=torch.int32, device="cuda")
    outs = []
    for size in (small, 2 * small):
        ws = torch.full((small // 2 + 4096,), float("nan"), device="cuda")  # what lies behind `size` bytes is left alone
        outs.append(torch.zeros_like(q))
        okvq.okvq_q8_attention(c, 0, lens, q, [n, 5], n_dev, n, 128 ** -0.5, outs[-1], ws[:size // 4])
        assert bool(ws[small // 4:].isnan().all())
    assert torch.equal(*outs) and bool(torch.isfinite(outs[0]).all())
