"""Window and tree attention over the paged 8-bit cache against float64 attention over the tokens that each row sees
(oracle.q8.window_seen, tree_seen), within the bound that oracle.q8.attention derives from the kernels' roundings: a mask
only removes terms from its sums, and the drafts' part, in fp32 from rows as they are, rounds less than the cache's."""

import math

import numpy as np
import pytest

from oracle import norm_rotary as nr
from oracle import q8 as oq
from test_gpu_u_q8_cache import HALF, SM, _append, _filled, _i32, _new, _numpy, _rows, _say

pytestmark = pytest.mark.gpu


def _np(x):
    return x.double().cpu().numpy()


def _worst(got, ref, bound):
    return float(np.nanmax(np.abs(got - ref) / np.maximum(bound, 1e-30))) if np.isfinite(got).all() else math.inf


def _window(c, lens, q, new, window, sinks, sm=SM, layer=0, fill=9.0, new_dev=None, ws=None, stream=None):
    import torch

    import paper_2609_11582_amd as okvq
    B, Hq, n, _ = q.shape
    out = torch.full((B, Hq, n, 128), fill, dtype=c.row_dtype, device="cuda")
    ws = okvq.q8_workspace(c.dims, max(lens), n) if ws is None else ws
    okvq.okvq_q8_window_attention(c, layer, lens, q.cuda(), new, _i32(new) if new_dev is None else new_dev, n, window, sinks, sm, out, ws,
                                  stream=stream)
    return out


def _check_window(c, out, lens, q, new, window, sinks, fmt, dtype, tag, sm=SM, layer=0, fill=9.0, rows=None):
    a, got = _numpy(c), _np(out)
    B, Hq, n, _ = q.shape
    H = c.dims.num_kv_heads
    G, worst = Hq // H, 0.0
    for b in range(B):
        assert np.all(got[b, :, new[b]:] == fill), f"{tag}: rows behind the last one were written"
        if not new[b]:
            continue
        pick = np.arange(new[b]) if rows is None else np.unique(np.clip(rows, 0, new[b] - 1))
        seen = oq.window_seen(lens[b], new[b], window, sinks)[pick]
        for h in range(H):
            k, v = oq.read_sequence(a, layer, b, h, lens[b], fmt)
            for j in range(h * G, (h + 1) * G):
                ref, bound = oq.attention_where(_np(q[b, j, pick]), k, v, seen, sm, HALF[dtype])
                assert np.all(got[b, j, pick][~seen.any(1)] == 0), f"{tag}: a row that sees nothing yields zeros"
                worst = max(worst, _worst(got[b, j, pick], ref, bound))
    _say(f"{tag}: worst err / bound {worst:.3f}")
    assert worst <= 1


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16"), ("int8", "bf16"), ("e4m3", "fp16")])
@pytest.mark.parametrize("H, Hq, page, lens, window, sinks", [
    (2, 14, 64, [0, 1, 31, 32, 33, 64, 65, 500], 20, 3),
    (1, 1, 32, [97, 5], 1, 0),                       # a row sees itself alone
    (1, 16, 256, [700, 256], 64, 32),                # whole blocks
    (3, 12, 128, [1300], 1000, 333),                 # sinks and window overlap
    (4, 32, 64, [2049, 2050, 17], 500, 1),
    (1, 7, 64, [3333, 3000, 40], 31, 33),
    (1, 4, 64, [640, 100], 1 << 30, 5),              # a window longer than anything
    (1, 4, 64, [640, 100], 2, 1 << 30),              # everything is a sink
    (1, 5, 64, [9000], 5000, 0),                     # split over many work-groups
])
def test_window_of_one_token(fmt, dtype, H, Hq, page, lens, window, sinks):
    B = len(lens)
    c = _filled(B, H, Hq, lens, page, fmt, dtype, 11)
    q = _rows(12, B, Hq, 1, 128, dtype=dtype, scale=2.0)
    out = _window(c, lens, q, [1] * B, window, sinks)
    _check_window(c, out, lens, q, [1] * B, window, sinks, fmt, dtype, f"window {fmt} {dtype} Hq={Hq} {lens} {window}+{sinks}")


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("H, Hq, lens, new, window, sinks", [
    (1, 4, [40], [40], 7, 2),                        # a whole prompt
    (2, 14, [129, 64, 200, 31], [129, 3, 0, 31], 33, 4),
    (1, 7, [300, 301], [17, 2], 40, 0),
    (1, 3, [100, 5, 2], [12, 12, 12], 3, 1),         # more rows than tokens: the first ones see nothing
    (1, 8, [1500, 1025], [130, 128], 200, 70),       # the prompt kernel, whole and half
    (1, 8, [1500, 900], [300, 300], 64, 64),
    (1, 8, [700], [700], 1, 0),
    (2, 6, [3000], [2], 1000, 5),
    (1, 5, [2500, 2400], [23, 20], 100, 1000),
    (1, 1, [700], [650], 129, 65),
    (1, 16, [4000, 3900], [100, 40], 3000, 17),      # splits of the prompt kernel
])
def test_window_of_chunks(fmt, dtype, H, Hq, lens, new, window, sinks):
    B, n = len(lens), max(new)
    c = _filled(B, H, Hq, lens, 64, fmt, dtype, 13)
    q = _rows(14, B, Hq, n + 1, 128, dtype=dtype, scale=1.5)  # a row more than any sequence has
    for b in range(B):
        q[b, :, new[b]:] = float("nan")
    out = _window(c, lens, q, new, window, sinks)
    rows = None if n < 200 else np.unique(np.concatenate([np.arange(0, n, 17), np.arange(n - 40, n)]))
    _check_window(c, out, lens, q, new, window, sinks, fmt, dtype, f"window chunk {fmt} {dtype} Hq={Hq} {lens} {new} {window}+{sinks}",
                  rows=rows)


def test_blocks_outside_are_not_read():
    """Pages between the sinks and the window hold NaN scales, which a single read of theirs would show."""
    n, window, sinks = 2000, 300, 10
    for new, Hq in ((1, 7), (40, 7), (20, 16)):
        c = _filled(1, 1, Hq, [n], 64, "int8", "fp16", 15)
        q = _rows(16, 1, Hq, new, 128)
        want = _window(c, [n], q, [new], window, sinks)
        first = (n - new + 1 - window) // 64
        for page in c["block_table"][0, 1:first].tolist():
            c["k_scale"][0, page] = float("nan")
            c["v_scale"][0, page] = float("nan")
        got = _window(c, [n], q, [new], window, sinks)
        assert np.array_equal(_np(got), _np(want)), new


def test_window_is_whole_attention_where_it_covers_all():
    import torch

    import paper_2609_11582_amd as okvq
    lens = [700, 64, 1]
    c = _filled(3, 2, 8, lens, 64, "e4m3", "bf16", 17)
    for new in ([1, 1, 1], [50, 20, 1]):
        n = max(new)
        q = _rows(18, 3, 8, n, 128, dtype="bf16")
        out = torch.full((3, 8, n, 128), 9.0, dtype=torch.bfloat16, device="cuda")
        okvq.okvq_q8_attention(c, 0, lens, q.cuda(), new, _i32(new), n, SM, out, okvq.q8_workspace(c.dims, 700, n))
        assert torch.equal(out, _window(c, lens, q, new, 700, 0))


@pytest.mark.parametrize("sm", [0.0, -0.05, 3.0])
def test_window_softmax_scales(sm):
    lens = [333, 40]
    c = _filled(2, 1, 4, lens, 64, "int8", "fp16", 31)
    for n in (1, 20, 60):
        q, new = _rows(32, 2, 4, n, 128), [n, min(n, 40)]
        _check_window(c, _window(c, lens, q, new, 50, 3, sm=sm), lens, q, new, 50, 3, "int8", "fp16", f"scale {sm} rows {n}", sm=sm)


def test_window_far_into_an_upper_layer():
    n = 131072
    c = _filled(1, 1, 8, [n], 256, "e4m3", "bf16", 51, drift=0.01, layers=2, layer=1)
    for m in (1, 24):
        q = _rows(52, 1, 8, m, 128, dtype="bf16")
        out = _window(c, [n], q, [m], 4097, 4, layer=1)
        _check_window(c, out, [n], q, [m], 4097, 4, "e4m3", "bf16", f"131072 tokens, {m} rows", layer=1, rows=np.array([0, 23]))


def test_window_counts_of_the_device_alone():
    """A captured call is replayed with lengths and counts that its host arrays do not have."""
    lens, host_lens, new, host_new = [700, 90, 300, 0], [300, 300, 0, 5], [3, 0, 4, 2], [4, 4, 0, 4]
    c = _filled(4, 1, 7, lens, 64, "int8", "fp16", 61)
    q = _rows(62, 4, 7, 4, 128)
    out = _window(c, host_lens, q, host_new, 60, 3, new_dev=_i32(new))
    _check_window(c, out, lens, q, new, 60, 3, "int8", "fp16", "other counts on the device")


# ---- trees ---------------------------------------------------------------------------------------


def _parents(rng, n, kind):
    if kind == "chain":
        return list(range(-1, n - 1))
    if kind == "star":
        return [-1] * n
    return [int(rng.integers(-1, i)) if rng.random() < 0.6 else i - 1 for i in range(n)]


def _tree(c, lens, q, k, v, visible, n_draft, window=0, sinks=0, sm=SM, layer=0, fill=9.0, n_dev=None, ws=None, stream=None):
    import torch

    import paper_2609_11582_amd as okvq
    B, Hq, n, _ = q.shape
    out = torch.full((B, Hq, n, 128), fill, dtype=c.row_dtype, device="cuda")
    ws = okvq.q8_tree_workspace(c.dims, n) if ws is None else ws
    vis = visible if isinstance(visible, torch.Tensor) else torch.from_numpy(visible.view(np.int32))
    okvq.okvq_q8_tree_attention(c, layer, lens, q.cuda(), k.cuda(), v.cuda(), vis.cuda(), n_draft,
                                _i32(n_draft) if n_dev is None else n_dev, n, sm, out, ws, window=window, sinks=sinks, stream=stream)
    return out


def _check_tree(c, out, lens, q, kd, vd, visible, n_draft, fmt, dtype, tag, window=0, sinks=0, sm=SM, layer=0, fill=9.0, scale=1.0,
                rows=None):
    """scale: what values and outputs are divided by before they are compared; rows: those compared, all if None"""
    a, got = _numpy(c), _np(out)
    B, Hq, n, _ = q.shape
    H = c.dims.num_kv_heads
    G, worst = Hq // H, 0.0
    for b in range(B):
        m = n_draft[b]
        assert np.all(got[b, :, m:] == fill), f"{tag}: rows behind the last draft were written"
        if not m:
            continue
        pick = np.arange(m) if rows is None else np.unique(np.clip(rows, 0, m - 1))
        seen = oq.tree_seen(lens[b], visible[b], m, window, sinks)[pick]
        for h in range(H):
            k, v = oq.read_sequence(a, layer, b, h, lens[b], fmt)
            k, v = np.concatenate([k, _np(kd[b, h, :m])]), np.concatenate([v, _np(vd[b, h, :m])]) / scale
            k, v = np.where(seen.any(0)[:, None], k, 0), np.where(seen.any(0)[:, None], v, 0)
            for j in range(h * G, (h + 1) * G):
                ref, bound = oq.attention_where(_np(q[b, j, pick]), k, v, seen, sm, HALF[dtype])
                assert np.all(got[b, j, pick][~seen.any(1)] == 0), f"{tag}: a row that sees nothing yields zeros"
                worst = max(worst, _worst(got[b, j, pick] / scale, ref, bound))
    _say(f"{tag}: worst err / bound {worst:.3f}")
    assert worst <= 1


def _drafts(seed, B, H, Hq, n, dtype):
    return (_rows(seed, B, Hq, n, 128, dtype=dtype, scale=1.5), _rows(seed + 1, B, H, n, 128, dtype=dtype, scale=1.2),
            _rows(seed + 2, B, H, n, 128, dtype=dtype, scale=2.0))


def _masks(parents, n):
    import paper_2609_11582_amd as okvq
    return okvq.q8_tree_visible(parents, n, device="cpu").numpy().view(np.uint32)


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16"), ("int8", "bf16"), ("e4m3", "fp16")])
@pytest.mark.parametrize("H, Hq, page, lens, n_draft, kind, window, sinks", [
    (1, 4, 64, [100], [1], "chain", 0, 0),
    (2, 14, 64, [0, 1, 33, 500], [5, 7, 0, 2], "any", 0, 0),        # a tree behind nothing
    (1, 16, 32, [700, 64], [16, 33], "any", 0, 0),
    (1, 1, 256, [1300], [64], "chain", 0, 0),
    (3, 12, 128, [300, 20], [40, 31], "star", 0, 0),
    (1, 8, 64, [2100], [65], "any", 0, 0),                          # prompt kernel
    (1, 7, 64, [5000], [30], "any", 0, 0),                          # splits of it
    (2, 2, 64, [900, 3000], [256, 3], "any", 0, 0),
    (1, 7, 64, [600, 90, 5], [12, 3, 12], "any", 50, 3),            # in a layer with a window
    (1, 8, 64, [3000], [70], "any", 700, 65),
    (1, 4, 64, [300], [9], "chain", 1, 0),                          # the window ends inside the line
    (1, 4, 64, [300], [9], "any", 40, 1 << 30),
])
def test_trees(fmt, dtype, H, Hq, page, lens, n_draft, kind, window, sinks):
    B, n = len(lens), min(max(n_draft) + 1, 256)  # a row more than any slot has, where a call may have so many
    c = _filled(B, H, Hq, lens, page, fmt, dtype, 71)
    q, k, v = _drafts(72, B, H, Hq, n, dtype)
    rng = np.random.default_rng(73)
    visible = _masks([_parents(rng, m, kind) for m in n_draft], n)
    for b, m in enumerate(n_draft):
        q[b, :, m:] = k[b, :, m:] = v[b, :, m:] = float("nan")
        visible[b, m:] = 0xffffffff
        if n > m and m:
            visible[b, :, m // 32] |= np.uint32((0xffffffff << m % 32) & 0xffffffff)  # bits behind the last draft say nothing
    out = _tree(c, lens, q, k, v, visible, n_draft, window, sinks)
    _check_tree(c, out, lens, q, k, v, visible, n_draft, fmt, dtype, f"tree {fmt} {dtype} Hq={Hq} {lens} {n_draft} {kind} {window}+{sinks}",
                window, sinks)


def test_any_masks():
    """Masks that are no trees: none, all, a row that does not see itself, drafts that see later ones; drafts that none
    names hold NaN."""
    import torch
    lens, n_draft, n = [0, 77, 200], [40, 40, 3], 40
    c = _filled(3, 1, 7, lens, 64, "int8", "fp16", 81)
    q, k, v = _drafts(82, 3, 1, 7, n, "fp16")
    rng = np.random.default_rng(83)
    visible = rng.integers(0, 1 << 32, (3, n, 2), dtype=np.uint32)
    visible[:, ::5] = 0
    visible[:, 1::5] = 0xffffffff
    visible[..., 0] &= np.uint32(0xffffffff ^ 1 << 6)
    for x in (k, v):
        x[:, :, 6] = float("nan")
        x[2, :, 3:] = float("nan")
    for window in (0, 25):
        out = _tree(c, lens, q, k, v, visible, n_draft, window, 2)
        _check_tree(c, out, lens, q, k, v, visible, n_draft, "int8", "fp16", f"any masks, window {window}", window, 2)
    assert bool((out[0, :, 0] == 0).all()) and torch.isfinite(out).all()


def test_a_line_is_what_its_appended_tokens_would_see():
    """A chain behind a cache and the same rows appended to it: the same within both bounds (the cache rounds the rows)."""
    lens, n = [130], 9
    q, kd, vd = _drafts(91, 1, 2, 8, n, "fp16")
    for window, sinks in ((0, 0), (40, 3)):
        c = _filled(1, 2, 8, lens, 64, "int8", "fp16", 90)
        got = _np(_tree(c, lens, q, kd, vd, _masks([list(range(-1, n - 1))], n), [n], window, sinks))
        a = _numpy(c)
        for h in range(2):
            k, v = oq.read_sequence(a, 0, 0, h, lens[0], "int8")
            k, v = np.concatenate([k, _np(kd[0, h])]), np.concatenate([v, _np(vd[0, h])])
            seen = oq.window_seen(lens[0] + n, n, window or 1 << 30, sinks)
            for j in range(4 * h, 4 * h + 4):
                ref, bound = oq.attention_where(_np(q[0, j]), k, v, seen, SM, HALF["fp16"])
                assert _worst(got[0, j], ref, bound) <= 1


def test_drafts_far_from_the_cache_in_size():
    """bfloat16 draft values of 1e38 and 1e-30 beside cached ones of unit size, scores that leave one part nothing, and all
    weights on 256 drafts of the largest size."""
    import torch
    n, L = 256, 100
    for vs, ks in ((1e37, 1.0), (1e-30, 1.0), (1.0, 30.0), (1e30, 0.01)):
        c = _filled(1, 1, 2, [L], 64, "e4m3", "bf16", 95)
        q, k, v = _drafts(96, 1, 1, 2, n, "bf16")
        k, v = (k.double() * ks).bfloat16(), (v.double() * vs).bfloat16()
        visible = _masks([list(range(-1, n - 1))], n)
        out = _tree(c, [L], q, k, v, visible, [n])
        _check_tree(c, out, [L], q, k, v, visible, [n], "e4m3", "bf16", f"drafts of {vs}, keys of {ks}", scale=max(vs, 1.0))
    c = _new(1, 1, 1, [0], 64, "int8", "bf16")
    c["seq_lens"].zero_()
    v = torch.full((1, 1, n, 128), 3e38).bfloat16()
    out = _tree(c, [0], q[:, :1], k * 0, v, np.full((1, n, 8), 0xffffffff, np.uint32), [n])
    assert torch.equal(out.cpu(), v)


@pytest.mark.parametrize("sm", [0.0, -0.05, 3.0])
def test_tree_softmax_scales(sm):
    lens, n_draft, n = [333, 40], [20, 60], 60
    c = _filled(2, 1, 4, lens, 64, "int8", "fp16", 31)
    q, k, v = _drafts(32, 2, 1, 4, n, "fp16")
    visible = _masks([_parents(np.random.default_rng(1), m, "any") for m in n_draft], n)
    out = _tree(c, lens, q, k, v, visible, n_draft, sm=sm)
    _check_tree(c, out, lens, q, k, v, visible, n_draft, "int8", "fp16", f"tree scale {sm}", sm=sm)


def test_tree_over_a_long_sequence_of_one_head():
    """128 splits, whose merge has 16 groups, and an upper layer."""
    L, n = 131072, 4
    c = _filled(1, 1, 2, [L], 256, "e4m3", "bf16", 51, drift=0.01, layers=2, layer=1)
    q, k, v = _drafts(52, 1, 1, 2, n, "bf16")
    visible = _masks([[-1, 0, 0, 2]], n)
    out = _tree(c, [L], q, k, v, visible, [n], layer=1)
    _check_tree(c, out, [L], q, k, v, visible, [n], "e4m3", "bf16", "tree over 131072 tokens", layer=1)


def test_tree_counts_of_the_device_alone():
    """Lengths and counts that the host arrays do not have: fewer, more (up to the largest), a slot the host calls idle."""
    lens, host_lens, n_dev, host_n = [700, 90, 300, 0, 2000], [300, 300, 0, 5, 2000], [3, 0, 6, 2, 1], [6, 4, 0, 4, 6]
    c = _filled(5, 1, 7, lens, 64, "int8", "fp16", 61)
    q, k, v = _drafts(62, 5, 1, 7, 6, "fp16")
    visible = _masks([_parents(np.random.default_rng(2), 6, "any")] * 5, 6)
    out = _tree(c, host_lens, q, k, v, visible, host_n, n_dev=_i32(n_dev))
    _check_tree(c, out, lens, q, k, v, visible, n_dev, "int8", "fp16", "other counts on the device")


def test_many_slots():
    """More tiles than the GPU holds at once: one split each, no split records."""
    B, H, G, n = 300, 2, 8, 5
    lens, n_draft = [17 * b % 90 for b in range(B)], [b % (n + 1) for b in range(B)]
    c = _filled(B, H, H * G, lens, 32, "int8", "fp16", 65)
    q, k, v = _drafts(66, B, H, H * G, n, "fp16")
    visible = _masks([_parents(np.random.default_rng(b), n_draft[b], "any") for b in range(B)], n)
    out = _tree(c, lens, q, k, v, visible, n_draft)
    _check_tree(c, out, lens, q, k, v, visible, n_draft, "int8", "fp16", "300 slots")
    new = [min(1, L) for L in lens]
    out = _window(c, lens, q[:, :, :1].contiguous(), new, 30, 4)
    _check_window(c, out, lens, q[:, :, :1].contiguous(), new, 30, 4, "int8", "fp16", "300 slots, a window")


# ---- the wide kernel: shapes that take it (q8_span_check.cpp holds the plan to that) --------------


@pytest.mark.parametrize("fmt, dtype, window, sinks", [("int8", "fp16", 0, 0), ("e4m3", "bf16", 0, 0), ("int8", "bf16", 17000, 33),
                                                       ("e4m3", "fp16", 16900, 0)])
def test_wide_tree_over_a_long_sequence(fmt, dtype, window, sinks):
    L, n, Hq = 20011 if not window else 30000, 16, 16
    c = _filled(1, 1, Hq, [L], 64, fmt, dtype, 121, drift=0.02)
    q, k, v = _drafts(122, 1, 1, Hq, n, dtype)
    visible = _masks([_parents(np.random.default_rng(123), n, "any")], n)
    out = _tree(c, [L], q, k, v, visible, [n], window, sinks)
    _check_tree(c, out, [L], q, k, v, visible, [n], fmt, dtype, f"wide tree {fmt} {dtype} {window}+{sinks}", window, sinks,
                rows=np.array([0, 3, 4, 15]))


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
def test_wide_window_of_a_chunk(fmt, dtype):
    L, n, Hq, window, sinks = 20000, 20, 16, 15000, 70
    c = _filled(1, 1, Hq, [L], 128, fmt, dtype, 124, drift=0.02)
    q = _rows(125, 1, Hq, n + 3, 128, dtype=dtype, scale=1.5)
    out = _window(c, [L], q, [n], window, sinks)
    _check_window(c, out, [L], q, [n], window, sinks, fmt, dtype, f"wide window {fmt} {dtype}", rows=np.array([0, 3, 4, 19]))


def _many(host=False):
    """40 slots, most with 16 drafts, of many lengths; host: what a captured call's host arrays may say instead"""
    lens = [(0, 1, 31, 32, 33, 64, 65, 100, 500, 1003)[(b * 7) % 10] for b in range(40)]
    n = [b % 16 if b % 5 == 0 else 16 for b in range(40)]
    return ([300] * 40, [16] * 40) if host else (lens, n)


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("window, sinks, host", [(0, 0, False), (50, 3, False), (0, 0, True)])
def test_wide_tree_of_many_slots(fmt, dtype, window, sinks, host):
    (lens, n_draft), n = _many(), 16
    host_lens, host_n = _many(host)
    c = _filled(40, 2, 16, lens, 32, fmt, dtype, 126)
    q, k, v = _drafts(127, 40, 2, 16, n, dtype)
    visible = _masks([_parents(np.random.default_rng(b), m, "any") for b, m in enumerate(n_draft)], n)
    out = _tree(c, host_lens, q, k, v, visible, host_n, window, sinks, n_dev=_i32(n_draft))
    _check_tree(c, out, lens, q, k, v, visible, n_draft, fmt, dtype, f"wide tree of 40 slots {fmt} {dtype} {window}+{sinks}", window, sinks,
                rows=np.arange(0, 16, 3))


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
def test_wide_window_of_many_slots(fmt, dtype):
    (lens, new), n = _many(), 16
    c = _filled(40, 2, 16, lens, 32, fmt, dtype, 128)
    q = _rows(129, 40, 16, n, 128, dtype=dtype, scale=1.5)
    out = _window(c, lens, q, new, 90, 40)
    _check_window(c, out, lens, q, new, 90, 40, fmt, dtype, f"wide window of 40 slots {fmt} {dtype}",
                  rows=np.arange(0, 16, 3))


def test_wide_of_few_rows():
    lens, n = [4096 - 37 * b for b in range(16)], 3
    c = _filled(16, 4, 28, lens, 64, "int8", "fp16", 130)
    q, k, v = _drafts(131, 16, 4, 28, n, "fp16")
    visible = _masks([[-1, 0, 0]] * 16, n)
    out = _tree(c, lens, q, k, v, visible, [n] * 16)
    _check_tree(c, out, lens, q, k, v, visible, [n] * 16, "int8", "fp16", "wide tree of 21 rows")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("case", range(4))
def test_wide_dominant_tokens_and_uneven_values(fmt, case):
    """A flat background with tokens 10 to 30 log2 units above it, growing and falling along the sequence, whose values
    are small where attention is large (and the other way round); blocks of zero values."""
    import torch
    L, n = 20000, 128
    c = _new(1, 1, 2, [L], 64, fmt)
    g = torch.Generator().manual_seed(140 + case)
    k, v = 0.01 * torch.randn(1, 1, L, 128, generator=g), 0.01 * torch.randn(1, 1, L, 128, generator=g) + 1.0
    at = torch.arange(0, L, 512)
    k[0, 0, at, 0] = torch.linspace(10, 30, len(at)) if case % 2 else torch.linspace(30, 10, len(at))
    v[0, 0] *= torch.where(torch.arange(L) % 512 < 32, 2.0 ** -9 if case < 2 else 2.0 ** 9, 1.0)[:, None]
    v[0, 0, 640:704] = 0
    k, v = k.half(), v.half()
    _append(c, 0, k, v, [0], [L])
    q = torch.zeros(1, 2, n, 128)
    q[:, :, :, 0] = math.log(2.0) / SM  # scores are the first channel, in log2 units
    q[:, 1] *= 0.3
    kd, vd = 0.01 * torch.randn(1, 1, n, 128, generator=g), torch.randn(1, 1, n, 128, generator=g)
    kd[0, 0, ::3, 0] = 29
    q, kd, vd = q.half(), kd.half(), vd.half()
    visible = _masks([[-1] * n], n)
    out = _tree(c, [L], q, kd, vd, visible, [n])
    _check_tree(c, out, [L], q, kd, vd, visible, [n], fmt, "fp16", f"wide dominant {fmt} case {case}", rows=np.array([0, 1, 31, 32, 127]))


@pytest.mark.parametrize("sm", [0.0, -0.05, 2.0])
def test_wide_softmax_scales_and_subnormal_values(sm):
    """Values of scales below 2^-126 count as nothing beside others; negative and zero scales."""
    import torch
    L, n, Hq = 20000, 16, 16
    c = _filled(1, 1, Hq, [L], 64, "int8", "bf16", 150, drift=0.02)
    k, v = _rows(151, 1, 1, 64, 128, dtype="bf16"), (_rows(152, 1, 1, 64, 128).double() * 1e-38).to(torch.bfloat16)
    c["seq_lens"].copy_(_i32([L]))
    page = int(c["block_table"][0, 3])
    code, _ = oq.quantize_block(v[0, 0, :32].float().numpy(), "int8")
    c["v_codes"][0, page, 0, 0] = torch.from_numpy(oq.pack_values(code)).cuda()
    c["v_scale"][0, page, 0, 0] = 2.0 ** -130
    q, kd, vd = _drafts(153, 1, 1, Hq, n, "bf16")
    visible = _masks([_parents(np.random.default_rng(154), n, "any")], n)
    out = _tree(c, [L], q, kd, vd, visible, [n], sm=sm)
    _check_tree(c, out, [L], q, kd, vd, visible, [n], "int8", "bf16", f"wide scale {sm}", sm=sm, rows=np.array([0, 3, 4, 15]))


# ---- the prompt kernel, whole and half tiles, split and not (q8_span_check.cpp again) ------------


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("n, L, window, sinks", [(600, 900, 130, 40), (1200, 1200, 333, 5), (2500, 2500, 100, 65), (1200, 3000, 1, 0), (600, 700, 1 << 30, 0)])
def test_window_of_prompts(fmt, dtype, n, L, window, sinks):
    c = _filled(1, 4, 28, [L], 64, fmt, dtype, 161)
    q = _rows(162, 1, 28, n, 128, dtype=dtype, scale=1.5)
    out = _window(c, [L], q, [n], window, sinks)
    rows = np.array([0, 1, 8, 9, 17, 18, 19, 35, 36, 37, 63, 64, 100, 300, 301, 302, 500, n - 40, n - 2, n - 1])
    _check_window(c, out, [L], q, [n], window, sinks, fmt, dtype, f"window prompt {fmt} {dtype} {n} of {L} {window}+{sinks}", rows=rows)


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("window, sinks", [(0, 0), (300, 33)])
def test_prompt_kernel_for_trees(fmt, dtype, window, sinks):
    """16 slots of 448 columns: tiles of 256 (of 128 with the window), two splits each, one without drafts."""
    lens, n_draft, n = [1500 - 90 * b for b in range(16)], [0 if b == 5 else 64 - b for b in range(16)], 64
    c = _filled(16, 4, 28, lens, 64, fmt, dtype, 163)
    q, k, v = _drafts(164, 16, 4, 28, n, dtype)
    visible = _masks([_parents(np.random.default_rng(b), m, "any") for b, m in enumerate(n_draft)], n)
    out = _tree(c, lens, q, k, v, visible, n_draft, window, sinks)
    _check_tree(c, out, lens, q, k, v, visible, n_draft, fmt, dtype, f"prompt kernel's tree {fmt} {dtype} {window}+{sinks}", window, sinks,
                rows=np.array([0, 9, 36, 37, 63]))


def test_windows_past_any_sequence():
    """The largest window and sinks, rows before the first token: what reaches past a sequence is everything."""
    import torch
    lens, new = [5, 300, 0], [40, 40, 40]
    c = _filled(3, 1, 7, lens, 64, "int8", "fp16", 165)
    q = _rows(166, 3, 7, 40, 128)
    big = (1 << 31) - 1
    out = _window(c, lens, q, new, big, big)
    _check_window(c, out, lens, q, new, 1 << 40, 0, "int8", "fp16", "largest window")
    qd, k, v = _drafts(167, 3, 1, 7, 9, "fp16")
    visible = _masks([_parents(np.random.default_rng(4), 9, "any")] * 3, 9)
    a = _tree(c, lens, qd, k, v, visible, [9] * 3, big, 0)
    b = _tree(c, lens, qd, k, v, visible, [9] * 3, 1 << 27, big)
    assert torch.equal(a, b)
    _check_tree(c, a, lens, qd, k, v, visible, [9] * 3, "int8", "fp16", "largest window of a tree")


def test_many_even_slots_take_one_split():
    """160 tiles of more rounds than a split has elsewhere, and one slot that is longer than the others."""
    for lens in ([2100] * 160, [2100] * 159 + [4000]):
        c = _filled(160, 1, 2, lens, 64, "int8", "fp16", 171)
        q = _rows(172, 160, 2, 1, 128)
        _check_window(c, _window(c, lens, q, [1] * 160, 2500, 3), lens, q, [1] * 160, 2500, 3, "int8", "fp16", f"even slots {lens[-1]}")
        n_draft = [2] * 159 + [1]
        qd, k, v = _drafts(173, 160, 1, 2, 2, "fp16")
        visible = _masks([[-1, 0][:m] for m in n_draft], 2)
        _check_tree(c, _tree(c, lens, qd, k, v, visible, n_draft), lens, qd, k, v, visible, n_draft, "int8", "fp16", f"even trees {lens[-1]}")


# ---- as they are used ----------------------------------------------------------------------------


def test_captured_and_replayed():
    """A window step and a tree call in two graphs with workspaces of their own, replayed on two streams while the counts on the
    device change; eager calls between them."""
    import torch

    import paper_2609_11582_amd as okvq
    lens = [333, 900]
    c = _filled(2, 1, 7, lens, 64, "int8", "fp16", 101)
    q1, n1 = _rows(102, 2, 7, 1, 128).cuda(), _i32([1, 1])
    q, k, v = (x.cuda() for x in _drafts(103, 2, 1, 7, 12, "fp16"))
    visible = okvq.q8_tree_visible([_parents(np.random.default_rng(3), 12, "any")] * 2, 12)
    nd = _i32([12, 12])
    o1, o2 = torch.zeros_like(q1), torch.zeros_like(q)
    ws1, ws2 = okvq.q8_workspace(c.dims, 900, 1), okvq.q8_tree_workspace(c.dims, 12)

    def window(out):
        okvq.okvq_q8_window_attention(c, 0, lens, q1, [1, 1], n1, 1, 200, 4, SM, out, ws1)

    def tree(out):
        okvq.okvq_q8_tree_attention(c, 0, lens, q, k, v, visible, [12, 12], nd, 12, SM, out, ws2)
    window(o1), tree(o2)
    torch.cuda.synchronize()
    graphs = []
    for f, o in ((window, o1), (tree, o2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f(o)
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for counts, shorter in (([12, 12], 0), ([3, 0], 100), ([0, 7], 33), ([12, 1], 0)):
        nd.copy_(_i32(counts))
        c["seq_lens"].copy_(_i32([L - shorter for L in lens]))
        for o in (o1, o2):
            o.fill_(9.0)
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        e1, e2 = torch.full_like(o1, 9.0), torch.full_like(o2, 9.0)
        window(e1), tree(e2)
        torch.cuda.synchronize()
        assert torch.equal(o1, e1) and torch.equal(o2, e2)
        now = [L - shorter for L in lens]
        _check_window(c, o1, now, q1.cpu(), [1, 1], 200, 4, "int8", "fp16", f"replayed window {now}")
        _check_tree(c, o2, now, q.cpu(), k.cpu(), v.cpu(), visible.cpu().numpy().view(np.uint32), counts, "int8", "fp16", f"replayed tree {counts}")


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
def test_a_prompt_then_drafts_that_are_verified(fmt, dtype):
    """Two layers, one whole and one with a window: a prompt in two chunks, then three turns of drafts of which some lines are
    accepted and appended; all against the oracle over a cache that the page model follows."""
    import torch

    import paper_2609_11582_amd as okvq
    B, H, Hq, n, window, sinks = 3, 2, 6, 7, 60, 4
    freq, axes = [1e4 ** (-i / 64) for i in range(64)], [0] * 16 + [1] * 24 + [2] * 24
    par, eps = okvq.make_rotary(freq, axes), 1e-6
    dt = torch.float16 if dtype == "fp16" else torch.bfloat16
    c = okvq.Q8Cache(B, H, Hq, 40, 10, layers=2, page_tokens=64, format=fmt, dtype=dtype)
    model, pw = oq.PagedModel(B, 40, 64, 10), okvq.q8_page_workspace(c.dims)
    granted = torch.zeros(B, dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(5)
    seed = [200]

    def turned(m, pos):
        """(q, k, v) of m new rows: projections' rows, normed and rotated"""
        seed[0] += 10
        wq, wk = (torch.rand(128, generator=torch.Generator().manual_seed(seed[0] + i)) + 0.5 for i in range(2))
        q, k, v = (_rows(seed[0] + 2 + i, B, m, h, 128, dtype=dtype, scale=3.0) for i, h in enumerate((Hq, H, H)))
        qo, ko = (torch.empty(B, h, m, 128, dtype=dt, device="cuda") for h in (Hq, H))
        p = torch.from_numpy(np.broadcast_to(pos[:, None], (B, 3, m)).astype(np.int32).copy())
        okvq.okvq_norm_rotary(par, q.cuda().transpose(1, 2), k.cuda().transpose(1, 2), wq.cuda(), wk.cuda(), eps, p.cuda(), qo, ko)
        for x, w, y in ((q, wq, qo), (k, wk, ko)):
            ref, size = nr.norm_rotate(_np(x.transpose(1, 2)), _np(w), eps, p.numpy(), freq, axes)
            assert np.all(np.abs(_np(y) - ref) <= HALF[dtype] * np.abs(ref) + 2.0 ** -19 * size + 2.0 ** -25)
        return qo, ko, v.transpose(1, 2).contiguous().cuda()

    def grow(new):
        okvq.okvq_q8_extend(c, _i32(new), granted, pw)
        assert model.extend(new) == new

    def append(layer, k, v, new):
        okvq.okvq_q8_append(c, layer, model.lens, k, v, new, granted, k.shape[2])

    for new in ([70, 0, 33], [61, 90, 1]):                                   # the prompt
        m = max(new)
        grow(new)
        pos = np.stack([np.arange(m) + L - x for L, x in zip(model.lens, new)])
        for layer in (0, 1):
            q, k, v = turned(m, pos)
            append(layer, k, v, new)
            if layer:
                out = _window(c, model.lens, q, new, window, sinks, layer=1)
                _check_window(c, out, model.lens, q, new, window, sinks, fmt, dtype, f"prompt {new}", layer=1)
    for turn in range(3):
        n_draft = [n, int(rng.integers(1, n)), n - 1]
        parents = [_parents(rng, m, "any") for m in n_draft]
        visible = _masks(parents, n)
        depth = np.array([[bin(int(x)).count("1") - 1 for x in visible[b, :, 0]] for b in range(B)])
        pos = np.array(model.lens)[:, None] + depth
        kept = []
        for layer in (0, 1):
            q, k, v = turned(n, pos)
            kept.append((k, v))
            w = (window, sinks) if layer else (0, 0)
            out = _tree(c, model.lens, q, k, v, visible, n_draft, *w, layer=layer)
            _check_tree(c, out, model.lens, q, k, v, visible, n_draft, fmt, dtype, f"turn {turn} layer {layer}", *w, layer=layer)
        ends = [int(rng.integers(0, m)) for m in n_draft]                    # the accepted lines
        lines = [[j for j in range(n) if visible[b, e, 0] >> j & 1] for b, e in enumerate(ends)]
        new = [len(x) for x in lines]
        grow(new)
        pick = torch.tensor([x + [0] * (n - len(x)) for x in lines], device="cuda")[:, None, :, None].expand(B, H, n, 128)
        for layer, (k, v) in enumerate(kept):
            append(layer, k.gather(2, pick), v.gather(2, pick), new)
        a = _numpy(c)
        for f, want in model.arrays().items():
            assert np.array_equal(a[f], want), f
    # one token more in both layers
    grow([1] * B)
    q, k, v = turned(1, np.array(model.lens)[:, None] - 1)
    for layer in (0, 1):
        append(layer, k, v, [1] * B)
        w = (window, sinks) if layer else (1 << 30, 0)
        _check_window(c, _window(c, model.lens, q, [1] * B, *w, layer=layer), model.lens, q, [1] * B, *w, fmt, dtype, f"last token, layer {layer}",
                      layer=layer)


def test_refuses_wrong_calls():
    import torch

    import paper_2609_11582_amd as okvq
    c = _filled(1, 1, 2, [40], 64, "int8", "fp16", 111)
    q, k, v = (x.cuda() for x in _drafts(112, 1, 1, 2, 3, "fp16"))
    vis, n_dev, out, ws = okvq.q8_tree_visible([[-1, 0, 1]], 3), _i32([3]), torch.zeros_like(q), okvq.q8_tree_workspace(c.dims, 3)

    def tree(q=q, k=k, v=v, vis=vis, n=(3,), n_max=3, out=out, ws=ws, window=0, sinks=0):
        okvq.okvq_q8_tree_attention(c, 0, [40], q, k, v, vis, n, n_dev, n_max, SM, out, ws, window=window, sinks=sinks)
    for bad in (dict(k=k.bfloat16()), dict(v=v.cpu()), dict(vis=vis.long()), dict(vis=vis[:, :2].contiguous()), dict(q=q[:, :, :2]),
                dict(out=torch.zeros(1, 3, 2, 128, dtype=torch.float16, device="cuda")), dict(n_max=2)):
        with pytest.raises(ValueError):
            tree(**bad)
    for bad in (dict(n=(4,)), dict(window=-1), dict(sinks=-1), dict(ws=ws[:4])):
        with pytest.raises(okvq.OkvqError):
            tree(**bad)
    for window, sinks in ((0, 0), (-1, 0), (5, -1)):
        with pytest.raises(okvq.OkvqError):
            okvq.okvq_q8_window_attention(c, 0, [40], q, [3], n_dev, 3, window, sinks, SM, out, ws)
    assert bool((out == 0).all())
