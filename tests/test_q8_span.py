"""Window and tree attention over the 8-bit cache without a GPU: the walk and the records (q8_span_check.cpp), masks and the
oracle's view of them, sizes and refusals."""

import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import q8 as oq
from paper_2609_11582_amd import _build, q8
from test_q8_abi import FAKE, OFF, cache, dims, i32


def test_walk_and_records(tmp_path):
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "q8_span_check.cpp")
    exe = str(tmp_path / "q8_span_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", _build.CSRC, src, "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout[-2000:] + r.stderr[-2000:]


def test_masks_of_trees():
    parents = [[-1, 0, 0, 2, -1], [], [-1] + list(range(39))]
    m = q8.q8_tree_visible(parents, 40, device="cpu").numpy().view(np.uint32)
    assert m.shape == (3, 40, 2)
    assert m[0, :6, 0].tolist() == [1, 0b11, 0b101, 0b1101, 0b10000, 0] and not m[1].any()
    assert m[2, 39].tolist() == [0xffffffff, 0xff] and m[2, 31].tolist() == [0xffffffff, 0]
    seen = oq.tree_seen(7, m[0], 5, 3, 2)
    assert seen[3].tolist() == [1, 1, 0, 0, 0, 0, 0, 1, 0, 1, 1, 0]      # a line of three drafts fills the window
    assert seen[0].tolist() == [1, 1, 0, 0, 0, 1, 1, 1, 0, 0, 0, 0]
    chain = oq.tree_seen(50, m[2], 40, 20, 4)                            # a line of 20: what its appended tokens would see
    want = oq.window_seen(90, 40, 20, 4)
    assert np.array_equal(chain[:20], want[:20])
    for bad in ([[0]], [[-1, 1]], [[-2]], [[-1] * 41]):
        with pytest.raises(ValueError):
            q8.q8_tree_visible(bad, 40, device="cpu")


def test_window_refused():
    L, d = q8.lib(), dims()

    def call(d=d, layer=0, lens=(700, 700), q=FAKE, n=(1, 1), nd=FAKE, n_max=1, window=5, sinks=0, sm=0.1, out=FAKE, ws=FAKE,
             nbytes=1 << 40):
        return L.okvq_q8_window_attention(ctypes.byref(cache(d)), layer, i32(*lens), q, i32(*n), nd, n_max, window, sinks,
                                          ctypes.c_float(sm), out, ws, nbytes, None)
    assert call(window=0) == -1 and call(window=-3) == -1 and call(sinks=-1) == -1
    assert call(layer=1) == -1 and call(q=OFF) == -1 and call(out=OFF) == -1 and call(nd=None) == -1 and call(sm=math.nan) == -1
    assert call(lens=(20 * 64 + 1, 0)) == -3 and call(lens=(-1, 0)) == -1 and call(n=(0, 2)) == -1 and call(n_max=-1) == -1
    assert call(ws=None) == -4 and call(ws=OFF) == -4 and call(nbytes=100) == -4
    assert call(d=dims(head_dim=64), window=0) == -2                     # the cache comes first
    assert call(n=(0, 0)) == 0
    assert L.okvq_q8_window_attention(None, 0, i32(1, 1), FAKE, i32(1, 1), FAKE, 1, 5, 0, 0.1, FAKE, FAKE, 1 << 40, None) == -1


def test_tree_refused():
    L, d = q8.lib(), dims()
    size = q8.okvq_q8_tree_workspace_bytes(d, 4)

    def call(d=d, layer=0, lens=(700, 700), q=FAKE, k=FAKE, v=FAKE, vis=FAKE, n=(4, 1), nd=FAKE, n_max=4, window=0, sinks=0, sm=0.1,
             out=FAKE, ws=FAKE, nbytes=size):
        return L.okvq_q8_tree_attention(ctypes.byref(cache(d)), layer, i32(*lens), q, k, v, vis, i32(*n), nd, n_max, window, sinks,
                                        ctypes.c_float(sm), out, ws, nbytes, None)
    assert call(window=-1) == -1 and call(sinks=-1) == -1 and call(n_max=257) == -1 and call(n_max=-1) == -1
    assert call(k=OFF) == -1 and call(v=None) == -1 and call(vis=None) == -1 and call(vis=OFF) == -1
    assert call(layer=-1) == -1 and call(q=OFF) == -1 and call(out=None) == -1 and call(nd=OFF) == -1 and call(sm=math.inf) == -1
    assert call(lens=(20 * 64 + 1, 0)) == -3 and call(n=(0, 5)) == -1 and call(n=(-1, 0)) == -1
    assert call(ws=None) == -4 and call(ws=OFF) == -4 and call(nbytes=100) == -4
    assert call(d=dims(batch=1025), window=-1) == -2
    assert call(n=(0, 0)) == 0 and call(n=(0, 0), n_max=0, q=None, k=None, v=None, vis=None, out=None) == 0


def test_tree_workspace():
    d = dims(batch=3, num_kv_heads=4, num_q_heads=28, max_pages=2048, num_pages=5000)
    sizes = [q8.okvq_q8_tree_workspace_bytes(d, n) for n in (1, 2, 4, 5, 16, 64, 256)]
    assert sizes == sorted(sizes) and sizes[0] >= q8.okvq_q8_workspace_bytes(d, 131072, 1) + 3 * 28 * 528
    assert sizes[-1] >= q8.okvq_q8_workspace_bytes(d, 131072, 256) + 3 * 28 * 256 * 528
    assert q8.okvq_q8_tree_workspace_bytes(d, 0) == 0 and q8.okvq_q8_tree_workspace_bytes(d, 257) == 0
    assert q8.okvq_q8_tree_workspace_bytes(dims(page_tokens=48), 4) == 0


@pytest.fixture
def host_cache(monkeypatch):
    monkeypatch.setattr(q8, "_device", lambda: -1)  # where host tensors say that they are
    return q8.Q8Cache(2, 2, 4, 10, 4, device="cpu")


def test_binding_checks_rows_and_numbers(host_cache):
    c, n_dev = host_cache, torch.zeros(4, dtype=torch.int32)

    def z(*s, dtype=torch.float16):
        return torch.zeros(*s, dtype=dtype)
    ws = q8.q8_tree_workspace(c.dims, 5, device="cpu")

    def window(q=z(2, 4, 5, 128), out=z(2, 4, 5, 128), window=3, sinks=1, n_max=5, lens=(9, 9)):
        return q8.okvq_q8_window_attention(c, 0, lens, q, (0, 0), n_dev, n_max, window, sinks, 0.1, out, ws, stream=0)

    def tree(q=z(2, 4, 5, 128), k=z(2, 2, 5, 128), v=z(2, 2, 5, 128), vis=z(2, 5, 1, dtype=torch.int32), out=z(2, 4, 5, 128), n_max=5,
             window=0, sinks=0):
        return q8.okvq_q8_tree_attention(c, 0, (9, 9), q, k, v, vis, (0, 0), n_dev, n_max, 0.1, out, ws, window=window, sinks=sinks,
                                         stream=0)
    assert window() == 0 and tree() == 0
    for call, kw in ((window, dict(q=z(2, 5, 4, 128))), (window, dict(out=z(2, 4, 5, 128, dtype=torch.bfloat16))),
                     (window, dict(window=1 << 32)), (window, dict(sinks=-(1 << 32))), (window, dict(n_max=4)), (window, dict(lens=(9,))),
                     (tree, dict(k=z(2, 4, 5, 128))), (tree, dict(v=z(2, 5, 2, 128))), (tree, dict(vis=z(2, 5, 2, dtype=torch.int32))),
                     (tree, dict(vis=z(2, 5, 1, dtype=torch.int64))), (tree, dict(q=z(2, 4, 6, 128))), (tree, dict(window=1 << 32)),
                     (tree, dict(k=z(2, 5, 2, 128).transpose(1, 2)))):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(ValueError):
        q8.okvq_q8_tree_workspace_bytes(c.dims, (1 << 32) + 4)
