"""The sizes of workspaces that the header states, and that no call accepts less."""

import ctypes

import pytest

from paper_2609_11582_amd import q8
from test_q8_abi import FAKE, cache, dims, i32

FEW = 512 * 16 * 528  # records of 528 bytes: one for each column of as many tiles as calls of up to 32 rows are split into


@pytest.mark.parametrize("G", [1, 4, 7, 16])
@pytest.mark.parametrize("B, H", [(1, 1), (8, 4), (1024, 3)])
def test_tree(B, H, G):
    d = dims(batch=B, num_kv_heads=H, num_q_heads=H * G)
    for n in list(range(1, 40)) + [63, 64, 65, 255, 256]:
        cols = n * G
        up = 16 if cols <= 16 else 64 if cols <= 32 else -(-cols // 256) * 256
        assert q8.okvq_q8_tree_workspace_bytes(d, n) == q8.okvq_q8_workspace_bytes(d, 1000, n) + B * H * up * 528


def test_attention():
    d = dims(num_kv_heads=2, num_q_heads=8)
    assert [q8.okvq_q8_workspace_bytes(d, 700, n) for n in (4, 5, 8, 9)] == [FEW, 2 * FEW, 2 * FEW, 8 * FEW]

    def call(n, nbytes, window=None):
        more = (0.1, FAKE, FAKE, nbytes) + ((0,) if window is None else ()) + (None,)
        head = (ctypes.byref(cache(d)), 0, i32(700, 700), FAKE, i32(n, 1), FAKE, n)
        if window is None:
            return q8.lib().okvq_q8_attention(*head, *more)
        return q8.lib().okvq_q8_window_attention(*head, window, 0, *more)
    for n in (1, 4, 5, 8):  # whole attention asks for no more up to 32 rows of a KV head (test_gpu_z_q8_span_kernels.py runs it with so much)
        assert call(n, FEW - 1) == -4
    assert call(9, FEW) == -4
    assert call(4, FEW - 1, 50) == -4 and call(5, 2 * FEW - 1, 50) == -4 and call(9, 8 * FEW - 1, 50) == -4
