"""Pins of the 8-bit cache's oracle: the e4m3 table and rounding against torch's conversion, the value byte order as
a permutation, exactness of representable rows, and the page model's invariants."""

import numpy as np
import pytest
import torch

from oracle import q8


def test_e4m3_table_and_rounding():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(q8.E4M3.astype(np.float32), want)
    x = np.concatenate([np.linspace(-448, 448, 20001), 2.0 ** np.linspace(-14, 8, 5001), [0.0, -0.0]]).astype(np.float32)
    mid = (q8.E4M3[1:0x7f] + q8.E4M3[:0x7e]) / 2  # ties
    x = np.concatenate([x, mid.astype(np.float32), -mid.astype(np.float32)])
    got = q8.e4m3_encode(x)
    np.testing.assert_array_equal(got, torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_value_bytes_are_a_permutation():
    assert sorted(q8.value_bytes().reshape(-1).tolist()) == list(range(4096))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_blocks(fmt):
    rng = np.random.default_rng(3)
    rows = rng.standard_normal((20, 128)).astype(np.float32)
    code, scale = q8.quantize_block(rows, fmt)
    x = q8.values_of(code, fmt) * float(scale)
    assert np.all(x[20:] == 0)
    step = scale * (0.5 if fmt == "int8" else 16)
    assert np.abs(x[:20] - rows).max() <= step * (1 + 1e-6)
    assert np.abs(x).max() == pytest.approx(np.abs(rows).max(), rel=1e-6)
    zero, one = q8.quantize_block(np.zeros((3, 128), np.float32), fmt)
    assert one == 1 and not zero.any()


def test_page_model_keeps_count():
    rng = np.random.default_rng(5)
    m = q8.PagedModel(5, 40, 64, 20)
    for _ in range(300):
        kind = rng.integers(4)
        if kind == 0:
            m.extend([int(x) for x in rng.integers(0, 90, 5)])
        elif kind == 1:
            a, b = rng.permutation(5)[:2]
            m.fork([int(a)], [int(b)])
        elif kind == 2:
            m.free([int(rng.integers(5))])
        else:
            n = m.compact()
            assert all(r > 0 for r in m.refs[:n]) and not any(m.refs[n:])
        held = [p for t in m.table for p in t]
        assert [held.count(p) for p in range(m.P)] == m.refs
        assert all(len(t) == -(-n // 64) for t, n in zip(m.table, m.lens))
