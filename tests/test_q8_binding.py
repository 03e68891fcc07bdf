"""Refusals of the 8-bit cache's binding, on a cache in host memory: every call here is refused, or has nothing to do,
before it could reach the device."""

import pytest
import torch

from paper_2609_11582_amd import q8

WRAP = 1 << 32  # what ctypes drops from a 32-bit argument


@pytest.fixture
def cache(monkeypatch):
    monkeypatch.setattr(q8, "_device", lambda: -1)  # where host tensors say that they are
    return q8.Q8Cache(2, 2, 4, 10, 4, layers=2, device="cpu")


def _append(c, layer=0, lens=(5, 5), n=(0, 0), n_max=1):
    k = torch.zeros(2, 2, 1, 128, dtype=torch.float16)
    return q8.okvq_q8_append(c, layer, lens, k, k, n, torch.zeros(4, dtype=torch.int32), n_max, stream=0)


def _attend(c, layer=0, lens=(5, 5), n=(0, 0), n_max=1, flags=0):
    q = torch.zeros(2, 4, 1, 128, dtype=torch.float16)
    return q8.okvq_q8_attention(c, layer, lens, q, n, torch.zeros(4, dtype=torch.int32), n_max, 0.1, torch.zeros_like(q),
                                q8.q8_workspace(c.dims, 64, device="cpu"), flags=flags, stream=0)


@pytest.mark.parametrize("call", [_append, _attend])
@pytest.mark.parametrize("kw", [dict(lens=(WRAP + 5, 5)), dict(lens=(5, 5 - WRAP)), dict(n=(0, WRAP)), dict(n=(-WRAP, 0)),
                                dict(layer=WRAP), dict(layer=WRAP + 1), dict(layer=-WRAP)])
def test_counts_past_32_bits(cache, call, kw):
    assert call(cache) == 0
    with pytest.raises(ValueError):
        call(cache, **kw)


def test_other_arguments_past_32_bits(cache):
    with pytest.raises(ValueError):
        _attend(cache, flags=WRAP)
    for slots in ([WRAP], [0, WRAP + 1], [-WRAP]):
        with pytest.raises(ValueError):
            q8.okvq_q8_free(cache, slots, stream=0)
        with pytest.raises(ValueError):
            q8.okvq_q8_fork(cache, slots, [1, 0][:len(slots)], stream=0)
        with pytest.raises(ValueError):
            q8.okvq_q8_fork(cache, [1, 0][:len(slots)], slots, stream=0)
    with pytest.raises(ValueError):
        q8.okvq_q8_workspace_bytes(cache.dims, WRAP + 100, 1)
    with pytest.raises(ValueError):
        q8.okvq_q8_workspace_bytes(cache.dims, 100, WRAP + 1)
    for name in ("batch", "num_kv_heads", "num_q_heads", "num_pages", "max_pages", "layers", "page_tokens"):
        sizes = dict(batch=2, num_kv_heads=2, num_q_heads=4, num_pages=10, max_pages=4)
        sizes[name] = WRAP + sizes.get(name, 64)
        with pytest.raises(ValueError):
            q8.make_q8_dims(**sizes)


@pytest.mark.parametrize("shape", [(2, 5, 2, 128), (2, 2, 6, 128), (4, 5, 128), (2, 2, 5, 256), (3, 2, 5, 128)])
def test_rows_in_another_order(cache, shape):
    """Enough bytes are not enough: rows that lie token by token, a longer buffer's rows."""
    good, bad = (torch.zeros(s, dtype=torch.float16) for s in ((2, 2, 5, 128), shape))
    n_dev, none, ws = torch.zeros(4, dtype=torch.int32), (0, 0), q8.q8_workspace(cache.dims, 64, 5, device="cpu")

    def append(k, v):
        return q8.okvq_q8_append(cache, 0, (9, 9), k, v, none, n_dev, 5, stream=0)

    def attend(q, out):
        return q8.okvq_q8_attention(own_heads, 0, (9, 9), q, none, n_dev, 5, 0.1, out, ws, stream=0)
    own_heads = q8.Q8Cache(2, 2, 2, 10, 4, device="cpu")
    for call in (append, attend):
        assert call(good, good) == 0
        for pair in ((bad, good), (good, bad)):
            with pytest.raises(ValueError):
                call(*pair)


@pytest.mark.parametrize("shape", [(2, 2, 128), (2, 1, 2, 128), (2, 2, 1, 128)])
def test_dimensions_of_one_entry_move_nothing(cache, shape):
    x = torch.zeros(shape, dtype=torch.float16)
    assert q8.okvq_q8_append(cache, 0, (9, 9), x, x, (0, 0), torch.zeros(4, dtype=torch.int32), 1, stream=0) == 0
    with pytest.raises(ValueError):
        q8.okvq_q8_append(cache, 0, (9, 9), x, x, (0, 0), torch.zeros(4, dtype=torch.int32), 2, stream=0)
