"""Host-side checks of the rotary positions and the 8-bit cache that need no GPU: sizes and refusals."""

import ctypes
import math

import pytest

from paper_2609_11582_amd import q8

FAKE = ctypes.c_void_p(4096)  # aligned, never dereferenced: validation fails first
OFF = ctypes.c_void_p(4104)


def dims(**kw):
    a = dict(batch=2, num_kv_heads=2, num_q_heads=8, num_pages=50, max_pages=20)
    a.update(kw)
    return q8.make_q8_dims(**a)


def cache(d, **kw):
    return q8.Q8Struct(d, *[kw.get(n, 4096) for n in q8.Q8_BUFFERS])


def i32(*xs):
    return (ctypes.c_int32 * len(xs))(*xs)


def test_buffer_bytes():
    d = dims(layers=3, page_tokens=128)
    got = [q8.okvq_q8_buffer_bytes(d, i) for i in range(len(q8.Q8_BUFFERS) + 1)]
    pool = 3 * 50 * 2 * 128
    assert got == [pool * 128, pool * 128, pool // 32 * 4, pool // 32 * 4, 3 * 2 * 2 * 32 * 256, 3 * 2 * 2 * 32 * 256, 2 * 20 * 4, 8,
                   200, 16, 0]


@pytest.mark.parametrize("kw, want", [
    (dict(head_dim=64), -2), (dict(batch=0), -1), (dict(batch=1025), -2), (dict(num_q_heads=7), -1),
    (dict(num_kv_heads=1, num_q_heads=17), -2), (dict(page_tokens=48), -1), (dict(page_tokens=512), -1), (dict(num_pages=0), -1),
    (dict(num_pages=(1 << 20) + 1), -2), (dict(max_pages=0), -1), (dict(max_pages=(1 << 21) + 1), -2), (dict(layers=0), -1),
    (dict(layers=4097), -2)])
def test_dims_refused(kw, want):
    d = dims(**kw)
    assert q8.okvq_q8_buffer_bytes(d, 0) == 0
    assert q8.okvq_q8_workspace_bytes(d, 100, 1) == 0
    assert q8.okvq_q8_page_workspace_bytes(d) == 0
    n = max(d.batch, 1)
    st = q8.lib().okvq_q8_append(ctypes.byref(cache(d)), 0, i32(*[5] * n), FAKE, FAKE, i32(*[1] * n), FAKE, 1, None)
    assert st == want
    assert q8.lib().okvq_q8_free(ctypes.byref(cache(d)), i32(0), 1, None) == want


def test_format_and_type_refused():
    for field, value in (("format", 2), ("dtype", 2), ("format", -1)):
        d = dims()
        setattr(d, field, value)
        assert q8.okvq_q8_buffer_bytes(d, 0) == 0


def test_append_refused():
    L, d = q8.lib(), dims()
    c = cache(d)

    def call(c=c, layer=0, lens=(10, 10), k=FAKE, v=FAKE, n=(1, 1), nd=FAKE, n_max=1):
        return L.okvq_q8_append(ctypes.byref(c), layer, i32(*lens), k, v, i32(*n), nd, n_max, None)
    assert call(layer=1) == -1 and call(layer=-1) == -1
    assert call(k=OFF) == -1 and call(v=None) == -1 and call(nd=OFF) == -1
    assert call(lens=(-1, 1)) == -1 and call(n=(2, 1)) == -1 and call(n=(-1, 0)) == -1 and call(n_max=-1) == -1
    assert call(lens=(0, 10)) == -1                     # more new tokens than tokens
    assert call(lens=(20 * 64 + 1, 1)) == -3
    for name in q8.Q8_BUFFERS:
        assert call(c=cache(d, **{name: 0})) == -1 and call(c=cache(d, **{name: 4100})) == -1
    assert call(n=(0, 0)) == 0                          # nothing to do, nothing launched
    assert L.okvq_q8_append(None, 0, i32(1, 1), FAKE, FAKE, i32(1, 1), FAKE, 1, None) == -1


def test_attention_refused():
    L, d = q8.lib(), dims()

    def call(layer=0, lens=(700, 700), q=FAKE, n=(1, 1), nd=FAKE, n_max=1, sm=0.1, out=FAKE, ws=FAKE, nbytes=1 << 40, flags=0):
        return L.okvq_q8_attention(ctypes.byref(cache(d)), layer, i32(*lens), q, i32(*n), nd, n_max, ctypes.c_float(sm), out, ws,
                                   nbytes, flags, None)
    assert call(layer=1) == -1 and call(q=OFF) == -1 and call(out=OFF) == -1 and call(nd=None) == -1
    assert call(sm=math.inf) == -1 and call(sm=math.nan) == -1 and call(flags=2) == -1
    assert call(lens=(20 * 64 + 1, 0)) == -3 and call(n=(0, 2)) == -1 and call(n=(0, -1)) == -1
    assert call(ws=None) == -4 and call(ws=OFF) == -4 and call(nbytes=100) == -4
    assert call(n=(0, 0)) == 0


def test_workspace_covers_smaller_calls():
    d = dims(batch=3, num_kv_heads=4, num_q_heads=28, max_pages=2048, num_pages=5000)
    sizes = [q8.okvq_q8_workspace_bytes(d, 131072, n) for n in (1, 2, 5, 40, 300, 4096)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert all(q8.okvq_q8_workspace_bytes(d, m, 5) <= q8.okvq_q8_workspace_bytes(d, 131072, 5) for m in (0, 1, 31, 4000))
    assert q8.okvq_q8_workspace_bytes(d, -1, 1) == 0 and q8.okvq_q8_workspace_bytes(d, 1, 0) == 0


def test_page_calls_refused():
    L, d = q8.lib(), dims(batch=4)
    c = ctypes.byref(cache(d))
    ws = q8.okvq_q8_page_workspace_bytes(d)
    assert L.okvq_q8_extend(c, OFF, FAKE, FAKE, ws, None) == -1 and L.okvq_q8_extend(c, FAKE, None, FAKE, ws, None) == -1
    assert L.okvq_q8_extend(c, FAKE, FAKE, FAKE, ws - 1, None) == -4 and L.okvq_q8_extend(c, FAKE, FAKE, None, ws, None) == -4
    assert L.okvq_q8_compact(c, FAKE, ws - 1, None) == -4 and L.okvq_q8_compact(c, OFF, ws, None) == -4
    assert L.okvq_q8_fork(c, i32(0, 0), i32(1, 1), 2, None) == -1     # a slot twice
    assert L.okvq_q8_fork(c, i32(0, 1), i32(1, 2), 2, None) == -1     # both a source and a copy
    assert L.okvq_q8_fork(c, i32(0), i32(0), 1, None) == -1
    assert L.okvq_q8_fork(c, i32(4), i32(0), 1, None) == -1 and L.okvq_q8_fork(c, i32(0), i32(-1), 1, None) == -1
    assert L.okvq_q8_fork(c, i32(0), i32(1), -1, None) == -1 and L.okvq_q8_fork(c, None, i32(1), 1, None) == -1
    assert L.okvq_q8_fork(c, i32(0, 0, 0, 0, 0), i32(1, 2, 3, 1, 2), 5, None) == -1
    assert L.okvq_q8_free(c, i32(1, 1), 2, None) == -1 and L.okvq_q8_free(c, i32(4), 1, None) == -1
    assert L.okvq_q8_free(c, None, 1, None) == -1
    assert L.okvq_q8_fork(c, None, None, 0, None) == 0 and L.okvq_q8_free(c, None, 0, None) == 0
    assert L.okvq_q8_status(c, None, None) == -1


def test_rotary_refused():
    L = q8.lib()
    par = q8.make_rotary([0.5] * 64, [0] * 64)
    ok = q8.Rows(4096, 128 * 8, 128, 128)

    def call(params=par, batch=1, hq=2, hk=2, n=4, q=ok, k=ok, pos=FAKE, lens=None, qo=ok, ko=ok, dtype=0, flags=0):
        r = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
        return L.okvq_rotary(r(params), batch, hq, hk, n, r(q), r(k), pos, lens, r(qo), r(ko), dtype, flags, None)
    assert call(params=None) == -1 and call(batch=0) == -1 and call(batch=65536) == -1 and call(n=-1) == -1
    assert call(pos=OFF) == -1 and call(pos=None) == -1 and call(dtype=2) == -1 and call(flags=4) == -1
    assert call(q=None) == -1 and call(ko=None) == -1 and call(q=None, k=None, qo=None, ko=None) == -1
    assert call(hq=0) == -1 and call(hk=0) == -1 and call(hq=65535) == -2
    assert call(lens=i32(5)) == -1 and call(lens=i32(-1)) == -1
    for bad in (q8.Rows(4104, 128, 128, 128), q8.Rows(0, 128, 128, 128), q8.Rows(4096, 4, 128, 128), q8.Rows(4096, 128, -128, 128)):
        assert call(q=bad) == -1 and call(ko=bad) == -1
    bad = q8.make_rotary([0.5] * 64, [0] * 64)
    bad.axis[3] = 3
    assert call(params=bad) == -1
    bad = q8.make_rotary([math.inf] * 64, [0] * 64)
    assert call(params=bad) == -1
    assert call(n=0) == 0
    with pytest.raises(ValueError):
        q8.make_rotary([1.0] * 63, [0] * 64)
    with pytest.raises(ValueError):
        q8.make_rotary([1.0] * 64, [3] * 64)


def test_binding_refuses_host_tensors():
    import torch
    par = q8.make_rotary([0.5] * 64, [0] * 64)
    x = torch.zeros(1, 2, 4, 128, dtype=torch.float16)
    with pytest.raises(ValueError):
        q8.okvq_rotary(par, x, None, torch.zeros(1, 3, 4, dtype=torch.int32), x, None)
    with pytest.raises(ValueError):
        q8.okvq_rotary(par, None, None, torch.zeros(1, 3, 4, dtype=torch.int32), None, None)


def test_empty_rows_may_be_null():
    """torch gives an empty tensor no address."""
    L, d = q8.lib(), dims()
    c, none = ctypes.byref(cache(d)), i32(0, 0)
    assert L.okvq_q8_append(c, 0, i32(5, 5), None, None, none, FAKE, 0, None) == 0
    assert L.okvq_q8_append(c, 0, i32(5, 5), None, FAKE, none, FAKE, 1, None) == -1
    assert L.okvq_q8_attention(c, 0, i32(5, 5), None, none, FAKE, 0, ctypes.c_float(0.1), None, FAKE, 0, 0, None) == 0
    assert L.okvq_q8_attention(c, 0, i32(5, 5), None, none, FAKE, 1, ctypes.c_float(0.1), FAKE, FAKE, 0, 0, None) == -1
    empty = ctypes.byref(q8.Rows(None, 0, 0, 0))
    par = ctypes.byref(q8.make_rotary([0.5] * 64, [0] * 64))
    assert L.okvq_rotary(par, 1, 2, 2, 0, empty, empty, None, None, empty, empty, 0, 0, None) == 0
    assert L.okvq_rotary(par, 1, 2, 2, 1, empty, empty, FAKE, None, empty, empty, 0, 0, None) == -1


def test_softmax_scale_past_the_range_of_base_two():
    d = dims()
    for sm, want in ((3.0e38, -1), (-3.0e38, -1), (2.0e38, 0)):
        st = q8.lib().okvq_q8_attention(ctypes.byref(cache(d)), 0, i32(5, 5), FAKE, i32(0, 0), FAKE, 1, ctypes.c_float(sm), FAKE, FAKE, 0, 0,
                                        None)
        assert st == want


def test_rotary_outputs_whose_rows_overlap():
    """Rows that would overwrite each other in any order: a dimension without a stride, or one within another's rows. Rows that
    lens leaves out do not count."""
    L = q8.lib()
    par = ctypes.byref(q8.make_rotary([0.5] * 64, [0] * 64))
    ok = ctypes.byref(q8.Rows(4096, 128 * 8, 128 * 4, 128))
    for batch, heads, n, bad in ((1, 2, 4, (0, 0, 128)), (1, 2, 4, (0, 512, 0)), (2, 2, 4, (0, 512, 128)), (1, 2, 4, (0, 384, 128)),
                                 (1, 2, 4, (0, 128, 128)), (1, 1, 4, (0, 0, 120)), (2, 2, 4, (960, 512, 128)), (2, 1, 2, (8, 0, 256))):
        out = ctypes.byref(q8.Rows(8192, *bad))
        for where in (dict(qo=out), dict(ko=out)):
            args = {"qo": ok, "ko": ok, **where}
            st = L.okvq_rotary(par, batch, heads, heads, n, ok, ok, FAKE, None, args["qo"], args["ko"], 0, 0, None)
            assert st == -1, (batch, heads, n, bad)
        assert L.okvq_rotary(par, batch, heads, heads, n, ok, ok, FAKE, i32(*[0] * batch), out, out, 0, 0, None) == 0


def test_attention_of_absurd_sizes():
    """Counts that no memory holds are refused, whatever the plan's arithmetic would make of them."""
    L = q8.lib()
    top = (1 << 31) - 1
    for B, H, Hq in ((1, 1, 1), (1, 1, 16), (1, 4096, 65536), (3, 64, 64), (1024, 4096, 65536)):
        d = dims(batch=B, num_kv_heads=H, num_q_heads=Hq, num_pages=1 << 20, max_pages=(1 << 27) // 64)
        for rows in (top, 1 << 30, 1 << 28):
            for n in (1 << 27, 1, 0):
                if -(-rows * Hq // H // 256) * H * 512 < 1 << 32:
                    continue  # a launch
                st = L.okvq_q8_attention(ctypes.byref(cache(d)), 0, i32(*[n] * B), FAKE, i32(*[rows] * B), FAKE, top, ctypes.c_float(0.1), FAKE,
                                         FAKE, 1 << 40, 0, None)
                assert st == -2, (B, H, Hq, rows, n)
