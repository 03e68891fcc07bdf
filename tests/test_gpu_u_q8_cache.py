"""The paged 8-bit cache against oracle.q8: codec bytes, attention, page calls, and all of them together.

Codes and scales are compared bit for bit (the fp32 order is the contract). Attention is held to the bound that
oracle.q8.attention derives from the kernels' roundings."""

import math

import numpy as np
import pytest

from oracle import q8 as oq

pytestmark = pytest.mark.gpu
SM = 1 / math.sqrt(128)
HALF = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def _new(B, H, Hq, lens, page=64, fmt="int8", dtype="fp16", layers=1, spare=3, seed=0, room=0):
    """A cache whose pages are dealt in shuffled order to sequences of these lengths; unused pages and scales hold
    bytes that would show (NaN)."""
    import torch

    import paper_2609_11582_amd as okvq
    need = [-(-n // page) for n in lens]
    P, mp = sum(need) + spare, max(max(need), 1) + room
    c = okvq.Q8Cache(B, H, Hq, P, mp, layers=layers, page_tokens=page, format=fmt, dtype=dtype)
    for f in ("k_codes", "v_codes"):
        c[f].fill_(0x7f)
    for f in ("k_scale", "v_scale", "k_stage", "v_stage"):
        c[f].fill_(float("nan"))
    order = np.random.default_rng(seed).permutation(P)
    at = 0
    for b, m in enumerate(need):
        c["block_table"][b, :m] = torch.from_numpy(order[at:at + m].astype(np.int32))
        at += m
    c["page_refs"][torch.from_numpy(order[:at].copy())] = 1
    return c


def _rows(seed, *shape, dtype="fp16", scale=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, generator=g) * scale
    return x.to(torch.float16 if dtype == "fp16" else torch.bfloat16)


def _i32(xs):
    import torch
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _append(c, layer, k, v, old, new):
    """The rows old[b] .. old[b] + new[b] of k, v [B][H][N][128]; the lengths are set first, as extend does."""
    import torch

    import paper_2609_11582_amd as okvq
    B, H, _, D = k.shape
    n = max(max(new), 1)
    kn, vn = (torch.full((B, H, n, D), float("nan"), dtype=k.dtype) for _ in range(2))
    for b in range(B):
        kn[b, :, :new[b]], vn[b, :, :new[b]] = (x[b, :, old[b]:old[b] + new[b]] for x in (k, v))
    lens = [a + m for a, m in zip(old, new)]
    c["seq_lens"].copy_(_i32(lens))
    okvq.okvq_q8_append(c, layer, lens, kn.cuda(), vn.cuda(), new, _i32(new), n)
    return lens


def _numpy(c):
    import torch
    torch.cuda.synchronize()
    return {f: (c[f].float() if f.endswith("stage") else c[f]).cpu().numpy() for f in c.buffers}


def _check_bytes(a, k, v, lens, fmt, layer=0):
    T = a["k_codes"].shape[3]
    for b, L in enumerate(lens):
        for h in range(k.shape[1]):
            for t0 in range(0, L, 32):
                page, sub = a["block_table"][b, t0 // T], t0 % T // 32
                where = f"sequence {b} head {h} token {t0}"
                code, scale = oq.quantize_block(k[b, h, t0:min(t0 + 32, L)].float().numpy(), fmt)
                assert a["k_scale"][layer, page, h, sub] == scale, where
                assert np.array_equal(a["k_codes"][layer, page, h, sub * 32:sub * 32 + 32], code), where
                code, scale = oq.quantize_block(v[b, h, t0:min(t0 + 32, L)].float().numpy(), fmt)
                assert a["v_scale"][layer, page, h, sub] == scale, where
                assert np.array_equal(a["v_codes"][layer, page, h, sub], oq.pack_values(code)), where
            r = L % 32
            assert np.array_equal(a["k_stage"][layer, b, h, :r], k[b, h, L - r:L].float().numpy())
            assert np.array_equal(a["v_stage"][layer, b, h, :r], v[b, h, L - r:L].float().numpy())


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("page, lens, plan", [
    (32, [70, 0, 1], [[1000] * 3]),
    (64, [131, 64, 33], [[1] * 3] * 3 + [[29] * 3, [1000] * 3]),
    (128, [257, 100, 31], [[20, 100, 31], [7] * 3, [70] * 3, [1000] * 3]),
    (256, [300, 32, 255], [[33] * 3, [0, 1, 200], [1000] * 3]),
])
def test_append_bytes(fmt, dtype, page, lens, plan):
    _say(f"append {fmt} {dtype} page {page} {lens}")
    B, H = 3, 2
    c = _new(B, H, H, lens, page, fmt, dtype)
    k, v = _rows(1, B, H, max(lens), 128, dtype=dtype), _rows(2, B, H, max(lens), 128, dtype=dtype, scale=30)
    k[:, :, :, 5] *= 20
    k[0, 0, 32:64] = 0                               # a block of zeros
    v[0, 1, 3, 7] = 60000
    v[2, 0] *= 2.0 ** -20                            # fp16 subnormals
    cur = [0] * B
    for step in plan:
        new = [min(s, L - n) for s, L, n in zip(step, lens, cur)]
        if max(new):
            cur = _append(c, 0, k, v, cur, new)
    assert cur == lens
    a = _numpy(c)
    _check_bytes(a, k, v, lens, fmt)
    free = np.flatnonzero(a["page_refs"] == 0)
    assert np.all(a["k_codes"][0, free] == 0x7f) and np.all(np.isnan(a["k_scale"][0, free]))


def test_append_extreme_scales():
    import torch
    B, H, n = 1, 1, 64
    for fmt in ("int8", "e4m3"):
        for top in (3e38, 1e-37, 1e-40):  # bf16: amax / M overflows nothing, and becomes subnormal
            _say(f"append {fmt} amax {top}")
            c = _new(B, H, H, [n], fmt=fmt, dtype="bf16")
            k = (_rows(3, B, H, n, 128, dtype="fp16").double().clamp(-1, 1) * top).to(torch.bfloat16)
            _append(c, 0, k, k, [0], [n])
            _check_bytes(_numpy(c), k, k, [n], fmt)


def test_append_layers_keep_apart():
    c = _new(2, 1, 1, [40, 70], layers=3)
    k, v = _rows(4, 2, 1, 70, 128), _rows(5, 2, 1, 70, 128)
    _append(c, 1, k, v, [0, 0], [40, 70])
    a = _numpy(c)
    _check_bytes(a, k, v, [40, 70], "int8", layer=1)
    for layer in (0, 2):
        assert np.all(a["k_codes"][layer] == 0x7f) and np.all(a["v_codes"][layer] == 0x7f) and np.all(np.isnan(a["k_stage"][layer]))


# ---- attention -----------------------------------------------------------------------------------


def _filled(B, H, Hq, lens, page, fmt, dtype, seed, drift=0.3, layers=1, layer=0):
    import torch
    c = _new(B, H, Hq, lens, page, fmt, dtype, layers=layers, seed=seed)
    n = max(max(lens), 1)
    g = torch.Generator().manual_seed(seed)
    walk = (drift * torch.randn(B, H, -(-n // 64), 128, generator=g)).cumsum(2).repeat_interleave(64, 2)[:, :, :n]
    k = (torch.randn(B, H, n, 128, generator=g) + walk).to(c.row_dtype)
    v = (torch.randn(B, H, n, 128, generator=g) * torch.exp(torch.randn(B, H, n, 1, generator=g))).to(c.row_dtype)
    _append(c, layer, k, v, [0] * B, lens)
    return c


def _attend(c, lens, q, new, cross=False, sm=SM, layer=0, fill=9.0, stream=None):
    import torch

    import paper_2609_11582_amd as okvq
    B, Hq, n, _ = q.shape
    out = torch.full((B, Hq, n, 128), fill, dtype=c.row_dtype, device="cuda")
    ws = okvq.q8_workspace(c.dims, max(lens), n)
    okvq.okvq_q8_attention(c, layer, lens, q.cuda(), new, _i32(new), n, sm, out, ws, flags=okvq.OKVQ_Q8_CROSS if cross else 0)
    return out


def _check_attention(c, out, lens, q, new, fmt, dtype, tag, cross=False, sm=SM, layer=0, fill=9.0, rows=None):
    a = _numpy(c)
    got = out.double().cpu().numpy()
    B, Hq, n, _ = q.shape
    H = c.dims.num_kv_heads
    G, worst = Hq // H, 0.0
    for b in range(B):
        assert np.all(got[b, :, new[b]:] == fill), f"{tag}: rows behind the last one were written"
        pick = np.arange(new[b]) if rows is None else np.unique(np.clip(rows, 0, new[b] - 1)) if new[b] else np.arange(0)
        seen = np.full(len(pick), lens[b]) if cross else lens[b] - new[b] + pick + 1
        for h in range(H):
            k, v = oq.read_sequence(a, layer, b, h, lens[b], fmt)
            for j in range(h * G, (h + 1) * G):
                ref, bound = oq.attention(q[b, j, pick].double().numpy(), k, v, seen, sm, HALF[dtype])
                r = np.abs(got[b, j, pick] - ref) / np.maximum(bound, 1e-30) if len(pick) else np.zeros(1)
                assert np.all(got[b, j, pick][seen <= 0] == 0), f"{tag}: a row that sees nothing yields zeros"
                worst = max(worst, float(np.nanmax(r)) if np.isfinite(got[b, j, pick]).all() else math.inf)
    _say(f"{tag}: worst err / bound {worst:.3f}")
    assert worst <= 1


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("H, Hq, page, lens", [
    (2, 14, 64, [0, 1, 31, 32, 33, 64, 65, 500]),
    (1, 1, 32, [97, 5]),
    (1, 16, 256, [700, 256]),
    (3, 12, 128, [1300]),
    (4, 32, 64, [2049, 2050, 17]),
])
def test_one_token(fmt, dtype, H, Hq, page, lens):
    B = len(lens)
    c = _filled(B, H, Hq, lens, page, fmt, dtype, 11)
    q = _rows(12, B, Hq, 1, 128, dtype=dtype, scale=2.0)
    new = [1] * B
    out = _attend(c, lens, q, new)
    _check_attention(c, out, lens, q, new, fmt, dtype, f"one token {fmt} {dtype} H={H} Hq={Hq} page={page} {lens}")


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("H, Hq, lens, new, cross", [
    (1, 4, [40], [40], False),                       # a whole prompt
    (2, 14, [129, 64, 200, 31], [129, 3, 0, 31], False),
    (1, 7, [300, 301], [17, 2], False),
    (1, 3, [100, 5, 2], [12, 12, 12], False),        # more rows than tokens: the first ones see nothing
    (2, 2, [77, 0, 1], [50, 50, 33], True),          # an encoder's states, one of them empty
    (1, 16, [260], [70], True),
    (1, 8, [1500, 1025], [130, 128], False),
    (2, 6, [3000], [2], False),
    (1, 5, [2500, 2400], [23, 20], False),           # few rows against long sequences
    (1, 1, [700], [650], False),
])
def test_chunks(fmt, dtype, H, Hq, lens, new, cross):
    B, n = len(lens), max(new)
    c = _filled(B, H, Hq, lens, 64, fmt, dtype, 13)
    q = _rows(14, B, Hq, n + 1, 128, dtype=dtype, scale=1.5)  # a row more than any sequence has
    for b in range(B):
        q[b, :, new[b]:] = float("nan")
    out = _attend(c, lens, q, new, cross)
    _check_attention(c, out, lens, q, new, fmt, dtype, f"chunk {fmt} {dtype} Hq={Hq} {lens} {new} cross={cross}", cross)


@pytest.mark.parametrize("n_q", [1, 40])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_dominant_tokens_and_uneven_values(fmt, n_q):
    """A flat background with tokens 10 to 30 log2 units above it, growing and falling along the sequence, whose values
    are small where attention is large (and the other way round)."""
    import torch
    n = 6000
    for case in range(4):
        c = _new(1, 1, 2, [n], 64, fmt)
        g = torch.Generator().manual_seed(20 + case)
        k = 0.01 * torch.randn(1, 1, n, 128, generator=g)
        v = 0.01 * torch.randn(1, 1, n, 128, generator=g) + 1.0
        at = torch.arange(0, n, 512)
        up = torch.linspace(10, 30, len(at)) if case % 2 else torch.linspace(30, 10, len(at))
        k[0, 0, at, 0] = up
        v[0, 0] *= torch.where(torch.arange(n) % 512 < 32, 2.0 ** -9 if case < 2 else 2.0 ** 9, 1.0)[:, None]
        k, v = k.half(), v.half()
        _append(c, 0, k, v, [0], [n])
        q = torch.zeros(1, 2, n_q, 128)
        q[:, :, :, 0] = math.log(2.0) / SM  # scores are the first channel, in log2 units
        q[:, 1] *= 0.3
        q = q.half()
        out = _attend(c, [n], q, [n_q])
        _check_attention(c, out, [n], q, [n_q], fmt, "fp16", f"dominant {fmt} case {case} rows {n_q}", rows=np.array([0, n_q - 1]))


@pytest.mark.parametrize("sm", [0.0, -0.05, 3.0])
def test_softmax_scales(sm):
    lens = [333, 40]
    c = _filled(2, 1, 4, lens, 64, "int8", "fp16", 31)
    for n in (1, 20):
        q = _rows(32, 2, 4, n, 128)
        new = [n, n]
        out = _attend(c, lens, q, new, sm=sm)
        _check_attention(c, out, lens, q, new, "int8", "fp16", f"scale {sm} rows {n}", sm=sm)


def test_bf16_range():
    """bfloat16 queries and values far outside fp16's range."""
    import torch
    n = 200
    for fmt in ("int8", "e4m3"):
        for qs, vs in ((1e-20, 1e30), (1e20, 1e-30)):
            c = _new(1, 1, 2, [n], 64, fmt, "bf16")
            k = _rows(41, 1, 1, n, 128).double() / qs
            v = _rows(42, 1, 1, n, 128).double() * vs
            _append(c, 0, k.to(torch.bfloat16), v.to(torch.bfloat16), [0], [n])
            for m in (1, 33):
                q = (_rows(43, 1, 2, m, 128).double() * qs).to(torch.bfloat16)
                out = _attend(c, [n], q, [m])
                a = _numpy(c)
                kk, vv = oq.read_sequence(a, 0, 0, 0, n, fmt)
                for j in range(2):
                    ref, bound = oq.attention(q[0, j].double().numpy(), kk, vv / vs, n - m + np.arange(m) + 1, SM, HALF["bf16"])
                    r = np.abs(out[0, j].double().cpu().numpy() / vs - ref) / bound
                    _say(f"bf16 range {fmt} q {qs} v {vs} rows {m}: worst err / bound {r.max():.3f}")
                    assert r.max() <= 1


def test_long_sequence_in_an_upper_layer():
    n = 131072
    c = _filled(1, 1, 8, [n], 256, "e4m3", "bf16", 51, drift=0.01, layers=2, layer=1)
    for m in (1, 24):
        q = _rows(52, 1, 8, m, 128, dtype="bf16")
        out = _attend(c, [n], q, [m], layer=1)
        _check_attention(c, out, [n], q, [m], "e4m3", "bf16", f"131072 tokens, {m} rows", layer=1, rows=np.array([0, 23]))


# ---- page calls ----------------------------------------------------------------------------------


def _pages_equal(c, m):
    a = _numpy(c)
    for f, want in m.arrays().items():
        assert np.array_equal(a[f], want), (f, a[f], want)
    return a


@pytest.mark.parametrize("page, layers, H", [(32, 1, 1), (64, 3, 2), (256, 2, 5)])
def test_page_calls_follow_the_model(page, layers, H):
    import torch

    import paper_2609_11582_amd as okvq
    B, P, mp = 6, 37, 9
    c = okvq.Q8Cache(B, H, H, P, mp, layers=layers, page_tokens=page)
    m = oq.PagedModel(B, P, page, mp)
    ws = okvq.q8_page_workspace(c.dims)
    pools = ("k_codes", "v_codes", "k_scale", "v_scale")
    g = torch.Generator(device="cuda").manual_seed(page)
    for f in pools + ("k_stage", "v_stage"):
        c[f].copy_(torch.randint(0, 100, c[f].shape, generator=g, device="cuda"))
    rng = np.random.default_rng(page)
    granted = torch.zeros(B, dtype=torch.int32, device="cuda")
    for step in range(120):
        before = {f: c[f].clone() for f in pools + ("k_stage", "v_stage")}
        kind = int(rng.integers(5))
        moves = []
        if kind <= 1:
            more = [int(x) if rng.random() < 0.6 else 0 for x in rng.integers(0, 3 * page, B)]
            more[int(rng.integers(B))] = -3
            okvq.okvq_q8_extend(c, _i32(more), granted, ws)
            want = m.extend(more)
            moves = m.moves
            assert granted.tolist() == want, (step, more)
        elif kind == 2:
            order = rng.permutation(B).tolist()
            dst = order[:int(rng.integers(1, 4))]
            src = [order[int(rng.integers(3, B))] for _ in dst]
            okvq.okvq_q8_fork(c, src, dst)
            m.fork(src, dst)
            for s, d in zip(src, dst):
                for f in ("k_stage", "v_stage"):
                    r = m.lens[s] % 32
                    before[f][:, d, :, :r] = before[f][:, s, :, :r]
        elif kind == 3:
            slots = rng.permutation(B)[:int(rng.integers(1, 3))].tolist()
            okvq.okvq_q8_free(c, slots)
            m.free(slots)
        else:
            okvq.okvq_q8_compact(c, ws)
            n = m.compact()
            moves = m.moves
            assert okvq.okvq_q8_status(c) == (m.short, n)
        for a, b in moves:
            for f in pools:
                before[f][:, b] = before[f][:, a]
        _pages_equal(c, m)
        for f, want in before.items():
            assert torch.equal(c[f], want), (step, kind, f)
    assert okvq.okvq_q8_status(c)[0] == m.short == 1


def test_extend_of_shared_pages_in_one_call():
    import paper_2609_11582_amd as okvq
    B, P = 5, 12
    for more in ([1, 1, 1, 1, 0], [0, 2, 3, 0, 1], [1, 0, 0, 0, 0], [70, 70, 1, 1, 1]):
        c = okvq.Q8Cache(B, 1, 1, P, 6)
        m = oq.PagedModel(B, P, 64, 6)
        ws, granted = okvq.q8_page_workspace(c.dims), _i32([0] * B)
        for call in ([100, 0, 0, 0, 0], more):
            okvq.okvq_q8_extend(c, _i32(call), granted, ws)
            m.extend(call)
            _pages_equal(c, m)
            if call is not more:
                okvq.okvq_q8_fork(c, [0, 0, 0, 0], [1, 2, 3, 4])
                m.fork([0] * 4, [1, 2, 3, 4])
        assert granted.tolist() == more


def test_extend_grants_all_or_nothing():
    import paper_2609_11582_amd as okvq
    c = okvq.Q8Cache(3, 1, 1, 4, 3)
    m = oq.PagedModel(3, 4, 64, 3)
    ws, granted = okvq.q8_page_workspace(c.dims), _i32([7] * 3)
    for more, ok in (([65, 64, 1], True), ([0, 1, 0], False), ([0, 0, 63], True), ([64, 0, 0], False), ([63, 0, 0], True),
                     ([(1 << 31) - 1] * 3, False), ([0, 0, 0], True)):
        okvq.okvq_q8_extend(c, _i32(more), granted, ws)
        assert granted.tolist() == m.extend(more) == (more if ok else [0] * 3)
        _pages_equal(c, m)
    c = okvq.Q8Cache(1, 1, 1, 9, 2)  # pages enough, but not table entries
    okvq.okvq_q8_extend(c, _i32([129]), granted, okvq.q8_page_workspace(c.dims))
    assert granted[0] == 0 and okvq.okvq_q8_status(c)[0] == 1 and int(c["seq_lens"][0]) == 0


def test_largest_batch_and_many_pages():
    import paper_2609_11582_amd as okvq
    B, P = 1024, 20000
    c = okvq.Q8Cache(B, 1, 1, P, 30, page_tokens=32)
    m = oq.PagedModel(B, P, 32, 30)
    ws, granted = okvq.q8_page_workspace(c.dims), _i32([0] * B)
    rng = np.random.default_rng(3)
    for step in range(3):
        more = rng.integers(0, 200, B).tolist()
        okvq.okvq_q8_extend(c, _i32(more), granted, ws)
        assert granted.tolist() == m.extend(more)
        slots = rng.permutation(B)[:600].tolist()
        okvq.okvq_q8_free(c, slots)
        m.free(slots)
        rest = [b for b in range(B) if b not in set(slots)]
        okvq.okvq_q8_fork(c, [rest[i % len(rest)] for i in range(300)], slots[:300])
        m.fork([rest[i % len(rest)] for i in range(300)], slots[:300])
        okvq.okvq_q8_compact(c, ws)
        m.compact()
        _pages_equal(c, m)


# ---- together ------------------------------------------------------------------------------------


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
def test_samples_of_one_prompt(fmt, dtype):
    """A prompt, forked into samples that go on apart (pages copied on write), one freed, the pool compacted, and on."""
    import torch

    import paper_2609_11582_amd as okvq
    H, Hq, S, n0, layers = 2, 6, 4, 77, 2
    rot = okvq.make_rotary([1e6 ** (-i / 64) for i in range(64)], [i % 3 for i in range(64)])
    c = okvq.Q8Cache(S, H, Hq, 40, 8, layers=layers, format=fmt, dtype=dtype)
    dt = c.row_dtype
    g = torch.Generator().manual_seed(61)
    prompt = [torch.randn(1, h, n0, 128, generator=g).to(dt) for h in (H, H, Hq)]
    tail = [torch.randn(S, h, 60, 128, generator=g).to(dt) for h in (H, H, Hq)]
    pos = torch.randint(0, 4000, (S, 3, n0 + 60), generator=g).to(torch.int32)
    pos[1:, :, :n0] = pos[:1, :, :n0]
    ws, granted = okvq.q8_page_workspace(c.dims), _i32([0] * S)
    # the prompt in slot 0 alone
    new = [n0] + [0] * (S - 1)
    k, v, q = (torch.cat([x, x.new_zeros(S - 1, *x.shape[1:])]).cuda() for x in prompt)
    okvq.okvq_rotary(rot, q, k, pos[:, :, :n0].contiguous().cuda(), q, k, lens=new)
    okvq.okvq_q8_extend(c, _i32(new), granted, ws)
    for layer in range(layers):
        okvq.okvq_q8_append(c, layer, new, k, v, new, granted, n0)
    okvq.okvq_q8_fork(c, [0] * (S - 1), list(range(1, S)))
    raw = [[x[:1].cpu() for _ in range(S)] for x in (k, v)]  # the rotated rows that each sample has cached
    lens = [n0] * S
    at = 0
    for step, n in enumerate([1, 1, 30, 1, 3, 1]):
        if step == 3:
            okvq.okvq_q8_free(c, [2])
            okvq.okvq_q8_fork(c, [0], [2])
            raw[0][2], raw[1][2] = raw[0][0], raw[1][0]
        if step == 4:
            okvq.okvq_q8_compact(c, ws)
        kk, vv, qq = (x[:, :, at:at + n].contiguous().cuda() for x in tail)
        okvq.okvq_rotary(rot, qq, kk, pos[:, :, n0 + at:n0 + at + n].contiguous().cuda(), qq, kk)
        new = [n] * S
        lens = [x + n for x in lens]
        okvq.okvq_q8_extend(c, _i32(new), granted, ws)
        assert granted.tolist() == new
        for layer in range(layers):
            okvq.okvq_q8_append(c, layer, lens, kk, vv, new, granted, n)
            out = torch.full_like(qq, 9.0)
            okvq.okvq_q8_attention(c, layer, lens, qq, new, granted, n, SM, out, okvq.q8_workspace(c.dims, max(lens), n))
        for b in range(S):
            raw[0][b] = torch.cat([raw[0][b], kk[b:b + 1].cpu()], 2)
            raw[1][b] = torch.cat([raw[1][b], vv[b:b + 1].cpu()], 2)
        a = _numpy(c)
        for layer in range(layers):
            _check_bytes(a, torch.cat(raw[0]), torch.cat(raw[1]), lens, fmt, layer)
        _check_attention(c, out, lens, qq.cpu(), new, fmt, dtype, f"samples {fmt} step {step}", layer=layers - 1)
        at += n
    assert okvq.okvq_q8_status(c)[0] == 0


def test_captured_step_grows_with_the_sequences():
    """One decode step captured and replayed: the kernels read lengths and tables on the device. Every replay is compared
    with an eager twin of the cache, with work of the program's own in between."""
    import torch

    import paper_2609_11582_amd as okvq
    B, H, Hq, n0 = 3, 2, 8, 61
    rot = okvq.make_rotary([1e4 ** (-i / 64) for i in range(64)], [0] * 64)
    caches = [okvq.Q8Cache(B, H, Hq, 40, 8) for _ in range(2)]
    k0, v0 = _rows(71, B, H, n0, 128).cuda(), _rows(72, B, H, n0, 128).cuda()
    state = []
    for c in caches:
        ws, granted = okvq.q8_page_workspace(c.dims), _i32([0] * B)
        okvq.okvq_q8_extend(c, _i32([n0, 5, 32]), granted, ws)
        okvq.okvq_q8_append(c, 0, [n0, 5, 32], k0, v0, [n0, 5, 32], granted, n0)
        okvq.okvq_q8_fork(c, [0], [1])
        state.append((ws, granted))
    one = _i32([1] * B)
    k, v, q = (torch.zeros(B, h, 1, 128, dtype=torch.float16, device="cuda") for h in (H, H, Hq))
    pos = torch.zeros(B, 3, 1, dtype=torch.int32, device="cuda")

    def step(c, ws, granted, aws, qr, kr, out, lens):
        okvq.okvq_rotary(rot, q, k, pos, qr, kr)
        okvq.okvq_q8_extend(c, one, granted, ws)
        okvq.okvq_q8_append(c, 0, lens, kr, v, [1] * B, granted, 1)
        okvq.okvq_q8_attention(c, 0, lens, qr, [1] * B, granted, 1, SM, out, aws)
    buf = [(torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(q)) for _ in caches]
    aws = [okvq.q8_workspace(c.dims, 512) for c in caches]
    plan = [300] * B  # the capture's host lengths plan for what is to come
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(caches[0], *state[0], aws[0], *buf[0], plan)
    lens = [n0, n0, 32]
    for t in range(70):  # across block and page borders, and the first copies on write
        x = _rows(100 + t, 3, B, Hq, 1, 128).cuda()
        q.copy_(x[0])
        k.copy_(x[1][:, :H])
        v.copy_(x[2][:, :H])
        pos.fill_(n0 + t)
        graph.replay()
        lens = [n + 1 for n in lens]
        step(caches[1], *state[1], aws[1], *buf[1], plan)
        for f in caches[0].buffers:
            assert torch.equal(caches[0][f].view(torch.uint8), caches[1][f].view(torch.uint8)), (t, f)
        assert torch.equal(buf[0][2], buf[1][2]), t
        torch.cuda.synchronize()
    assert caches[0]["seq_lens"].tolist() == lens
    _check_attention(caches[0], buf[0][2], lens, buf[0][0].cpu(), [1] * B, "int8", "fp16", "captured step")


def test_another_stream_and_a_given_stream():
    import torch

    import paper_2609_11582_amd as okvq
    lens = [500, 300]
    c = _filled(2, 2, 8, lens, 64, "int8", "fp16", 81)
    q = _rows(82, 2, 8, 1, 128).cuda()
    want = _attend(c, lens, q, [1, 1])
    side = torch.cuda.Stream()
    out, ws, one = torch.zeros_like(q), okvq.q8_workspace(c.dims, 500), _i32([1, 1])
    side.wait_stream(torch.cuda.current_stream())
    okvq.okvq_q8_attention(c, 0, lens, q, [1, 1], one, 1, SM, out, ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        okvq.okvq_q8_attention(c, 0, lens, q, [1, 1], one, 1, SM, out, ws)
    side.synchronize()
    assert torch.equal(out, want)


def test_repeated_calls_are_equal():
    import torch
    lens = [9000, 8000]
    c = _filled(2, 1, 8, lens, 64, "int8", "fp16", 91)
    for n in (1, 50):
        q = _rows(92, 2, 8, n, 128)
        first = _attend(c, lens, q, [n, n])
        assert all(torch.equal(first, _attend(c, lens, q, [n, n])) for _ in range(3))


def test_binding_refuses():
    import torch

    import paper_2609_11582_amd as okvq
    lens = [40]
    c = _filled(1, 1, 4, lens, 64, "int8", "fp16", 95)
    q, one = _rows(96, 1, 4, 1, 128).cuda(), _i32([1])
    ws = okvq.q8_workspace(c.dims, 40)
    out = torch.zeros_like(q)

    def call(q=q, n=[1], nd=one, out=out, ws=ws, lens=lens, n_max=1):
        okvq.okvq_q8_attention(c, 0, lens, q, n, nd, n_max, SM, out, ws)
    call()
    for kw in (dict(q=q.cpu()), dict(q=q.bfloat16()), dict(out=out.float()), dict(nd=one.long()), dict(lens=[40, 1]), dict(n=[1, 1]),
               dict(n_max=2), dict(q=q.repeat(1, 1, 1, 2)[..., ::2]), dict(ws=ws.cpu())):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(okvq.OkvqError):
        call(n=[2])
    with pytest.raises(ValueError):
        okvq.Q8Cache(1, 1, 1, 4, 2, buffers={f: t.cpu() for f, t in okvq.Q8Cache(1, 1, 1, 4, 2).buffers.items()})
    with pytest.raises(okvq.OkvqError):
        okvq.Q8Cache(1, 1, 17, 4, 2)


@pytest.mark.parametrize("n_q", [1, 40])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_blocks_of_zero_values(fmt, n_q):
    """Blocks of zero values (scale 1) that take most of the attention, among blocks of tiny values."""
    import torch
    n = 1000
    c = _new(1, 1, 2, [n], 64, fmt)
    g = torch.Generator().manual_seed(7)
    k, v = 0.1 * torch.randn(1, 1, n, 128, generator=g), 1e-4 * torch.randn(1, 1, n, 128, generator=g)
    k[0, 0, 32:64, 0] += 8.0
    v[0, 0, 32:64] = 0.0
    v[0, 0, 320:352] = -0.0
    k, v = k.half(), v.half()
    _append(c, 0, k, v, [0], [n])
    q = torch.zeros(1, 2, n_q, 128)
    q[:, :, :, 0] = math.log(2.0) / SM
    q[:, 1] = 0.0
    q = q.half()
    out = _attend(c, [n], q, [n_q])
    a = _numpy(c)
    kk, vv = oq.read_sequence(a, 0, 0, 0, n, fmt)
    for j in range(2):
        ref, bound = oq.attention(q[0, j].double().numpy(), kk, vv, n - n_q + np.arange(n_q) + 1, SM, HALF["fp16"])
        r = np.abs(out[0, j].double().cpu().numpy() - ref) / bound
        _say(f"zero blocks {fmt} rows {n_q} head {j}: worst err / bound {r.max():.3f}")
        assert r.max() <= 1


@pytest.mark.parametrize("n_q", [1, 30])
def test_pool_beyond_32_bits(n_q):
    """Pages whose codes lie past 2^32 bytes of a pool, in the second layer, against the same rows in a small cache."""
    import torch

    import paper_2609_11582_amd as okvq
    H, Hq, P, n = 8, 16, 9000, 700
    k, v, q = _rows(101, 1, H, n, 128), _rows(102, 1, H, n, 128), _rows(103, 1, Hq, n_q, 128)
    outs = []
    for pages, layers in ((P, 2), (20, 1)):
        c = okvq.Q8Cache(1, H, Hq, pages, 4, layers=layers, page_tokens=256)
        c["block_table"][0, :3] = _i32([pages - 1, pages - 3, pages - 2])
        _append(c, layers - 1, k, v, [0], [n])
        outs.append((_attend(c, [n], q, [n_q], layer=layers - 1), c["k_codes"][-1, -1].clone(), c["v_codes"][-1, -3].clone()))
    assert 2 * P * H * 256 * 128 > 1 << 32 and (P - 1) * H * 256 * 128 * 2 > 1 << 32
    assert all(torch.equal(x, y) for x, y in zip(*outs))


def test_two_graphs_and_two_streams():
    """Two captured steps with workspaces of their own, replayed on two streams at once, several times."""
    import torch

    import paper_2609_11582_amd as okvq
    B, H, Hq, lens = 2, 2, 14, [5000, 3000]
    sides, want = [], []
    for i in range(2):
        c = _filled(B, H, Hq, lens, 64, "int8", "fp16", 110 + i)
        q = _rows(120 + i, B, Hq, 1 + 20 * i, 128).cuda()
        n = q.shape[2]
        want.append(_attend(c, lens, q, [n] * B))
        out, ws, new = torch.zeros_like(q), okvq.q8_workspace(c.dims, 5000, n), _i32([n] * B)
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            okvq.okvq_q8_attention(c, 0, lens, q, [n] * B, new, n, SM, out, ws)
        sides.append((stream, graph, out, c, q, ws, new))
    for t in range(5):
        for _, _, out, *_ in sides:
            out.fill_(t)
        torch.cuda.synchronize()
        for stream, graph, *_ in sides:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for (_, _, out, *_), ref in zip(sides, want):
            assert torch.equal(out, ref), t


def test_lengths_on_the_device_rule():
    """Host lengths only plan: a plan for shorter, longer or empty sequences gives the same rows up to the roundings of
    another number of splits."""
    import torch

    import paper_2609_11582_amd as okvq
    lens = [2500, 900, 1]
    c = _filled(3, 1, 4, lens, 64, "int8", "fp16", 130)
    for n in (1, 24):
        q = _rows(131, 3, 4, n, 128)
        new, nd = [min(n, m) for m in lens], _i32([min(n, m) for m in lens])
        ws = okvq.q8_workspace(c.dims, 2560, n)
        for plan in ([0, 0, 0], [2560, 2560, 2560], [100, 1, 2000]):
            out = torch.full(q.shape, 9.0, dtype=torch.float16, device="cuda")
            okvq.okvq_q8_attention(c, 0, plan, q.cuda(), new, nd, n, SM, out, ws)
            _check_attention(c, out, lens, q, new, "int8", "fp16", f"planned as {plan}, rows {n}")


def test_counts_of_numpy():
    import paper_2609_11582_amd as okvq
    c = okvq.Q8Cache(2, 1, 1, 10, 4)
    k = _rows(140, 2, 1, 33, 128)
    lens = np.array([33, 20], np.int64)
    c["block_table"][:, 0] = _i32([3, 4])
    c["seq_lens"].copy_(_i32(lens.tolist()))
    okvq.okvq_q8_append(c, np.int64(0), lens, k.cuda(), k.cuda(), np.array([33, 20]), _i32([33, 20]), np.int32(33))
    _check_bytes(_numpy(c), k, k, [33, 20], "int8")


@pytest.mark.parametrize("n_q", [1, 150])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_value_scales_far_apart(fmt, n_q):
    """Blocks of bfloat16 values whose scales lie 2^150 apart share the attention: the small ones count in the softmax sum."""
    import torch
    n = 400
    c = _new(1, 1, 2, [n], 64, fmt, "bf16")
    large = (torch.arange(n) // 32 % 3 == 1)[:, None]
    k = _rows(61, 1, 1, n, 128, dtype="bf16")
    v = (torch.where(large, 2.0 ** 75, 2.0 ** -75) * _rows(62, 1, 1, n, 128).double()).to(torch.bfloat16)
    _append(c, 0, k, v, [0], [n])
    q = _rows(63, 1, 2, n_q, 128, dtype="bf16")
    out = _attend(c, [n], q, [n_q])
    a = _numpy(c)
    kk, vv = oq.read_sequence(a, 0, 0, 0, n, fmt)
    for j in range(2):
        ref, bound = oq.attention(q[0, j].double().numpy(), kk, vv / 2.0 ** 75, n - n_q + np.arange(n_q) + 1, SM, HALF["bf16"])
        r = np.abs(out[0, j].double().cpu().numpy() / 2.0 ** 75 - ref) / bound
        _say(f"far scales {fmt} rows {n_q} head {j}: worst err / bound {r.max():.3f}")
        assert r.max() <= 1


@pytest.mark.parametrize("n_q", [1, 150])
def test_small_weights_of_large_values(n_q):
    """A block with weights of 2^-100 whose values are 2^180 times the others': its products are the largest by 2^80. It
    is met by the wave that has the dominant block (every eighth is the same wave's), before it and after it."""
    import torch
    n = 320
    for dominant, far in ((0, 8), (9, 1)):
        c = _new(1, 1, 1, [n], 32, "int8", "bf16")
        k = torch.zeros(1, 1, n, 128)
        k[0, 0, 32 * dominant:32 * dominant + 32, 0] = 100.0
        v = 2.0 ** -90 * _rows(65, 1, 1, n, 128).double()
        v[0, 0, 32 * far:32 * far + 32] *= 2.0 ** 180
        _append(c, 0, k.to(torch.bfloat16), v.to(torch.bfloat16), [0], [n])
        q = torch.zeros(1, 1, n_q, 128)
        q[..., 0] = 1.0
        out = _attend(c, [n], q.to(torch.bfloat16), [n_q], cross=True, sm=math.log(2.0))  # scores: the first channel, in log2 units
        kk, vv = oq.read_sequence(_numpy(c), 0, 0, 0, n, "int8")
        ref, bound = oq.attention(q[0, 0].double().numpy(), kk, vv * 2.0 ** 10, np.full(n_q, n), math.log(2.0), HALF["bf16"])
        r = np.abs(out[0, 0].double().cpu().numpy() * 2.0 ** 10 - ref) / bound
        _say(f"small weights rows {n_q} dominant block {dominant}: largest {np.abs(ref).max():.3f}, worst err / bound {r.max():.3f}")
        assert r.max() <= 1


@pytest.mark.parametrize("case", ["dominant", "zero blocks"])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_uneven_values_many_rows(fmt, case):
    """The prompts' kernel on tokens that dominate and on blocks of zero values that take most of the attention."""
    import torch
    n, n_q = 1500, 200
    c = _new(1, 1, 2, [n], 64, fmt)
    g = torch.Generator().manual_seed(67)
    k, v = 0.1 * torch.randn(1, 1, n, 128, generator=g), 1e-2 * torch.randn(1, 1, n, 128, generator=g)
    if case == "dominant":
        at = torch.arange(5, n, 200)
        k[0, 0, at, 0] = torch.linspace(10, 30, len(at))
        v[0, 0] *= torch.where(torch.arange(n) % 200 < 32, 2.0 ** -9, 8.0)[:, None]
    else:
        k[0, 0, 32:64, 0] += 8.0
        v[0, 0, 32:64] = 0.0
        v[0, 0, 320:352] = -0.0
    _append(c, 0, k.half(), v.half(), [0], [n])
    q = torch.zeros(1, 2, n_q, 128)
    q[:, 0, :, 0] = math.log(2.0) / SM  # scores of head 0 are the first channel, in log2 units; head 1 sees all alike
    q = q.half()
    out = _attend(c, [n], q, [n_q])
    _check_attention(c, out, [n], q, [n_q], fmt, "fp16", f"uneven {fmt} {case}", rows=np.array([0, 50, n_q - 1]))


def test_empty_rows():
    import torch

    import paper_2609_11582_amd as okvq
    c = _filled(2, 1, 4, [40, 3], 64, "int8", "fp16", 71)
    before, zero = {f: t.clone() for f, t in c.buffers.items()}, _i32([0, 0])
    none = torch.empty(2, 1, 0, 128, dtype=torch.float16, device="cuda")
    okvq.okvq_q8_append(c, 0, [40, 3], none, none, [0, 0], zero, 0)
    q = torch.empty(2, 4, 0, 128, dtype=torch.float16, device="cuda")
    okvq.okvq_q8_attention(c, 0, [40, 3], q, [0, 0], zero, 0, SM, q.clone(), okvq.q8_workspace(c.dims, 40))
    rot = okvq.make_rotary([1.0] * 64, [0] * 64)
    okvq.okvq_rotary(rot, q, none, torch.empty(2, 3, 0, dtype=torch.int32, device="cuda"), q, none)
    torch.cuda.synchronize()
    for f, t in c.buffers.items():
        assert torch.equal(t.view(torch.uint8), before[f].view(torch.uint8)), f


@pytest.mark.parametrize("n, n_q", [(400, 1), (6000, 1), (400, 150), (6000, 150), (6000, 20)])
@pytest.mark.parametrize("fmt, e", [("int8", -115), ("int8", -118), ("e4m3", -112), ("e4m3", -115)])
def test_small_values(fmt, e, n, n_q):
    """bfloat16 values around 2^e: their scales are above 2^-126 and their means normal numbers, but the factor of the summed
    products, 2^-7 of a scale over the weights' sum, is not. Splits, the merge and both kernels."""
    import torch
    c = _new(1, 1, 2, [n], 64, fmt, "bf16")
    k = 0.05 * _rows(151, 1, 1, n, 128).double()
    v = 2.0 ** e * (1 + 0.3 * _rows(152, 1, 1, n, 128).double().clamp(-3, 3))
    _append(c, 0, k.to(torch.bfloat16), v.to(torch.bfloat16), [0], [n])
    q = _rows(153, 1, 2, n_q, 128, dtype="bf16")
    out = _attend(c, [n], q, [n_q], cross=True)
    a = _numpy(c)
    assert np.nanmin(a["v_scale"]) > 2.0 ** -126
    kk, vv = oq.read_sequence(a, 0, 0, 0, n, fmt)
    for j in range(2):
        pick = np.unique([0, n_q // 2, n_q - 1])
        ref, bound = oq.attention(q[0, j, pick].double().numpy(), kk, vv * 2.0 ** -e, np.full(len(pick), n), SM, HALF["bf16"])
        r = np.abs(out[0, j, pick].double().cpu().numpy() * 2.0 ** -e - ref) / bound
        _say(f"small values {fmt} 2^{e} {n} tokens rows {n_q} head {j}: worst err / bound {r.max():.3f}")
        assert r.max() <= 1


@pytest.mark.parametrize("n_q", [1, 4, 90])
@pytest.mark.parametrize("parked", [0, 700])
def test_idle_slots_take_no_part(n_q, parked):
    """One sequence with new rows in a cache of 64 slots, the others empty or parked: it is attended as in a cache of its own
    (bit for bit: the same splits), and the other slots' rows are left as they were."""
    import torch

    import paper_2609_11582_amd as okvq
    B, H, Hq, n, at = 64, 4, 16, 20000, 37
    lens = [parked] * B
    lens[at] = n
    c = _new(B, H, Hq, lens, 256, "int8", "fp16", seed=161)
    k, v = _rows(162, 1, H, n, 128), _rows(163, 1, H, n, 128)
    alone = dict(c.buffers, block_table=c["block_table"][at:at + 1].clone(), seq_lens=_i32([n]),
                 k_stage=torch.zeros(1, 1, H, 32, 128, dtype=torch.float16, device="cuda"),
                 v_stage=torch.zeros(1, 1, H, 32, 128, dtype=torch.float16, device="cuda"))
    c1 = okvq.Q8Cache(1, H, Hq, c.dims.num_pages, c.dims.max_pages, page_tokens=256, buffers=alone)
    _append(c1, 0, k, v, [0], [n])
    c["seq_lens"].copy_(_i32(lens))
    q = torch.full((B, Hq, n_q, 128), float("nan"), dtype=torch.float16)
    q[at] = _rows(164, Hq, n_q, 128)
    new = [n_q if b == at else 0 for b in range(B)]
    want = _attend(c1, [n], q[at:at + 1], [n_q])
    out = _attend(c, lens, q, new)
    assert torch.equal(out[at], want[0])
    assert bool((out[torch.arange(B) != at] == 9).all())
    a = _numpy(c1)
    ref, bound = oq.attention(q[at, 0, -1:].double().numpy(), *oq.read_sequence(a, 0, 0, 0, n, "int8"), np.array([n]), SM, HALF["fp16"])
    assert np.all(np.abs(want[0, 0, -1:].double().cpu().numpy() - ref) <= bound)


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("H, Hq, lens, new", [
    (1, 7, [5000, 3000, 2000, 40, 0, 6000], [300, 1, 1, 0, 0, 1]),       # a chunk beside single tokens
    (2, 8, [9000, 50, 60, 0, 70, 30, 20, 8000], [2, 1, 3, 0, 1, 0, 1, 1]),
    (4, 16, [20, 4000, 700], [20, 3, 700]),
])
def test_uneven_counts(fmt, dtype, H, Hq, lens, new):
    B, n = len(lens), max(new)
    c = _filled(B, H, Hq, lens, 64, fmt, dtype, 171)
    q = _rows(172, B, Hq, n, 128, dtype=dtype)
    out = _attend(c, lens, q, new)
    _check_attention(c, out, lens, q, new, fmt, dtype, f"uneven counts {fmt} {lens} {new}", rows=np.array([0, 1, 19, 150, 299, 699]))


def test_rows_that_the_host_did_not_count():
    """A captured call's host counts are those of the capture: slots that have rows on the device alone, or more of them than
    the host said (up to the call's largest count), are attended too."""
    import torch

    import paper_2609_11582_amd as okvq
    lens, n = [6000, 900, 40, 5000], 40
    for Hq in (2, 8):  # split kernel and prompt kernel
        c = _filled(4, 2, Hq, lens, 64, "int8", "fp16", 181)
        q = _rows(182, 4, Hq, n, 128)
        for planned, real in (([1, 0, 0, 40], [1, 1, 40, 3]), ([40, 0, 0, 0], [0, 40, 30, 40]), ([5, 40, 1, 0], [40, 0, 40, 40])):
            out = torch.full(q.shape, 9.0, dtype=torch.float16, device="cuda")
            okvq.okvq_q8_attention(c, 0, lens, q.cuda(), planned, _i32(real), n, SM, out, okvq.q8_workspace(c.dims, 6000, n))
            _check_attention(c, out, lens, q, real, "int8", "fp16", f"planned {planned}, real {real}", rows=np.array([0, 20, 39]))


@pytest.mark.parametrize("n_q", [1, 20])
def test_a_long_sequence_among_many_short_ones(n_q):
    """More short sequences than the GPU holds at once, and a long one that is split all the same."""
    import torch
    B, H, Hq, at = 200, 3, 12, 70
    lens = [20 + 7 * (b % 5) for b in range(B)]
    lens[at] = 30000
    c = _new(B, H, Hq, lens, 64, "int8", "fp16", seed=191)
    g = torch.Generator(device="cuda").manual_seed(192)
    for f in ("k_codes", "v_codes"):
        c[f].random_(0, 256, generator=g)
    c["k_scale"].uniform_(0.005, 0.01, generator=g)
    c["v_scale"].uniform_(0.01, 0.04, generator=g)
    c["seq_lens"].copy_(_i32(lens))
    q = _rows(193, B, Hq, n_q, 128)
    out = _attend(c, lens, q, [n_q] * B).double().cpu().numpy()
    a = _numpy(c)
    for b in (0, 1, at - 1, at, at + 1, B - 1):
        for h in range(H):
            k, v = oq.read_sequence(a, 0, b, h, lens[b], "int8")
            for j in range(h * Hq // H, (h + 1) * Hq // H):
                ref, bound = oq.attention(q[b, j].double().numpy(), k, v, lens[b] - n_q + np.arange(n_q) + 1, SM, HALF["fp16"])
                assert np.all(np.abs(out[b, j] - ref) <= bound), (b, j)
    assert np.isfinite(out).all()


@pytest.mark.parametrize("n", [700, 2500])
@pytest.mark.parametrize("kind, fmt, dtype", [
    ("causal", "int8", "fp16"), ("causal", "e4m3", "bf16"), ("cross", "int8", "bf16"), ("few tokens", "e4m3", "fp16"), ("negative", "int8", "fp16"),
    ("flat", "e4m3", "bf16"), ("dominant", "int8", "fp16"), ("dominant", "e4m3", "fp16"), ("zero blocks", "int8", "fp16"),
    ("zero blocks", "e4m3", "fp16"), ("far scales", "int8", "bf16"), ("far scales", "e4m3", "bf16"), ("small values", "int8", "bf16"),
    ("small values", "e4m3", "bf16")])
def test_many_rows_of_many_heads(kind, fmt, dtype, n):
    """Calls of more tiles than the split kernel takes (300 rows x 16 heads of 2 KV heads), with 128 and with 256 columns."""
    import torch
    H, Hq, n_q, cross, sm, unit = 2, 32, 300, kind in ("cross", "small values"), SM, 0
    g = torch.Generator().manual_seed(211)
    k, v = 0.1 * torch.randn(1, H, n, 128, generator=g).double(), torch.randn(1, H, n, 128, generator=g).double()
    q = torch.randn(1, Hq, n_q, 128, generator=g).double()
    lens, block = [n], torch.arange(n) // 32
    if kind == "few tokens":     # more rows than tokens: the first ones see nothing
        lens, k, v = [130], k[:, :, :130], v[:, :, :130]
    elif kind == "negative":
        sm = -1.5
    elif kind == "flat":
        sm = 0.0
    elif kind in ("dominant", "zero blocks"):
        q[:, ::2] = 0.0
        q[:, ::2, :, 0] = math.log(2.0) / SM  # scores of every other head are the first channel, in log2 units
        v *= 1e-2
        if kind == "dominant":
            at = torch.arange(5, n, 150)
            k[0, :, at, 0] = torch.linspace(10, 30, len(at)).double()
            v *= torch.where(torch.arange(n) % 150 < 32, 2.0 ** -9, 8.0)[:, None]
        else:
            k[:, :, 32:64, 0] += 8.0
            v[:, :, 32:64] = 0.0
            v[:, :, 320:352] = -0.0
    elif kind == "far scales":
        unit = 75
        v *= torch.where(block % 3 == 1, 2.0 ** 75, 2.0 ** -75)[:, None]
    elif kind == "small values":
        unit = -115
        v = 2.0 ** -115 * (1 + 0.3 * v.clamp(-3, 3))
    c = _new(1, H, Hq, lens, 64, fmt, dtype, seed=212)
    k, v, q = (x.to(c.row_dtype) for x in (k, v, q))
    _append(c, 0, k, v, [0], lens)
    out = _attend(c, lens, q, [n_q], cross, sm)
    a, got = _numpy(c), out.double().cpu().numpy() * 2.0 ** -unit
    assert np.isfinite(got).all()
    pick = np.array([0, 1, 150, 169, 170, 171, 299])
    seen = np.full(len(pick), lens[0]) if cross else lens[0] - n_q + pick + 1
    worst = 0.0
    for j in range(Hq):
        kk, vv = oq.read_sequence(a, 0, 0, j // 16, lens[0], fmt)
        ref, bound = oq.attention(q[0, j, pick].double().numpy(), kk, vv * 2.0 ** -unit, seen, sm, HALF[dtype])
        assert np.all(got[0, j, pick][seen <= 0] == 0)
        worst = max(worst, float((np.abs(got[0, j, pick] - ref) / np.maximum(bound, 1e-30)).max()))
    _say(f"many rows of many heads, {kind} {fmt} {dtype} {n}: worst err / bound {worst:.3f}")
    assert worst <= 1


@pytest.mark.parametrize("fmt, dtype", [("int8", "fp16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("lens, new", [
    ([300, 500, 40, 0, 500, 2, 300, 7], [250, 1, 1, 0, 17, 2, 1, 0]),       # one split each, the first alone has many tiles
    ([3000, 2500, 700, 60, 3100, 0, 2900, 4], [40, 1, 3, 1, 2, 0, 0, 4]),  # splits of some
])
def test_many_tiles_beside_few(fmt, dtype, lens, new):
    """The split kernel with a slot of many tiles beside slots of one."""
    B, n = len(lens), max(new)
    c = _filled(B, 1, 7, lens, 64, fmt, dtype, 221)
    q = _rows(222, B, 7, n, 128, dtype=dtype)
    for b in range(B):
        q[b, :, new[b]:] = float("nan")
    out = _attend(c, lens, q, new)
    _check_attention(c, out, lens, q, new, fmt, dtype, f"many tiles beside few {fmt} {new}", rows=np.array([0, 1, 2, 16, 39, 120, 249]))
