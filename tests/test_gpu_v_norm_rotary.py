"""Head norms with rotary positions and their gradient against the float64 formulas (oracle.norm_rotary).

Tolerance of a row's element: its rounding, half a step of its type (fp16 2^-11, bf16 2^-8; 2^-25 absolute for fp16's
subnormals), and 2^-19 of size = |a| + |b| of the normed, weighted pair: the inverse root mean square is off by half of the
sum's 20 roundings and an ulp of its own (12 2^-24), angle, sine and cosine by 2^-21 (test_gpu_t_rotary), the products
by 4 2^-24. Of a gradient's element 2^-18 of its size: the same, and the mean's 20 roundings of products that carry all of the
former. Of the weights' gradient 2^-19 of the absolute sum for its terms and 2^-24 for each addition in fp32: a lane's rows
(64 at most in these cases), 2 + 3 + 3 steps of lanes and waves, the last rounding."""

import numpy as np
import pytest

from oracle import norm_rotary as nr

pytestmark = pytest.mark.gpu
FREQ = [1e6 ** (-i / 64) for i in range(64)]
AXES = [0] * 16 + [1] * 24 + [2] * 24
HALF = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
EPS = 1e-6


def _t(dtype):
    import torch
    return torch.float16 if dtype == "fp16" else torch.bfloat16


def _inputs(B, heads, n, dtype, seed):
    """Rows [B][n][heads][128] as a projection leaves them, gradients [B][heads][n][128], weights, positions."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(B, n, heads, 128, generator=g) * torch.exp(torch.randn(B, n, heads, 1, generator=g))).to(_t(dtype))
    up = (torch.randn(B, heads, n, 128, generator=g) * 0.1).to(_t(dtype))
    w = torch.rand(128, generator=g) * 2 - 0.3
    pos = torch.randint(0, 140000, (B, 3, n), generator=g).to(torch.int32)
    return x, up, w, pos


def _np(x):
    return x.double().cpu().numpy()


def _within(got, ref, size, rel, half, tag):
    err = np.abs(got - ref) / (half * np.abs(ref) + rel * size + 2.0 ** -25)
    worst = float(err.max()) if err.size else 0.0
    print(f"[gpu-case] {tag}: worst err / tolerance {worst:.3f}", flush=True)
    assert worst <= 1


def _weights_within(got, ref, size, tag):
    err = np.abs(got - ref) / ((2.0 ** -19 + 73 * 2.0 ** -24) * size + 1e-30)
    print(f"[gpu-case] {tag}: worst err / tolerance {err.max():.3f}", flush=True)
    assert err.max() <= 1


def _backward(par, q, k, pos, dqk, lens=None, flags=0, ws=None, stream=None):
    """q, k: (x as a view [B][heads][n][128], weight, gradient) on the device or None; dqk: the row gradients' tensors."""
    import torch

    import paper_2609_11582_amd as okvq
    some = q or k
    ws = okvq.norm_rotary_workspace(some[0].shape[0], some[0].shape[2]) if ws is None else ws
    dw = [None if a is None else torch.full((128,), float("nan"), device="cuda") for a in (q, k)]
    pick = [[None if a is None else a[i] for a in (q, k)] for i in range(3)]
    okvq.okvq_norm_rotary_backward(par, *pick[0], *pick[1], EPS, pos, *pick[2], *dqk, *dw, ws, lens=lens, flags=flags, stream=stream)
    return dw


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("B, hq, hk, n", [(1, 28, 4, 1), (3, 7, 1, 37), (1, 1, 1, 8), (2, 16, 2, 9), (1, 33, 5, 2), (2, 6, 3, 700),
                                         (1, 12, 2, 301), (1, 3, 2, 4101), (1, 17, 2, 2571)])
def test_forward_and_gradient(dtype, adjacent, B, hq, hk, n):
    import torch

    import paper_2609_11582_amd as okvq
    q, gq, wq, pos = _inputs(B, hq, n, dtype, 1)
    k, gk, wk, _ = _inputs(B, hk, n, dtype, 2)
    flags = okvq.OKVQ_ROTARY_ADJACENT if adjacent else 0
    par, posd = okvq.make_rotary(FREQ, AXES), pos.cuda()
    qd, kd = q.cuda().transpose(1, 2), k.cuda().transpose(1, 2)
    qo, ko = torch.empty(B, hq, n, 128, dtype=q.dtype, device="cuda"), torch.empty(B, hk, n, 128, dtype=q.dtype, device="cuda")
    okvq.okvq_norm_rotary(par, qd, kd, wq.cuda(), wk.cuda(), EPS, posd, qo, ko, flags=flags)
    dq, dk = torch.empty_like(q, device="cuda"), torch.empty_like(k, device="cuda")  # token by token
    dws = _backward(par, (qd, wq.cuda(), gq.cuda()), (kd, wk.cuda(), gk.cuda()), posd, (dq.transpose(1, 2), dk.transpose(1, 2)), flags=flags)
    for x, up, w, y, dx, dw, h in ((q, gq, wq, qo, dq, dws[0], hq), (k, gk, wk, ko, dk, dws[1], hk)):
        tag = f"{B}x{h}x{n} {dtype}"
        a, wn, p = _np(x.transpose(1, 2)), _np(w), pos.numpy()
        ref, size = nr.norm_rotate(a, wn, EPS, p, FREQ, AXES, adjacent)
        _within(_np(y), ref, size, 2.0 ** -19, HALF[dtype], "norm " + tag)
        rdx, dxs, rdw, dws_ = nr.norm_rotate_grad(a, wn, EPS, p, _np(up), FREQ, AXES, adjacent)
        _within(_np(dx.transpose(1, 2)), rdx, dxs, 2.0 ** -18, HALF[dtype], "gradient " + tag)
        _weights_within(_np(dw), rdw, dws_, "weights " + tag)


def test_rows_of_other_sizes():
    """Zero rows, rows far below eps, rows at the end of fp16, and bfloat16 rows of 1e15 and 1e-15."""
    import torch

    import paper_2609_11582_amd as okvq
    par = okvq.make_rotary(FREQ, AXES)
    for dtype, sizes in (("fp16", [0.0, 1e-6, 1e-3, 60000.0]), ("bf16", [0.0, 1e-15, 1e-4, 1e15])):
        x, up, w, pos = _inputs(1, len(sizes), 9, dtype, 3)
        x = (x.float().clamp(-1, 1) * torch.tensor(sizes)[:, None]).to(x.dtype)
        d = x.cuda().transpose(1, 2)
        y, dx = (torch.empty(1, len(sizes), 9, 128, dtype=x.dtype, device="cuda") for _ in range(2))
        okvq.okvq_norm_rotary(par, None, d, None, w.cuda(), EPS, pos.cuda(), None, y)
        dw = _backward(par, None, (d, w.cuda(), up.cuda()), pos.cuda(), (None, dx))[1]
        a = _np(x.transpose(1, 2))
        ref, size = nr.norm_rotate(a, _np(w), EPS, pos.numpy(), FREQ, AXES)
        _within(_np(y), ref, size, 2.0 ** -19, HALF[dtype], f"sizes {dtype}")
        assert bool((y[:, 0] == 0).all())
        rdx, dxs, rdw, dwsize = nr.norm_rotate_grad(a, _np(w), EPS, pos.numpy(), _np(up), FREQ, AXES)
        got = _np(dx)
        if dtype == "fp16":
            over = np.abs(rdx) * (1 + 2.0 ** -11) >= 65520  # gradients of rows below eps pass the type's largest number
            assert np.all(np.isinf(got[over])) or not over.any()
            got, rdx, dxs = got[~over], rdx[~over], dxs[~over]
        _within(got, rdx, dxs, 2.0 ** -18, HALF[dtype], f"gradient of sizes {dtype}")
        _weights_within(_np(dw), rdw, dwsize, f"weights of sizes {dtype}")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("lens", [[19, 0, 1, 8, 17], [700, 0, 701, 1]])
def test_ragged_rows_layouts_and_in_place(dtype, lens):
    import torch

    import paper_2609_11582_amd as okvq
    B, H, n = len(lens), 3, max(lens)
    x, up, w, pos = _inputs(B, H, n, dtype, 4)
    for b, m in enumerate(lens):
        x[b, m:] = float("nan")
        up[b, :, m:] = float("nan")
    par, wd, pd = okvq.make_rotary(FREQ, AXES), w.cuda(), pos.cuda()
    # a slice of one fused projection's heads
    wide = torch.full((B, n, H + 2, 128), 7.0, dtype=x.dtype, device="cuda")
    wide[:, :, 1:1 + H] = x.cuda()
    src = wide[:, :, 1:1 + H].transpose(1, 2)
    out = torch.full((B, n, H, 128), 5.0, dtype=x.dtype, device="cuda")
    okvq.okvq_norm_rotary(par, src, None, wd, None, EPS, pd, out.transpose(1, 2), None, lens=lens)
    dx = torch.full((B, n, H, 128), 5.0, dtype=x.dtype, device="cuda")
    dw = _backward(par, (src, wd, up.cuda()), None, pd, (dx.transpose(1, 2), None), lens=lens)[0]
    inside = wide.clone()
    view = inside[:, :, 1:1 + H].transpose(1, 2)
    okvq.okvq_norm_rotary(par, view, None, wd, None, EPS, pd, view, None, lens=lens)         # in place, strided
    over = up.cuda()
    dw2 = _backward(par, (src, wd, over), None, pd, (over, None), lens=lens)[0]              # over the gradient that came in
    mine = src.contiguous()
    dw3 = _backward(par, (mine, wd, up.cuda()), None, pd, (mine, None), lens=lens)[0]        # over the rows
    assert torch.equal(dw, dw2) and torch.equal(dw, dw3)
    assert bool((inside[:, :, 0] == 7).all()) and bool((inside[:, :, 1 + H:] == 7).all())
    total, size_total = 0, 0
    for b, m in enumerate(lens):
        assert bool((out[b, m:] == 5).all()) and bool((dx[b, m:] == 5).all()) and bool(over[b, :, m:].isnan().all())
        if not m:
            continue
        got, gdx = out[b, :m].transpose(0, 1), dx[b, :m].transpose(0, 1)
        assert torch.equal(got, view[b, :, :m]) and torch.equal(gdx, over[b, :, :m]) and torch.equal(gdx, mine[b, :, :m])
        a, p = _np(x[b:b + 1, :m].transpose(1, 2)), pos.numpy()[b:b + 1, :, :m]
        ref, size = nr.norm_rotate(a, _np(w), EPS, p, FREQ, AXES)
        _within(_np(got)[None], ref, size, 2.0 ** -19, HALF[dtype], f"sequence {b}")
        rdx, dxs, rdw, dwsize = nr.norm_rotate_grad(a, _np(w), EPS, p, _np(up[b:b + 1, :, :m]), FREQ, AXES)
        _within(_np(gdx)[None], rdx, dxs, 2.0 ** -18, HALF[dtype], f"gradient of sequence {b}")
        total, size_total = total + rdw, size_total + dwsize
    _weights_within(_np(dw), total, size_total, "weights")


def test_many_sequences():
    import torch

    import paper_2609_11582_amd as okvq
    B = 515  # three launches of up to 256
    x, up, w, pos = _inputs(B, 2, 3, "fp16", 6)
    lens = [b % 4 for b in range(B)]
    par = okvq.make_rotary(FREQ, AXES)
    live = (np.arange(3) < np.array(lens)[:, None])[:, None, :, None]
    d, dx = x.cuda().transpose(1, 2), torch.zeros(B, 2, 3, 128, dtype=torch.float16, device="cuda")
    y = torch.zeros_like(dx)
    okvq.okvq_norm_rotary(par, None, d, None, w.cuda(), EPS, pos.cuda(), None, y, lens=lens)
    dw = _backward(par, None, (d, w.cuda(), up.cuda()), pos.cuda(), (None, dx), lens=lens)[1]
    a = _np(x.transpose(1, 2))
    ref, size = nr.norm_rotate(a, _np(w), EPS, pos.numpy(), FREQ, AXES)
    assert np.all(np.where(live, 0, _np(y)) == 0) and np.all(np.where(live, 0, _np(dx)) == 0)
    _within(_np(y), np.where(live, ref, 0), size, 2.0 ** -19, HALF["fp16"], "515 sequences")
    rdx, dxs, rdw, dwsize = nr.norm_rotate_grad(a, _np(w), EPS, pos.numpy(), np.where(live, _np(up), 0), FREQ, AXES)
    _within(_np(dx), np.where(live, rdx, 0), dxs, 2.0 ** -18, HALF["fp16"], "gradient of 515 sequences")
    _weights_within(_np(dw), rdw, dwsize, "weights of 515 sequences")
    # no rows at all: the weights' gradient is zero and nothing else changes
    dw = _backward(par, None, (d, w.cuda(), up.cuda()), pos.cuda(), (None, y), lens=[0] * B)[1]
    assert bool((dw == 0).all())
    _within(_np(y), np.where(live, ref, 0), size, 2.0 ** -19, HALF["fp16"], "left as they were")


def test_gradient_against_differences_of_the_loss():
    """loss = sum up * y(x, w). Along a line a row's unit vector f has |f'''| <= 12 kappa^3 with kappa the step over the row's
    length (1 / length has derivatives n! kappa^n at most), so that a central difference of step 1 is off by 2 kappa^3
    times the lengths of the row's y and up at most; y is linear in w. Both sides round y to half a step (random signs,
    6 sigma)."""
    import torch

    import paper_2609_11582_amd as okvq
    B, H, n = 1, 2, 40
    par = okvq.make_rotary(FREQ, AXES)
    x, up, w, pos = _inputs(B, H, n, "fp16", 8)
    x = x.transpose(1, 2).contiguous()
    g = torch.Generator().manual_seed(9)

    def norm(v, wt):
        out = torch.empty(B, H, n, 128, dtype=torch.float16, device="cuda")
        okvq.okvq_norm_rotary(par, v.cuda(), None, wt.cuda(), None, EPS, pos.cuda(), out, None)
        return out.double().cpu()
    dx = torch.empty(B, H, n, 128, dtype=torch.float16, device="cuda")
    dw = _backward(par, (x.cuda(), w.cuda(), up.cuda()), None, pos.cuda(), (dx, None))[0].double().cpu()
    dx = dx.double().cpu()
    length = x.double().norm(dim=-1, keepdim=True)
    way = dx.sign() * length / 128 ** 0.5 / 16 * (0.5 + torch.rand(x.shape, generator=g))
    above, below = (x.double() + way).half(), (x.double() - way).half()
    way = (above.double() - below.double()) / 2
    middle = (above.double() + below.double()) / 2 - x.double()  # what rounding moved the middle by, along the gradient
    u, y = up.double(), norm(x, w)
    change = float((u * (norm(above, w) - norm(below, w))).sum()) / 2
    kappa = way.norm(dim=-1) / (length[..., 0] - way.norm(dim=-1))
    yu = y.norm(dim=-1) * (u * w.abs().max()).norm(dim=-1)
    noise = 6 * 2.0 ** -11 * float((u * y).pow(2).sum().sqrt())
    bound = float((2 * kappa ** 3 * yu).sum()) + noise + float((kappa * middle.norm(dim=-1) / length[..., 0] * 6 * yu).sum()) \
        + 2.0 ** -11 * float((way * dx).abs().sum())
    slope = float((way * dx).sum())
    print(f"[gpu-case] change {change:.4f}, slope {slope:.4f}, bound {bound:.4f}", flush=True)
    assert abs(change - slope) <= bound and bound < 0.1 * abs(slope)
    # in the weights: linear
    step = (torch.rand(128, generator=g) - 0.5) * 0.25 + 0.2 * dw.sign().float()
    moved = w + step
    change = float((u * (norm(x, moved) - y)).sum())
    slope = float(((moved - w).double() * dw).sum())
    print(f"[gpu-case] change {change:.4f}, slope {slope:.4f}, bound {2 * noise:.4f}", flush=True)
    assert abs(change - slope) <= 2 * noise + 2.0 ** -17 * float((u.abs() * y.abs()).sum())


def test_captured_and_replayed():
    """Two graphs with workspaces of their own, forward and backward, replayed with eager calls between; another stream."""
    import torch

    import paper_2609_11582_amd as okvq
    par = okvq.make_rotary(FREQ, AXES)
    B, H, n = 2, 5, 333
    sets = []
    for seed in (11, 12):
        x, up, w, pos = _inputs(B, H, n, "bf16", seed)
        s = dict(x=x.cuda().transpose(1, 2), up=up.cuda(), w=w.cuda(), pos=pos.cuda(), ws=okvq.norm_rotary_workspace(B, n),
                 y=torch.empty_like(up, device="cuda"), dx=torch.empty_like(up, device="cuda"), dw=torch.empty(128, device="cuda"))
        sets.append(s)

    def step(s):
        okvq.okvq_norm_rotary(par, s["x"], None, s["w"], None, EPS, s["pos"], s["y"], None)
        okvq.okvq_norm_rotary_backward(par, s["x"], None, s["w"], None, EPS, s["pos"], s["up"], None, s["dx"], None, s["dw"], None, s["ws"])
    want = []
    for s in sets:
        step(s)
        torch.cuda.synchronize()
        want.append([s[f].clone() for f in ("y", "dx", "dw")])
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(s)
        graphs.append(g)
    for _ in range(3):
        for s in sets:
            for f in ("y", "dx", "dw"):
                s[f].fill_(float("nan"))
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for s, w in zip(sets, want):
            assert all(torch.equal(s[f], v) for f, v in zip(("y", "dx", "dw"), w))
    with torch.cuda.stream(streams[0]):  # the current stream, and a given one
        for s in sets:
            s["y"].zero_()
        step(sets[0])
    streams[0].synchronize()
    assert torch.equal(sets[0]["y"], want[0][0]) and torch.equal(sets[0]["dw"], want[0][2])


def test_far_rows():
    """Rows past 2^32 bytes from their start."""
    import torch

    import paper_2609_11582_amd as okvq
    par = okvq.make_rotary(FREQ, AXES)
    x, up, w, pos = _inputs(1, 2, 5, "fp16", 13)
    pool = torch.empty((5 << 30) // 2, dtype=torch.float16, device="cuda")
    far = torch.as_strided(pool, (1, 2, 5, 128), (0, (1 << 31) + 1024, 1 << 14, 1))
    far.copy_(x.transpose(1, 2))
    okvq.okvq_norm_rotary(par, far, None, w.cuda(), None, EPS, pos.cuda(), far, None)
    near = torch.empty(1, 2, 5, 128, dtype=torch.float16, device="cuda")
    okvq.okvq_norm_rotary(par, x.cuda().transpose(1, 2), None, w.cuda(), None, EPS, pos.cuda(), near, None)
    assert torch.equal(far, near)


def test_refuses_wrong_tensors():
    import torch

    import paper_2609_11582_amd as okvq
    par = okvq.make_rotary(FREQ, AXES)
    x = torch.zeros(1, 2, 4, 128, dtype=torch.float16, device="cuda")
    pos = torch.zeros(1, 3, 4, dtype=torch.int32, device="cuda")
    w, ws = torch.ones(128, device="cuda"), okvq.norm_rotary_workspace(1, 4)

    def forward(q=x, w=w, pos=pos, out=x, k=None, eps=EPS, flags=0):
        okvq.okvq_norm_rotary(par, q, k, w, None, eps, pos, out, None, flags=flags)

    def backward(q=x, w=w, pos=pos, out=x, up=x, dw=w, ws=ws, eps=EPS, flags=0):
        okvq.okvq_norm_rotary_backward(par, q, None, w, None, eps, pos, up, None, out, None, dw, None, ws, flags=flags)
    for call in (forward, backward):
        for bad in (x.float(), x[..., :64], x[:, :, :3], x.cpu(), torch.zeros(1, 2, 4, 256, dtype=torch.float16, device="cuda")[..., ::2]):
            with pytest.raises(ValueError):
                call(out=bad)
        for bad in (w.half(), w[:64], w.cpu(), None, torch.ones(256, device="cuda")[::2]):
            with pytest.raises(ValueError):
                call(w=bad)
        with pytest.raises(ValueError):
            call(pos=pos.long())
        with pytest.raises(ValueError):
            call(pos=pos[:, :, :3].contiguous())
        with pytest.raises(okvq.OkvqError):
            call(eps=0.0)
        with pytest.raises(okvq.OkvqError):
            call(flags=okvq.OKVQ_ROTARY_INVERSE)
    with pytest.raises(ValueError):
        forward(k=x)
    with pytest.raises(ValueError):
        backward(up=None)
    with pytest.raises(ValueError):
        backward(dw=None)
    with pytest.raises(okvq.OkvqError):
        backward(ws=ws[:100])
