"""The weights' gradient of head norms over batches that take several launches (of 256 sequences each): every launch has the whole
GPU and adds to the same work-groups' sums. Tolerances as in test_gpu_v_norm_rotary: 2^-19 of the absolute sum for its terms, 2^-24 for
each addition in fp32 (a lane's rows, 64 at most here, 8 steps of lanes and waves, the last rounding), and one for each launch."""

import numpy as np
import pytest

from oracle import norm_rotary as nr
from test_gpu_v_norm_rotary import AXES, EPS, FREQ, HALF, _backward, _inputs, _np, _weights_within, _within

pytestmark = pytest.mark.gpu


def test_rows_of_one_launch_among_many_are_shared_by_the_gpu():
    """65535 sequences, 256 launches, of which the first alone has rows: 131072 of them, all the same, so that a sum of many in
    one register would round the same way time and again (over 3 work-groups a lane's 1365 were off by several times the bound)."""
    import torch

    import paper_2609_11582_amd as okvq
    B, H, n = 65535, 64, 8
    x, up, w, _ = _inputs(1, 1, 1, "bf16", 21)
    par, pos = okvq.make_rotary(FREQ, AXES), torch.full((B, 3, n), 77, dtype=torch.int32, device="cuda")
    lens = [n] * 256 + [0] * (B - 256)
    dx = torch.empty(B, H, n, 128, dtype=torch.bfloat16, device="cuda")
    rows = [t.cuda().expand(B, H, n, 128) for t in (x, up)]
    dw = _backward(par, (rows[0], w.cuda(), rows[1]), None, pos, (dx, None), lens=lens)[0]
    rdx, size, rdw, dwsize = nr.norm_rotate_grad(_np(x), _np(w), EPS, pos[:1, :, :1].cpu().numpy(), _np(up), FREQ, AXES)
    _weights_within(_np(dw), rdw * 256 * H * n, dwsize * 256 * H * n, "weights of one launch among 256")
    assert bool((dx[:256] == dx[0, 0, 0]).all())
    _within(_np(dx[0, 0, 0]), rdx[0, 0, 0], size[0, 0, 0], 2.0 ** -18, HALF["bf16"], "rows of one launch among 256")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("kinds", ["qk", "q", "k"])
def test_launches_of_different_sizes(dtype, kinds):
    """Four launches: 3 rows in all, none, more work-groups than before, fewer again. The same bits each time, captured too."""
    import torch

    import paper_2609_11582_amd as okvq
    B, n = 900, 40
    lens = [1 if b < 3 else 0 if b < 512 else 1 + b * 7 % n if b < 768 else b % 3 for b in range(B)]
    par = okvq.make_rotary(FREQ, AXES)
    live = (np.arange(n) < np.array(lens)[:, None])[:, None, :, None]
    sets, pos = [], None
    for i, (kind, H) in enumerate((("q", 3), ("k", 1))):
        x, up, w, p = _inputs(B, H, n, dtype, 22 + i)
        pos = p if pos is None else pos
        sets.append((x, up, w) if kind in kinds else None)
    args = [None if s is None else (s[0].cuda().transpose(1, 2), s[2].cuda(), s[1].cuda()) for s in sets]
    pos_dev, ws = pos.cuda(), okvq.norm_rotary_workspace(B, n)
    ws.fill_(float("nan"))  # no initial contents are needed
    dx = [None if s is None else torch.zeros(s[1].shape, dtype=s[1].dtype, device="cuda") for s in sets]
    dw = _backward(par, *args, pos_dev, dx, lens=lens, ws=ws)
    again = _backward(par, *args, pos_dev, dx, lens=lens, ws=ws)
    for s, d, a, y in zip(sets, dw, again, dx):
        if s is None:
            assert d is None
            continue
        assert torch.equal(d, a)
        x, up, w = s
        rdx, size, rdw, dwsize = nr.norm_rotate_grad(_np(x.transpose(1, 2)), _np(w), EPS, pos.numpy(), np.where(live, _np(up), 0), FREQ, AXES)
        _weights_within(_np(d), rdw, dwsize, f"weights of four launches {dtype}")
        _within(_np(y), np.where(live, rdx, 0), size, 2.0 ** -18, HALF[dtype], f"rows of four launches {dtype}")
    held = [None if a is None else torch.empty(128, device="cuda") for a in args]
    pick = [[None if a is None else a[i] for a in args] for i in range(3)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        okvq.okvq_norm_rotary_backward(par, *pick[0], *pick[1], EPS, pos_dev, *pick[2], *dx, *held, ws, lens=lens)
    for _ in range(3):
        for h in held:
            if h is not None:
                h.fill_(float("nan"))
        ws.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(h is None or torch.equal(h, d) for h, d in zip(held, dw))
