"""Head norms with rotary positions and their gradient, and attention with a sliding window and for drafted trees over
the paged 8-bit cache, as cases whose speed and results can be measured.

``own`` chooses between the plain form (elementary torch operations in 32 bits) and the package's
calls. ``op`` names the operator:

* ``norm``      -- every head's row of queries and keys divided by its root mean square, weighted, and rotated by
  positions on three axes; rows as the projections leave them (token by token), out head by head;
* ``norm_grad`` -- the gradients of the rows and of both weights;
* ``window``    -- attention over the cache in which a row sees the newest ``window`` tokens up to its own and the first
  ``sinks``: one token (``new`` 1), a chunk of a prompt or a whole one;
* ``tree``      -- attention of drafted tokens that are not in the cache yet: a row sees the cache (all of it, or sinks
  and window) and those drafts that its mask names, its ancestors and itself.

Cache layout (one layer, P pages, H KV heads, T tokens a page; a block is 32 tokens of one head):
``k_codes`` [1][P][H][T][128]; ``v_codes`` [1][P][H][T/32][4096], where token 16a + 4g + i and channel
32j + 16b + n of a block are at byte 1024j + 16(16g + n) + 8b + 4a + i; ``k_scale``, ``v_scale``
[1][P][H][T/32] fp32; ``block_table`` [B][max_pages] (-1: none), ``seq_lens`` [B].
"""

from __future__ import annotations

import math
import random

import torch

own = False

D, W, PAIRS = 128, 32, 64
SM_SCALE = 1.0 / math.sqrt(D)
EPS = 1e-6
TOP = {"int8": 127.0, "e4m3": 448.0}
SECTIONS = (16, 24, 24)  # pairs of channels turned by the time, height and width positions
THETA = 1e6


def _case(name, op, batch, kv_heads, q_heads, tokens, **more):
    c = {"name": name, "op": op, "batch": batch, "kv_heads": kv_heads, "q_heads": q_heads, "tokens": tokens, "new": 1,
         "page": 64, "format": "int8", "dtype": "fp16", "ragged": False, "drift": 0.02, "adjacent": False, "window": 0,
         "sinks": 0}
    c.update(more)
    return c


def listed():
    return [
        # the smallest call: the one new token of a decode step of a 7B model
        _case("norm_7b_step", "norm", 1, 4, 28, 1),
        # a decode step of a serving batch of a 30B model
        _case("norm_30b_b32_step", "norm", 32, 4, 32, 1, dtype="bf16"),
        # queries and keys of a whole long prompt
        _case("norm_7b_32k", "norm", 1, 4, 28, 32768, new=32768),
        # the backward pass of a training batch of odd lengths, neighbouring channels paired
        _case("norm_grad_3b_b4", "norm_grad", 4, 2, 16, 2999, new=2999, ragged=True, dtype="bf16", adjacent=True),
        # the backward pass of one long sequence
        _case("norm_grad_7b_8k", "norm_grad", 1, 4, 28, 8192, new=8192),
        # one decode step in a layer with a window, far into a long sequence
        _case("window_7b_32k", "window", 1, 4, 28, 32768, window=4096, sinks=4),
        # the same for a serving batch of sequences of different lengths
        _case("window_7b_b16_ragged", "window", 16, 4, 28, 16384, ragged=True, window=1024, sinks=16, format="e4m3", dtype="bf16",
              page=128),
        # the attention of a whole prompt, eight windows long
        _case("window_7b_prompt_8k", "window", 1, 4, 28, 8192, new=8192, window=1024, sinks=4),
        # chunks of four streams against their long caches
        _case("window_3b_b4_64k_chunk", "window", 4, 2, 16, 65536, new=512, window=4096, sinks=64, format="e4m3", dtype="bf16"),
        # sixteen drafts to be verified at 32k tokens
        _case("tree_7b_32k", "tree", 1, 4, 28, 32768, new=16),
        # a serving batch whose sequences have different numbers of drafts, one none at all
        _case("tree_7b_b8_ragged", "tree", 8, 4, 28, 8192, new=25, ragged=True, format="e4m3", dtype="bf16"),
        # a large tree at the long context of a 30B model
        _case("tree_30b_128k", "tree", 1, 4, 32, 131072, new=64),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "window", "window", "window", "tree", "tree", "tree"])
    kv, q = rng.choice([(1, 4), (1, 7), (2, 6), (2, 16), (4, 28), (4, 28), (4, 32), (8, 8), (8, 32), (1, 16), (3, 36)])
    batch = rng.choice([1, 1, 1, 2, 3, 4, 8, 16])
    more = {"page": rng.choice([32, 64, 64, 128, 256]), "format": rng.choice(["int8", "e4m3"]), "dtype": rng.choice(["fp16", "bf16"]),
            "ragged": batch > 1 and rng.random() < 0.7, "drift": rng.choice([0.0, 0.02, 0.5])}
    if op in ("norm", "norm_grad"):
        tokens = _log_int(rng, 1, (1 << (20 if op == "norm" else 19)) // (batch * (kv + q)))
        more.update(new=tokens, adjacent=rng.random() < 0.4)
    else:
        tokens = _log_int(rng, 40, min(131072, (1 << 19) // (batch * kv)))
        new = 1
        if op == "tree":
            new = _log_int(rng, 2, min(128, max(2, (1 << 27) // (batch * q * tokens))))
            if rng.random() < 0.3:
                more.update(window=_log_int(rng, 64, 8192), sinks=rng.choice([0, 1, 4, 37, 64]))
        else:
            more.update(window=_log_int(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 4, 37, 64]))
            kind = rng.choice(["one", "one", "chunk", "prompt"])
            if kind == "prompt":
                new = tokens = _log_int(rng, 16, min(8192, 229376 // (batch * q)))
            elif kind == "chunk":
                new = _log_int(rng, 2, max(2, min(tokens, 1024, (1 << 27) // (batch * q * (more["window"] + 64)))))
        more.update(new=new)
    c = _case("", op, batch, kv, q, tokens, **more)
    del c["name"]
    return c


# ---- sizes ----------------------------------------------------------------------------------------


def _lengths(case):
    """The sequences' lengths (with the new tokens, but without drafts): the full one, or spread over its upper half."""
    n, B = case["tokens"], case["batch"]
    if not case["ragged"]:
        return [n] * B
    return [n - (b * 7919) % max(n // 2, 1) for b in range(B)]


def _news(case):
    """New tokens or drafts of each sequence: ragged batches have fewer of them here and there, one none at all."""
    most = [case["new"] if case["op"] == "tree" else min(case["new"], L) for L in _lengths(case)]
    if not case["ragged"] or case["new"] == 1:
        return most
    return [0 if b % 8 == 7 else max(1, m - (b * 37) % max(m // 2, 1)) for b, m in enumerate(most)]


def _up(a, b):
    return -(-a // b)


def _seen(L, first, last, sinks):
    """Tokens 0 .. L - 1 that are sinks or in first .. last - 1."""
    return min(sinks, L) + max(min(last, L) - max(first, min(sinks, L)), 0)


def work(case):
    H, Hq, op = case["kv_heads"], case["q_heads"], case["op"]
    lens, news = _lengths(case), _news(case)
    row = 2 * D
    if op == "norm":
        n = sum(news)
        return {"bytes": n * (2 * row * (H + Hq) + 12) + 8 * D, "flops": n * (H + Hq) * (4 * D + 6 * PAIRS)}
    if op == "norm_grad":
        n = sum(news)
        return {"bytes": n * (3 * row * (H + Hq) + 12) + 16 * D, "flops": n * (H + Hq) * (12 * D + 6 * PAIRS)}
    nbytes, flops = 0, 0
    w, sinks = case["window"] or (1 << 40), case["sinks"]
    for L, n in zip(lens, news):
        if not n:
            continue
        if op == "window":
            pairs = sum(_seen(L, L - n + i + 1 - w, L - n + i + 1, sinks) for i in range(n))
            held = _seen(L, L - n + 1 - w, L, sinks)
        else:  # the cache, as a first draft sees it, and the row's own draft at least
            pairs = n * (_seen(L, L + 1 - w, L, sinks) + 1)
            held = _seen(L, L + 1 - w, L, sinks)
            nbytes += 2 * H * n * row + 4 * n * _up(n, 32)
        nbytes += H * (_up(held, W) * (2 * D * W + 8)) + 2 * n * Hq * row
        flops += 4 * D * Hq * pairs
    return {"bytes": nbytes, "flops": flops}


# ---- inputs ---------------------------------------------------------------------------------------


def _dtype(case):
    return torch.float16 if case["dtype"] == "fp16" else torch.bfloat16


def _inv_freq():
    return [THETA ** (-i / PAIRS) for i in range(PAIRS)]


def _axes():
    return [a for a, n in enumerate(SECTIONS) for _ in range(n)]


def _i32(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _stream_positions(n, start=0):
    """[3][n] positions of an audio-visual stream: chunks of 10 x 15 video tokens that share a time, then 25 audio
    tokens a time step apart."""
    at = torch.arange(start, start + n, device="cuda")
    chunk, i = at // 175, at % 175
    video = i < 150
    t = chunk * 50 + torch.where(video, 0, i - 150)
    return torch.stack((t, torch.where(video, chunk * 50 + i // 15, t), torch.where(video, chunk * 50 + i % 15, t))).to(torch.int32)


def _rows(g, B, H, n, drift):
    """Keys or values [B][H][n][128]: noise, a mean that wanders along the sequence, a few large channels."""
    x = torch.randn(B, H, n, D, generator=g, device="cuda")
    if drift:
        step = drift * torch.randn(B, H, _up(n, 64), D, generator=g, device="cuda")
        x += step.cumsum(2).repeat_interleave(64, dim=2)[:, :, :n]
    for h in range(H):
        x[:, h, :, torch.randperm(D, generator=g, device="cuda")[:4]] *= 8.0
    return x


def _pack_values(x):
    """Codes [..][32][128] in the byte order of a value block."""
    lead = x.shape[:-2]
    x = x.reshape(*lead, 2, 4, 4, 4, 2, 16)  # a g i j b n
    d = len(lead)
    return x.permute(*range(d), d + 3, d + 1, d + 5, d + 4, d, d + 2).reshape(*lead, D * W)


def _unpack_values(x):
    lead = x.shape[:-1]
    x = x.reshape(*lead, 4, 4, 16, 2, 2, 4)  # j g n b a i
    d = len(lead)
    return x.permute(*range(d), d + 4, d + 1, d + 5, d, d + 3, d + 2).reshape(*lead, W, D)


def _cache(case, g, lens):
    """A cache whose sequences hold `lens` tokens in pages of any order."""
    B, H, T, dt = case["batch"], case["kv_heads"], case["page"], _dtype(case)
    mp, N = _up(max(lens), T), _up(max(lens), W) * W
    P = sum(_up(L, T) for L in lens) + 5
    z = lambda *s, dtype: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    c = {"k_codes": z(1, P, H, T, D, dtype=torch.uint8), "v_codes": z(1, P, H, T // W, D * W, dtype=torch.uint8),
         "k_scale": z(1, P, H, T // W, dtype=torch.float32), "v_scale": z(1, P, H, T // W, dtype=torch.float32),
         "k_stage": z(1, B, H, W, D, dtype=dt), "v_stage": z(1, B, H, W, D, dtype=dt),
         "block_table": z(B, mp, dtype=torch.int32) - 1, "seq_lens": _i32(lens),
         "page_refs": z(P, dtype=torch.int32), "status": z(4, dtype=torch.int32)}
    order = torch.randperm(P, generator=g, device="cuda").to(torch.int32)
    used = 0
    for b, L in enumerate(lens):
        n = _up(L, T)
        c["block_table"][b, :n] = order[used:used + n]
        c["page_refs"][order[used:used + n].long()] = 1
        used += n
    b, j = (torch.arange(N // W, device="cuda") * W < c["seq_lens"][:, None]).nonzero(as_tuple=True)
    page, sub = c["block_table"][b, j * W // T].long(), j * W % T // W
    held = (torch.arange(N, device="cuda") < c["seq_lens"][:, None])[:, None, :, None]
    for f in ("k", "v"):
        x = torch.where(held, _rows(g, B, H, N, case["drift"]).to(dt).float(), 0.0).view(B, H, N // W, W, D)
        scale = x.abs().amax((-2, -1)) / TOP[case["format"]]
        t = x / torch.where(scale > 0, scale, 1.0)[..., None, None]
        code = torch.round(t).to(torch.int8) if case["format"] == "int8" else t.to(torch.float8_e4m3fn)
        code = code.view(torch.uint8)[b, :, j]
        if f == "k":
            c["k_codes"][0].view(P, H, T // W, W, D)[page, :, sub] = code
        else:
            c["v_codes"][0][page, :, sub] = _pack_values(code)
        c[f + "_scale"][0][page, :, sub] = torch.where(scale > 0, scale, 1.0)[b, :, j]
    return c


def _trees(case, seed, news, n):
    """Masks [B][n][ceil(n / 32)] of drafted trees: bit j of a row's words names draft j, an ancestor or the row itself."""
    r = random.Random(seed * 7919 + 3)
    words = torch.zeros(len(news), n, _up(n, 32), dtype=torch.int64)
    for b, m in enumerate(news):
        masks = []
        for i in range(m):
            parent = i - 1 if r.random() < 0.4 else r.randrange(-1, i) if i else -1
            masks.append((masks[parent] if parent >= 0 else 0) | 1 << i)
            for k in range(words.shape[2]):
                words[b, i, k] = masks[i] >> 32 * k & 0xffffffff
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + 31)
    B, H, Hq, op, dt = case["batch"], case["kv_heads"], case["q_heads"], case["op"], _dtype(case)
    lens, news = _lengths(case), _news(case)
    n = max(max(news), 1)
    s = {"case": case, "lens": lens, "news": news, "news_dev": _i32(news), "n": n}
    if op in ("norm", "norm_grad"):
        for f, h in (("q", Hq), ("k", H)):
            s[f] = (4.0 * torch.rand(h, 1, generator=g, device="cuda") * torch.randn(B, n, h, D, generator=g, device="cuda")).to(dt)
            s[f + "_weight"] = 0.3 + 1.4 * torch.rand(D, generator=g, device="cuda")
            s[f + "_out"] = torch.zeros(B, h, n, D, dtype=dt, device="cuda")
            if op == "norm_grad":
                s[f + "_grad"] = (0.05 * torch.randn(B, h, n, D, generator=g, device="cuda")).to(dt)
                s["d" + f] = torch.zeros(B, n, h, D, dtype=dt, device="cuda")
                s["d" + f + "_weight"] = torch.zeros(D, device="cuda")
        # each sequence's stream goes on from where its earlier tokens ended
        s["pos"] = torch.stack([_stream_positions(n, int(seed) % 1000 + 30000 * (b % 3)) for b in range(B)]).contiguous()
        if own:
            import paper_2609_11582_amd as okvq
            s["rotary"] = okvq.make_rotary(_inv_freq(), _axes())
            s["ws"] = okvq.norm_rotary_workspace(B, n) if op == "norm_grad" else None
        return s
    s["cache"] = _cache(case, g, lens)
    s["q"] = torch.randn(B, Hq, n, D, generator=g, device="cuda").to(dt)
    s["out"] = torch.zeros_like(s["q"])
    if op == "tree":
        s["k"], s["v"] = (_rows(g, B, H, n, 0).to(dt) for _ in range(2))
        s["visible"] = _trees(case, seed, news, n)
    if own:
        import paper_2609_11582_amd as okvq
        c = s["cache"]
        s["own"] = okvq.Q8Cache(B, H, Hq, c["k_codes"].shape[1], c["block_table"].shape[1], page_tokens=case["page"],
                                format=case["format"], dtype=case["dtype"], buffers=c)
        s["ws"] = okvq.q8_tree_workspace(s["own"].dims, n) if op == "tree" else okvq.q8_workspace(s["own"].dims, max(lens), n)
    return s


# ---- the plain form -------------------------------------------------------------------------------


def _angles(pos):
    """cos and sin [B][1][n][64] of positions [B][3][n]; angles in 64 bits."""
    f = torch.tensor(_inv_freq(), dtype=torch.float64, device=pos.device)
    angle = pos.double()[:, _axes(), :].transpose(1, 2)[:, None] * f
    return angle.cos().float(), angle.sin().float()


def _rotate(y, c, s, adjacent):
    a, b = (y[..., 0::2], y[..., 1::2]) if adjacent else (y[..., :PAIRS], y[..., PAIRS:])
    a, b = a * c - b * s, b * c + a * s
    return torch.stack((a, b), -1).flatten(-2) if adjacent else torch.cat((a, b), -1)


def _norm(case, x, w, pos):
    """x [B][heads][n][128]: normed, weighted, rotated."""
    x = x.float()
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    return _rotate(y, *_angles(pos), case["adjacent"])


def _norm_grad(case, x, w, pos, grad):
    """Gradients of the rows and of the weights (of the rows given, zero elsewhere)."""
    x = x.float()
    c, s = _angles(pos)
    g = _rotate(grad.float(), c, -s, case["adjacent"])
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    xn = x * r
    h = g * w
    return r * (h - xn * (h * xn).mean(-1, keepdim=True)), (g * xn).sum((0, 1, 2), dtype=torch.float64).float()


def _blocks(case, c, blocks):
    """Keys and values [B][H][32 nb][128] of the blocks [B][nb] of the sequences, in 32 bits."""
    T, H = case["page"], case["kv_heads"]
    B, nb = blocks.shape
    mp = c["block_table"].shape[1]
    page = c["block_table"].gather(1, (blocks * W // T).clamp(0, mp - 1)).clamp(min=0).long()
    sub = blocks * W % T // W
    kind = torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn
    k = c["k_codes"][0].view(-1, H, T // W, W, D)[page, :, sub].view(kind).float() * c["k_scale"][0][page, :, sub][..., None, None]
    v = _unpack_values(c["v_codes"][0][page, :, sub].view(kind).float()) * c["v_scale"][0][page, :, sub][..., None, None]
    return (x.transpose(1, 2).reshape(B, H, nb * W, D) for x in (k, v))


def _visible_blocks(case, c, n, news):
    """Blocks that the rows may see [B][nb], and the tokens in them [B][32 nb], -1 where a token is none or is there twice."""
    lens, nall = c["seq_lens"].long()[:, None], _up(case["tokens"], W)
    sink = min(_up(case["sinks"], W), nall)
    count = min(_up(case["window"] + n, W) + 1, nall) if case["window"] else nall
    first = ((lens - news.long()[:, None] + 1 - case["window"]).clamp(min=0) // W).clamp(max=max(nall - count, 0)) if case["window"] else lens * 0
    at = torch.arange(count, device="cuda")
    blocks = torch.cat((torch.arange(sink, device="cuda").expand(len(lens), sink), first + at), 1)
    twice = torch.cat((torch.zeros(len(lens), sink, dtype=torch.bool, device="cuda"), first + at < sink), 1)
    token = blocks[..., None] * W + torch.arange(W, device="cuda")
    token = torch.where(twice[..., None] | (token >= lens[..., None]), -1, token).flatten(1)
    return blocks, token


def _softmax(q, k, v, seen):
    """Rows q [B][H][G][n][128] over k, v [B][H][N][128]; seen [B][n][N]. Zeros for a row that sees nothing."""
    B, H, G, n, _ = q.shape
    N = k.shape[2]
    score = (torch.matmul(q.reshape(B, H, G * n, D), k.transpose(2, 3).contiguous()) * SM_SCALE).view(B, H, G, n, N)
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p.view(B, H, G * n, N), v).view(B, H, G, n, D) / torch.where(total > 0, total, 1.0)


def _bits(words, n):
    """bool [B][n][n]: whether a row's mask names a draft."""
    j = torch.arange(n, device="cuda")
    return (words[..., j // 32] >> (j % 32) & 1).bool()


def _attend(case, c, q, news, out, draft=None):
    B, Hq, n, _ = q.shape
    H = case["kv_heads"]
    i = torch.arange(n, device="cuda")
    lens, rows = c["seq_lens"].long()[:, None], news.long()[:, None]
    blocks, token = _visible_blocks(case, c, n, news if draft is None else news * 0)
    k, v = _blocks(case, c, blocks)
    if draft is None:
        last = lens - rows + i                           # [B][n]: the row's own token
    else:
        named = _bits(draft[2], n) & (i < rows[..., None])
        last = lens + named.sum(-1) - 1                  # the place behind the cache that the row's line has come to
    seen = (token[:, None] >= 0) & (token[:, None] <= last[..., None])
    if case["window"]:
        seen &= (token[:, None] < case["sinks"]) | (token[:, None] > last[..., None] - case["window"])
    if draft is not None:
        k, v = torch.cat((k, draft[0].float()), 2), torch.cat((v, draft[1].float()), 2)
        seen = torch.cat((seen, named), 2)
    o = _softmax(q.float().view(B, H, Hq // H, n, D), k, v, seen)
    return torch.where((i < rows)[:, None, :, None], o.reshape(B, Hq, n, D).to(q.dtype), out)


# ---- one pass -------------------------------------------------------------------------------------


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        import paper_2609_11582_amd as okvq
    if op in ("norm", "norm_grad"):
        q, k = s["q"].transpose(1, 2), s["k"].transpose(1, 2)
        if own:
            flags = okvq.OKVQ_ROTARY_ADJACENT if case["adjacent"] else 0
            if op == "norm":
                okvq.okvq_norm_rotary(s["rotary"], q, k, s["q_weight"], s["k_weight"], EPS, s["pos"], s["q_out"], s["k_out"],
                                      lens=s["news"], flags=flags)
                return {"q": s["q_out"], "k": s["k_out"]}
            okvq.okvq_norm_rotary_backward(s["rotary"], q, k, s["q_weight"], s["k_weight"], EPS, s["pos"], s["q_grad"], s["k_grad"],
                                           s["dq"].transpose(1, 2), s["dk"].transpose(1, 2), s["dq_weight"], s["dk_weight"], s["ws"],
                                           lens=s["news"], flags=flags)
            return {f: s[f] for f in ("dq", "dk", "dq_weight", "dk_weight")}
        here = (torch.arange(s["n"], device="cuda") < s["news_dev"][:, None])[:, None, :, None]
        out = {}
        for f, x in (("q", q), ("k", k)):
            if op == "norm":
                out[f] = torch.where(here, _norm(case, x, s[f + "_weight"], s["pos"]).to(x.dtype), s[f + "_out"])
            else:
                dx, dw = _norm_grad(case, x, s[f + "_weight"], s["pos"], torch.where(here, s[f + "_grad"], 0.0))
                out["d" + f] = torch.where(here, dx.to(x.dtype), s["d" + f].transpose(1, 2)).transpose(1, 2)
                out["d" + f + "_weight"] = dw
        return out
    if op == "window":
        if own:
            okvq.okvq_q8_window_attention(s["own"], 0, s["lens"], s["q"], s["news"], s["news_dev"], s["n"], case["window"],
                                          case["sinks"], SM_SCALE, s["out"], s["ws"])
            return s["out"]
        return _attend(case, s["cache"], s["q"], s["news_dev"], s["out"])
    if own:
        okvq.okvq_q8_tree_attention(s["own"], 0, s["lens"], s["q"], s["k"], s["v"], s["visible"], s["news"], s["news_dev"], s["n"],
                                    SM_SCALE, s["out"], s["ws"], window=case["window"], sinks=case["sinks"])
        return s["out"]
    return _attend(case, s["cache"], s["q"], s["news_dev"], s["out"], (s["k"], s["v"], s["visible"]))


# ---- from the definitions, in 64 bits -------------------------------------------------------------


def _turned(x, pos, adjacent):
    """x [heads][n][128] in 64 bits, a pair as a complex number times exp(i angle)."""
    first, second = (x[..., 0::2], x[..., 1::2]) if adjacent else x.chunk(2, -1)
    freq = torch.tensor([math.exp(-math.log(THETA) * i / PAIRS) for i in range(PAIRS)], dtype=torch.float64, device="cuda")
    which = torch.tensor([a for a in range(3) for _ in range(SECTIONS[a])], device="cuda")
    angle = pos[which].double().T * freq
    z = torch.complex(first, second) * torch.polar(torch.ones_like(angle), angle)
    return torch.view_as_real(z).flatten(-2) if adjacent else torch.cat((z.real, z.imag), -1)


def _sequence(case, c, b, h, n):
    """Keys and values [n][128] of one sequence and head as the cache holds them."""
    T = case["page"]
    kind = torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn
    table = c["block_table"][b, :_up(n, T)].long()
    t, ch = torch.arange(W, device="cuda")[:, None], torch.arange(D, device="cuda")[None]
    byte = 1024 * (ch // 32) + 16 * (16 * (t // 4 % 4) + ch % 16) + 8 * (ch // 16 % 2) + 4 * (t // 16) + t % 4
    k = c["k_codes"][0, table, h].view(kind).double().reshape(-1, W, D) * c["k_scale"][0, table, h].double().reshape(-1, 1, 1)
    v = c["v_codes"][0, table, h].view(kind).double().reshape(-1, D * W)[:, byte.reshape(-1)].reshape(-1, W, D)
    v = v * c["v_scale"][0, table, h].double().reshape(-1, 1, 1)
    return k.reshape(-1, D)[:n], v.reshape(-1, D)[:n]


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    B, H, Hq, op, n = case["batch"], case["kv_heads"], case["q_heads"], case["op"], s["n"]
    if op in ("norm", "norm_grad"):
        out = {}
        for f in ("q", "k"):
            x = s[f].double().requires_grad_(op == "norm_grad")
            w = s[f + "_weight"].double().requires_grad_(op == "norm_grad")
            rows = []
            for b, m in enumerate(s["news"]):
                own_rows = x[b, :m].transpose(0, 1)
                length = torch.linalg.vector_norm(own_rows, dim=-1, keepdim=True)
                y = _turned(own_rows * w / torch.sqrt(length ** 2 / D + EPS), s["pos"][b, :, :m], case["adjacent"])
                rows.append(y)
            if op == "norm":
                out[f] = torch.zeros(B, x.shape[2], n, D, dtype=torch.float64, device="cuda")
                for b, y in enumerate(rows):
                    out[f][b, :, :y.shape[1]] = y
            else:
                total = sum((y * s[f + "_grad"][b, :, :y.shape[1]].double()).sum() for b, y in enumerate(rows))
                out["d" + f], out["d" + f + "_weight"] = torch.autograd.grad(total, (x, w))
        return out
    out = torch.zeros(B, Hq, n, D, dtype=torch.float64, device="cuda")
    G, window, sinks = Hq // H, case["window"] or (1 << 40), case["sinks"]
    for b, (L, m) in enumerate(zip(s["lens"], s["news"])):
        if op == "tree":
            masks = [sum((int(x) & 0xffffffff) << 32 * i for i, x in enumerate(row)) for row in s["visible"][b, :m].tolist()]
            named = [[j for j in range(m) if mask >> j & 1] for mask in masks]
        for h in range(H if m else 0):
            k, v = _sequence(case, s["cache"], b, h, L)
            step = m if op == "tree" else 512
            for i0 in range(0, m, step):
                i1 = min(i0 + step, m)
                q = s["q"][b, h * G:(h + 1) * G, i0:i1].double()
                if op == "tree":
                    at = torch.tensor([L + len(x) - 1 for x in named], device="cuda")
                else:
                    at = torch.arange(L - m + i0, L - m + i1, device="cuda")
                lo = max(0, int(at.min()) - window + 1)
                t = torch.arange(L, device="cuda")
                t = t[(t < sinks) | ((t >= lo) & (t <= int(at.max())))]
                hidden = (t > at[:, None]) | ((t <= at[:, None] - window) & (t >= sinks))
                kk, vv = k[t], v[t]
                if op == "tree":
                    kk, vv = torch.cat((kk, s["k"][b, h, :m].double())), torch.cat((vv, s["v"][b, h, :m].double()))
                    drafts = torch.ones(m, m, dtype=torch.bool, device="cuda")
                    for i, x in enumerate(named):
                        drafts[i, x] = False
                    hidden = torch.cat((hidden, drafts), 1)
                score = (q.reshape(-1, D) @ kk.T.contiguous()).view(G, i1 - i0, -1) * SM_SCALE
                p = torch.softmax(score.masked_fill(hidden, -math.inf), -1).nan_to_num(0.0)
                out[b, h * G:(h + 1) * G, i0:i1] = (p.view(G * (i1 - i0), -1) @ vv).view(G, i1 - i0, D)
    return out
