"""Rotary positions and the paged 8-bit cache in plain numpy.

* ``rotate``: the rotation of include/okvq.h's okvq_rotary in float64;
* ``quantize_block`` / ``pack_values``: the 8-bit codec's documented fp32 order and value byte order;
* ``attention``: softmax attention in float64 over dequantized rows, with the error bound that the kernels'
  roundings leave;
* ``PagedModel``: the page calls as a sequential program over Python lists.
"""

from __future__ import annotations

import numpy as np

W, D = 32, 128
TOP = {"int8": np.float32(127), "e4m3": np.float32(448)}


def rotate(x, pos, inv_freq, axes, inverse=False, adjacent=False):
    """x [B][heads][n][128] (float64), pos [B][3][n] integers."""
    angle = pos[:, list(axes), :].astype(np.float64).transpose(0, 2, 1)[:, None] * np.asarray(inv_freq)
    c, s = np.cos(angle), np.sin(angle) * (-1.0 if inverse else 1.0)
    y = np.empty_like(x)
    i, j = (slice(0, D, 2), slice(1, D, 2)) if adjacent else (slice(0, 64), slice(64, D))
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    return y


def _e4m3_table():
    """Values of the 256 codes (NaN for 0x7f and 0xff)."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v[c] = (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) * (-1 if c & 128 else 1)
    v[0x7f] = v[0xff] = np.nan
    return v


E4M3 = _e4m3_table()


def e4m3_encode(t):
    """Nearest e4m3 code of t (float32, |t| <= 448), ties to the even code."""
    a = np.abs(t.astype(np.float64))
    pos = E4M3[:0x7f]
    hi = np.searchsorted(pos, a).clip(0, 0x7e)
    lo = (hi - 1).clip(0)
    up, down = pos[hi] - a, a - pos[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)) | (a == pos[hi]), hi, lo)
    return (code | np.where(np.signbit(t), 128, 0)).astype(np.uint8)


def quantize_block(rows, fmt):
    """rows [<= 32][128] float32 -> (codes u8 [32][128], scale float32)."""
    x = np.zeros((W, D), np.float32)
    x[:len(rows)] = rows
    scale = np.float32(np.abs(x).max()) * (np.float32(1) / TOP[fmt])
    if not scale > 0:
        scale = np.float32(1)
    t = np.clip(x / scale, -TOP[fmt], TOP[fmt])
    code = np.rint(t).astype(np.int8).view(np.uint8) if fmt == "int8" else e4m3_encode(t)
    return code, scale


def values_of(codes, fmt):
    return codes.view(np.int8).astype(np.float64) if fmt == "int8" else E4M3[codes]


def value_bytes():
    """Byte of (token, channel) in a value block, [32][128]."""
    t, c = np.arange(W)[:, None], np.arange(D)[None]
    return 1024 * (c // 32) + 16 * (16 * (t // 4 % 4) + c % 16) + 8 * (c // 16 % 2) + 4 * (t // 16) + t % 4


def pack_values(codes):
    out = np.empty(W * D, np.uint8)
    out[value_bytes().reshape(-1)] = codes.reshape(-1)
    return out


def read_sequence(cache, layer, b, h, n, fmt):
    """Dequantized keys and values [n][128] (float64) of a slot; cache: numpy arrays by buffer name."""
    T = cache["k_codes"].shape[3]
    ks, vs = [], []
    for t0 in range(0, n, W):
        page, sub = cache["block_table"][b, t0 // T], t0 % T // W
        ks.append(values_of(cache["k_codes"][layer, page, h, sub * W:(sub + 1) * W], fmt) * float(cache["k_scale"][layer, page, h, sub]))
        v = values_of(cache["v_codes"][layer, page, h, sub], fmt)[value_bytes()]
        vs.append(v * float(cache["v_scale"][layer, page, h, sub]))
    if not ks:
        return np.zeros((0, D)), np.zeros((0, D))
    return np.concatenate(ks)[:n], np.concatenate(vs)[:n]


def attention(q, k, v, seen, sm_scale, half_step):
    """q [rows][128], k, v [n][128] in float64; row r sees the first seen[r] tokens. Returns (output, bound).

    The bound per element, for a kernel that accumulates in fp32: the weights enter the value product rounded to
    fp16 (2^-11 of each term); a score is off by its 128 sums and its scaling (132 roundings of 2^-24 of its absolute
    sum) and the difference to the reference by 2^-23 of the largest score, which the exponential carries into
    numerator and denominator; exponential, sums over tokens and the final factor 2^-18; the output's own rounding
    half_step. Weights below fp16's normal range are off by 2^-32 of the largest term, codes being at most 448."""
    out, bound = np.zeros((len(q), D)), np.zeros((len(q), D))
    for r, n in enumerate(seen):
        if n <= 0:
            continue
        s = k[:n] @ q[r] * sm_scale
        p = np.exp(s - s.max())
        out[r] = p @ v[:n] / p.sum()
        mass = p @ np.abs(v[:n]) / p.sum()
        delta = 132 * 2.0 ** -24 * (np.abs(k[:n]) @ np.abs(q[r])).max() * abs(sm_scale) + 2.0 ** -22 * np.abs(s).max()
        least = n * 2.0 ** -31 * 448 * (p[:, None] * np.abs(v[:n])).max() / p.sum()
        bound[r] = mass * (2.0 ** -11 + 2 * delta + 2.0 ** -18) * (1 + half_step) + half_step * np.abs(out[r]) + least + 2.0 ** -24
    return out, bound


class PagedModel:
    """Tables, lengths and holders of a cache under the page calls, one slot after the other, with the page copies
    that they make in `moves` (from, to)."""

    def __init__(self, batch, num_pages, page_tokens, max_pages):
        self.B, self.P, self.T, self.mp = batch, num_pages, page_tokens, max_pages
        self.table = [[] for _ in range(batch)]
        self.lens = [0] * batch
        self.refs = [0] * num_pages
        self.short = 0
        self.moves = []

    def _page(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def extend(self, more):
        self.moves = []
        more = [max(m, 0) for m in more]
        saved = ([list(t) for t in self.table], list(self.lens), list(self.refs))
        try:
            for b, m in enumerate(more):
                if m == 0:
                    continue
                if self.lens[b] + m > self.mp * self.T:
                    raise ValueError
                if self.lens[b] % self.T and self.refs[self.table[b][-1]] > 1:
                    old = self.table[b][-1]
                    self.refs[old] -= 1
                    new = self._page()
                    self.table[b][-1] = new
                    self.moves.append((old, new))
                while len(self.table[b]) * self.T < self.lens[b] + m:
                    self.table[b].append(self._page())
                self.lens[b] += m
        except ValueError:
            self.table, self.lens, self.refs = saved
            self.moves, self.short = [], 1
            return [0] * self.B
        return more

    def free(self, slots):
        for b in slots:
            for p in self.table[b]:
                self.refs[p] -= 1
            self.table[b], self.lens[b] = [], 0

    def fork(self, src, dst):
        for s, d in zip(src, dst):
            self.free([d])
            self.table[d], self.lens[d] = list(self.table[s]), self.lens[s]
            for p in self.table[s]:
                self.refs[p] += 1

    def compact(self):
        live = [p for p in range(self.P) if self.refs[p] > 0]
        n = len(live)
        holes = [p for p in range(n) if self.refs[p] == 0]
        self.moves = list(zip([p for p in live if p >= n], holes))
        to = dict(self.moves)
        self.table = [[to.get(p, p) for p in t] for t in self.table]
        for a, b in self.moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
        return n

    def arrays(self):
        table = np.full((self.B, self.mp), -1, np.int32)
        for b, t in enumerate(self.table):
            table[b, :len(t)] = t
        return {"block_table": table, "seq_lens": np.array(self.lens, np.int32), "page_refs": np.array(self.refs, np.int32)}
