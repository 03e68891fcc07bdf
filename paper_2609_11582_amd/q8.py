"""Binding of the rotary positions, of the head norms and of the paged 8-bit cache of libokvq.so (include/okvq.h): argument
marshalling and size checks only, as in ``okvq``. Tensors have to be on the current device and of the stated
type; the stream is torch's current one unless one is given."""

from __future__ import annotations

import ctypes
import functools
import struct
from typing import Sequence

import torch

from .okvq import OkvqError, _check, _need_len, _stream
from .okvq import lib as _okvq_lib

OKVQ_F16 = 0
OKVQ_BF16 = 1
OKVQ_ROTARY_INVERSE = 1   # the opposite angle: the gradient of the rotation
OKVQ_ROTARY_ADJACENT = 2  # pairs of channels (2i, 2i + 1) instead of (i, i + 64)
OKVQ_Q8_INT8 = 0
OKVQ_Q8_E4M3 = 1
OKVQ_Q8_CROSS = 1         # every row sees the whole sequence
Q8_FORMATS = {"int8": OKVQ_Q8_INT8, "e4m3": OKVQ_Q8_E4M3}
Q8_DTYPES = {"fp16": (OKVQ_F16, torch.float16), "bf16": (OKVQ_BF16, torch.bfloat16)}
_ROW_TYPES = {torch.float16: OKVQ_F16, torch.bfloat16: OKVQ_BF16}
# buffer ids 0..9 of okvq_q8_buffer_bytes (OKVQ_Q8_BUF_*)
Q8_BUFFERS = ("k_codes", "v_codes", "k_scale", "v_scale", "k_stage", "v_stage", "block_table", "seq_lens", "page_refs",
              "status")


class RotaryParams(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_double * 64), ("axis", ctypes.c_uint8 * 64)]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64)]


class Q8Dims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("layers", "batch", "num_kv_heads", "num_q_heads", "head_dim", "num_pages",
                                              "page_tokens", "max_pages", "format", "dtype")]


class Q8Struct(ctypes.Structure):
    _fields_ = [("dims", Q8Dims)] + [(n, ctypes.c_void_p) for n in Q8_BUFFERS]


_ready = None


def lib() -> ctypes.CDLL:
    global _ready
    if _ready is None:
        L = _okvq_lib()
        vp, i32, u32, sz, f32, P = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_size_t, ctypes.c_float,
                                   ctypes.POINTER)
        for name, res, args in (
                # okvq_rows as packed bytes (_rows_of) or Rows structures, host counts as packed bytes (_ints) or arrays
                ("okvq_rotary", i32, [P(RotaryParams), i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, i32, u32, vp]),
                ("okvq_norm_rotary", i32, [P(RotaryParams), i32, i32, i32, i32, vp, vp, vp, vp, f32, vp, vp, vp, vp, i32, u32, vp]),
                ("okvq_norm_rotary_workspace_bytes", sz, [i32, i32]),
                ("okvq_norm_rotary_backward", i32, [P(RotaryParams), i32, i32, i32, i32, vp, vp, vp, vp, f32, vp, vp, vp, vp, vp, vp,
                                                    vp, vp, i32, vp, sz, u32, vp]),
                ("okvq_q8_buffer_bytes", sz, [P(Q8Dims), i32]),
                ("okvq_q8_append", i32, [P(Q8Struct), i32, vp, vp, vp, vp, vp, i32, vp]),
                ("okvq_q8_workspace_bytes", sz, [P(Q8Dims), i32, i32]),
                ("okvq_q8_attention", i32, [P(Q8Struct), i32, vp, vp, vp, vp, i32, ctypes.c_float, vp, vp, sz, u32, vp]),
                ("okvq_q8_window_attention", i32, [P(Q8Struct), i32, vp, vp, vp, vp, i32, i32, i32, f32, vp, vp, sz, vp]),
                ("okvq_q8_tree_workspace_bytes", sz, [P(Q8Dims), i32]),
                ("okvq_q8_tree_attention", i32, [P(Q8Struct), i32, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, f32, vp, vp, sz, vp]),
                ("okvq_q8_page_workspace_bytes", sz, [P(Q8Dims)]),
                ("okvq_q8_extend", i32, [P(Q8Struct), vp, vp, vp, sz, vp]),
                ("okvq_q8_fork", i32, [P(Q8Struct), vp, vp, i32, vp]),
                ("okvq_q8_free", i32, [P(Q8Struct), vp, i32, vp]),
                ("okvq_q8_compact", i32, [P(Q8Struct), vp, sz, vp]),
                ("okvq_q8_status", i32, [P(Q8Struct), P(i32), vp])):
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _ready = L
    return _ready


# Host time of a call counts at a decode step: the checks below read each property of a tensor once, and a call asks
# for the current device once.
_device = torch.cuda.current_device


def _need(t: torch.Tensor, nbytes: int, dtype, name: str, device: int) -> int:
    """The tensor's address, once it is contiguous, on the current device, of the type and large enough."""
    if not isinstance(t, torch.Tensor) or not t.is_contiguous() or t.get_device() != device:
        _refuse(t, name, device)
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: {t.dtype}, expected {dtype}")
    if t.nbytes < nbytes:
        raise ValueError(f"{name}: {t.nbytes} bytes, at least {nbytes} needed")
    return t.data_ptr()


def _need_rows(t: torch.Tensor, shape, dtype, name: str, device: int) -> int:
    """The address of contiguous rows of this shape, dimensions of one entry aside: as many bytes in another order (token by
    token, or rows of a longer buffer) would be read as other rows."""
    if isinstance(t, torch.Tensor) and t.shape != shape and [n for n in t.shape if n != 1] != [n for n in shape if n != 1]:
        raise ValueError(f"{name}: {list(t.shape)}, expected {list(shape)}")
    return _need(t, 0, dtype, name, device)


def _refuse(t, name: str, device: int):
    if not isinstance(t, torch.Tensor) or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous device tensor")
    raise ValueError(f"{name}: on {t.device}, but the current device is {device}")


def _int(x, name: str, low=-(1 << 31), high=(1 << 31) - 1) -> int:
    """x as a whole number of 32 bits: ctypes would drop the bits above them."""
    x = int(x)
    if not low <= x <= high:
        raise ValueError(f"{name}: {x} does not fit 32 bits")
    return x


@functools.lru_cache(maxsize=None)
def _int_packer(n: int):
    return struct.Struct(f"{n}i").pack


def _ints(xs: Sequence[int], n: int, name: str) -> bytes:
    """int32 [n] as packed bytes, which refuse what 32 bits do not hold."""
    if len(xs) != n:
        raise ValueError(f"{name}: {len(xs)} entries, expected {n}")
    try:
        return _int_packer(n)(*xs)
    except struct.error:
        try:
            return _int_packer(n)(*[int(x) for x in xs])
        except struct.error:
            raise ValueError(f"{name}: entries have to fit 32 bits") from None


# ---- rotary positions ----------------------------------------------------------------------------


def make_rotary(inv_freq: Sequence[float], axes: Sequence[int]) -> RotaryParams:
    """Frequencies (radians per position) of a row's 64 pairs of channels and the axis (0..2) that turns each."""
    _need_len(inv_freq, 64, "inv_freq")
    _need_len(axes, 64, "axes")
    if any(not 0 <= int(a) <= 2 for a in axes):
        raise ValueError("axes: 0, 1 or 2 for every pair")
    return RotaryParams((ctypes.c_double * 64)(*[float(f) for f in inv_freq]), (ctypes.c_uint8 * 64)(*[int(a) for a in axes]))


_pack_rows = struct.Struct("Pqqq").pack  # the layout of Rows


def _rows_of(t: torch.Tensor, shape, dtype, name: str, device: int) -> bytes:
    if not isinstance(t, torch.Tensor) or t.get_device() != device:
        raise ValueError(f"{name}: expected a tensor on the current device {device}")
    if t.shape != shape or t.dtype != dtype:
        raise ValueError(f"{name}: {list(t.shape)} {t.dtype}, expected {list(shape)} {dtype}")
    b, h, n, c = t.stride()
    if c != 1:
        raise ValueError(f"{name}: the channels of a row have to lie side by side")
    # the stride of a dimension of one entry is whatever torch left there: it moves nothing
    return _pack_rows(t.data_ptr(), b if shape[0] > 1 else 0, h if shape[1] > 1 else 0, n if shape[2] > 1 else 0)


def okvq_rotary(rotary: RotaryParams, q, k, positions, q_out, k_out, lens=None, flags=0, stream=None, check=True) -> int:
    """Rotate queries and keys: q, k, q_out, k_out [batch][heads][tokens][128] with any strides over the first
    three dimensions (``x.view(B, n, heads, 128).transpose(1, 2)`` for a projection's rows), or None in pairs;
    positions int32 [batch][3][tokens]; lens: rows of each sequence (None: all). In place where an output is its
    input."""
    some = q if q is not None else k
    if (not isinstance(some, torch.Tensor) or not some.is_cuda or some.dim() != 4 or some.dtype not in _ROW_TYPES
            or some.shape[3] != 128):
        raise ValueError("q, k: expected fp16 or bf16 device tensors [batch][heads][tokens][128]")
    if (q is None) != (q_out is None) or (k is None) != (k_out is None):
        raise ValueError("q, k: an input and an output of each, or neither")
    B, _, n, _ = some.shape
    dt, device = some.dtype, _device()
    rq = oq = rk = ok = None
    hq = hk = 0
    if q is not None:
        shape = q.shape
        hq = shape[1]
        rq, oq = _rows_of(q, shape, dt, "q", device), _rows_of(q_out, shape, dt, "q_out", device)
    if k is not None:
        hk = k.shape[1] if isinstance(k, torch.Tensor) and k.dim() == 4 else 0
        shape = (B, hk, n, 128)
        rk, ok = _rows_of(k, shape, dt, "k", device), _rows_of(k_out, shape, dt, "k_out", device)
    pos = _need(positions, 0, torch.int32, "positions", device)
    if positions.shape != (B, 3, n):
        raise ValueError(f"positions: {list(positions.shape)}, expected {[B, 3, n]}")
    st = lib().okvq_rotary(ctypes.byref(rotary), B, hq, hk, n, rq, rk, pos, None if lens is None else _ints(lens, B, "lens"),
                           oq, ok, _ROW_TYPES[dt], _int(flags, "flags", 0, (1 << 32) - 1), _stream(stream))
    if check and st:
        _check(st, "okvq_rotary")
    return st


# ---- head norms with the rotation ------------------------------------------------------------------


def _norm_sizes(q, k, positions):
    """(batch, tokens, type, device, address of the positions) of a call; which of q and k is given, and how their tensors agree, is
    checked with the rows."""
    some = q if q is not None else k
    if (not isinstance(some, torch.Tensor) or not some.is_cuda or some.dim() != 4 or some.dtype not in _ROW_TYPES
            or some.shape[3] != 128):
        raise ValueError("q, k: expected fp16 or bf16 device tensors [batch][heads][tokens][128]")
    B, _, n, _ = some.shape
    device = _device()
    pos = _need(positions, 0, torch.int32, "positions", device)
    if positions.shape != (B, 3, n):
        raise ValueError(f"positions: {list(positions.shape)}, expected {[B, 3, n]}")
    return B, n, some.dtype, device, pos


def _heads_of(x, name: str, *others) -> int:
    for y in others:
        if (y is None) != (x is None):
            raise ValueError(f"{name}: the rows and all that belongs to them, or none of it")
    return 0 if x is None else x.shape[1] if isinstance(x, torch.Tensor) and x.dim() == 4 else 0


def _norm_weight(w, name: str, device: int) -> int:
    if not isinstance(w, torch.Tensor) or w.shape != (128,):
        raise ValueError(f"{name}: expected 128 values")
    return _need(w, 0, torch.float32, name, device)


def okvq_norm_rotary(rotary: RotaryParams, q, k, q_weight, k_weight, eps, positions, q_out, k_out, lens=None, flags=0, stream=None,
                     check=True) -> int:
    """okvq_rotary of rows divided by their root mean square (of the 128 channels, with eps) and weighted: q_weight,
    k_weight fp32 [128], or None with their rows."""
    B, n, dt, device, pos = _norm_sizes(q, k, positions)
    hq, hk = _heads_of(q, "q", q_weight, q_out), _heads_of(k, "k", k_weight, k_out)
    rq = oq = wq = rk = ok = wk = None
    if q is not None:
        shape = (B, hq, n, 128)
        rq, oq = _rows_of(q, shape, dt, "q", device), _rows_of(q_out, shape, dt, "q_out", device)
        wq = _norm_weight(q_weight, "q_weight", device)
    if k is not None:
        shape = (B, hk, n, 128)
        rk, ok = _rows_of(k, shape, dt, "k", device), _rows_of(k_out, shape, dt, "k_out", device)
        wk = _norm_weight(k_weight, "k_weight", device)
    st = lib().okvq_norm_rotary(ctypes.byref(rotary), B, hq, hk, n, rq, rk, wq, wk, float(eps), pos,
                                None if lens is None else _ints(lens, B, "lens"), oq, ok, _ROW_TYPES[dt],
                                _int(flags, "flags", 0, (1 << 32) - 1), _stream(stream))
    if check and st:
        _check(st, "okvq_norm_rotary")
    return st


def okvq_norm_rotary_workspace_bytes(batch: int, n_tokens: int) -> int:
    return lib().okvq_norm_rotary_workspace_bytes(_int(batch, "batch"), _int(n_tokens, "n_tokens"))


def norm_rotary_workspace(batch: int, n_tokens: int, device="cuda") -> torch.Tensor:
    """A workspace of okvq_norm_rotary_workspace_bytes bytes for okvq_norm_rotary_backward (no contents needed)."""
    return torch.empty(max(okvq_norm_rotary_workspace_bytes(batch, n_tokens) + 15, 16) // 16 * 4, dtype=torch.float32, device=device)


def okvq_norm_rotary_backward(rotary: RotaryParams, q, k, q_weight, k_weight, eps, positions, q_grad, k_grad, dq, dk, dq_weight,
                              dk_weight, workspace, lens=None, flags=0, stream=None, check=True) -> int:
    """Gradients of okvq_norm_rotary: q_grad, k_grad of its outputs; dq, dk (rows, any strides) and dq_weight, dk_weight
    (fp32 [128], overwritten) are written."""
    B, n, dt, device, pos = _norm_sizes(q, k, positions)
    hq, hk = _heads_of(q, "q", q_weight, q_grad, dq, dq_weight), _heads_of(k, "k", k_weight, k_grad, dk, dk_weight)
    of_q = of_k = (None,) * 5
    if q is not None:
        shape = (B, hq, n, 128)
        of_q = (_rows_of(q, shape, dt, "q", device), _rows_of(q_grad, shape, dt, "q_grad", device), _rows_of(dq, shape, dt, "dq", device),
                _norm_weight(q_weight, "q_weight", device), _norm_weight(dq_weight, "dq_weight", device))
    if k is not None:
        shape = (B, hk, n, 128)
        of_k = (_rows_of(k, shape, dt, "k", device), _rows_of(k_grad, shape, dt, "k_grad", device), _rows_of(dk, shape, dt, "dk", device),
                _norm_weight(k_weight, "k_weight", device), _norm_weight(dk_weight, "dk_weight", device))
    st = lib().okvq_norm_rotary_backward(ctypes.byref(rotary), B, hq, hk, n, of_q[0], of_k[0], of_q[3], of_k[3], float(eps), pos,
                                         None if lens is None else _ints(lens, B, "lens"), of_q[1], of_k[1], of_q[2], of_k[2], of_q[4],
                                         of_k[4], _ROW_TYPES[dt], _need(workspace, 0, None, "workspace", device), workspace.nbytes,
                                         _int(flags, "flags", 0, (1 << 32) - 1), _stream(stream))
    if check and st:
        _check(st, "okvq_norm_rotary_backward")
    return st


# ---- paged 8-bit cache ---------------------------------------------------------------------------


def make_q8_dims(batch, num_kv_heads, num_q_heads, num_pages, max_pages, layers=1, page_tokens=64, format="int8",  # noqa: A002
                 dtype="fp16", head_dim=128) -> Q8Dims:
    sizes = layers, batch, num_kv_heads, num_q_heads, head_dim, num_pages, page_tokens, max_pages
    for x, (name, _) in zip(sizes, Q8Dims._fields_):
        _int(x, name)
    return Q8Dims(*sizes, Q8_FORMATS[format], Q8_DTYPES[dtype][0])


def okvq_q8_buffer_bytes(dims: Q8Dims, which: int) -> int:
    return lib().okvq_q8_buffer_bytes(ctypes.byref(dims), _int(which, "which"))


class Q8Cache:
    """The paged 8-bit cache of `layers` layers: device buffers sized by okvq_q8_buffer_bytes (torch allocations,
    a new cache's contents), or the caller's (`buffers`, by name, taken as they are).
    format "int8" or "e4m3"; dtype "fp16" or "bf16": the rows of keys, values, queries and outputs."""

    def __init__(self, batch, num_kv_heads, num_q_heads, num_pages, max_pages, layers=1, page_tokens=64,
                 format="int8", dtype="fp16", device="cuda", buffers=None):  # noqa: A002
        self.dims = make_q8_dims(batch, num_kv_heads, num_q_heads, num_pages, max_pages, layers, page_tokens, format, dtype)
        self.format, self.row_dtype = format, Q8_DTYPES[dtype][1]
        types = dict(k_codes=torch.uint8, v_codes=torch.uint8, k_scale=torch.float32, v_scale=torch.float32,
                     k_stage=self.row_dtype, v_stage=self.row_dtype)
        L, B, H, P, T, W = layers, batch, num_kv_heads, num_pages, page_tokens, 32
        shapes = dict(k_codes=(L, P, H, T, 128), v_codes=(L, P, H, T // W, 128 * W), k_scale=(L, P, H, T // W),
                      v_scale=(L, P, H, T // W), k_stage=(L, B, H, W, 128), v_stage=(L, B, H, W, 128),
                      block_table=(B, max_pages), seq_lens=(B,), page_refs=(P,), status=(4,))
        self.buffers = {}
        for i, name in enumerate(Q8_BUFFERS):
            dt = types.get(name, torch.int32)
            nbytes = okvq_q8_buffer_bytes(self.dims, i)
            if nbytes == 0:
                raise OkvqError(-1, f"okvq_q8_buffer_bytes({name})")
            if buffers is not None:
                t = buffers[name]
                _need(t, nbytes, dt, name, _device())
            else:
                t = torch.full(shapes[name], -1 if name == "block_table" else 0, dtype=dt, device=device)
            self.buffers[name] = t
        self.struct = Q8Struct(self.dims, *[self.buffers[n].data_ptr() for n in Q8_BUFFERS])
        self.device_index = self.buffers["k_codes"].get_device()
        self._ref = ctypes.byref(self.struct)
        self._sizes = batch, num_kv_heads, num_q_heads

    def __getitem__(self, name):
        return self.buffers[name]


def _cache_ref(cache: Q8Cache, device: int):
    if cache.device_index != device:
        raise ValueError(f"cache: on device {cache.device_index}, but the current device is {device}")
    return cache._ref


def okvq_q8_append(cache: Q8Cache, layer, lens, k_new, v_new, n_new, n_new_dev, n_max, stream=None, check=True) -> int:
    """Quantize the newest n_new[b] tokens (rows of k_new, v_new [B][H][n_max][128], contiguous) into one layer's pages,
    after okvq_q8_extend; lens: the lengths with them."""
    B, H, _ = cache._sizes
    dev, dt, n_max = _device(), cache.row_dtype, _int(n_max, "n_max")
    shape = (B, H, n_max, 128)
    st = lib().okvq_q8_append(_cache_ref(cache, dev), _int(layer, "layer"), _ints(lens, B, "lens"), _need_rows(k_new, shape, dt, "k_new", dev),
                              _need_rows(v_new, shape, dt, "v_new", dev), _ints(n_new, B, "n_new"),
                              _need(n_new_dev, B * 4, torch.int32, "n_new_dev", dev), n_max, _stream(stream))
    if check and st:
        _check(st, "okvq_q8_append")
    return st


def okvq_q8_workspace_bytes(dims: Q8Dims, max_seq_len: int, n_max: int = 1) -> int:
    return lib().okvq_q8_workspace_bytes(ctypes.byref(dims), _int(max_seq_len, "max_seq_len"), _int(n_max, "n_max"))


def q8_workspace(dims: Q8Dims, max_seq_len: int, n_max: int = 1, device="cuda") -> torch.Tensor:
    """A workspace of okvq_q8_workspace_bytes bytes for okvq_q8_attention (no contents needed)."""
    return torch.empty(max(okvq_q8_workspace_bytes(dims, max_seq_len, n_max) + 15, 16) // 16 * 4, dtype=torch.float32,
                       device=device)


def okvq_q8_attention(cache: Q8Cache, layer, lens, q, n_new, n_new_dev, n_max, sm_scale, out, workspace, flags=0,
                      stream=None, check=True) -> int:
    """Attention of contiguous rows q [B][Hq][n_max][128] over one layer into out (same shape and type): the newest n_new[b]
    tokens of each sequence, causal, or OKVQ_Q8_CROSS. lens: the lengths with the new tokens."""
    B, _, Hq = cache._sizes
    dev, dt, n_max = _device(), cache.row_dtype, _int(n_max, "n_max")
    shape = (B, Hq, n_max, 128)
    st = lib().okvq_q8_attention(_cache_ref(cache, dev), _int(layer, "layer"), _ints(lens, B, "lens"), _need_rows(q, shape, dt, "q", dev),
                                 _ints(n_new, B, "n_new"), _need(n_new_dev, B * 4, torch.int32, "n_new_dev", dev), n_max, float(sm_scale),
                                 _need_rows(out, shape, dt, "out", dev), _need(workspace, 0, None, "workspace", dev), workspace.nbytes,
                                 _int(flags, "flags", 0, (1 << 32) - 1), _stream(stream))
    if check and st:
        _check(st, "okvq_q8_attention")
    return st


def okvq_q8_window_attention(cache: Q8Cache, layer, lens, q, n_new, n_new_dev, n_max, window, sinks, sm_scale, out, workspace,
                             stream=None, check=True) -> int:
    """okvq_q8_attention of rows that see the newest `window` tokens up to their own and the first `sinks`; its workspace."""
    B, _, Hq = cache._sizes
    dev, dt, n_max = _device(), cache.row_dtype, _int(n_max, "n_max")
    shape = (B, Hq, n_max, 128)
    st = lib().okvq_q8_window_attention(
        _cache_ref(cache, dev), _int(layer, "layer"), _ints(lens, B, "lens"), _need_rows(q, shape, dt, "q", dev), _ints(n_new, B, "n_new"),
        _need(n_new_dev, B * 4, torch.int32, "n_new_dev", dev), n_max, _int(window, "window"), _int(sinks, "sinks"), float(sm_scale),
        _need_rows(out, shape, dt, "out", dev), _need(workspace, 0, None, "workspace", dev), workspace.nbytes, _stream(stream))
    if check and st:
        _check(st, "okvq_q8_window_attention")
    return st


def okvq_q8_tree_workspace_bytes(dims: Q8Dims, n_max: int) -> int:
    return lib().okvq_q8_tree_workspace_bytes(ctypes.byref(dims), _int(n_max, "n_max"))


def q8_tree_workspace(dims: Q8Dims, n_max: int, device="cuda") -> torch.Tensor:
    """A workspace of okvq_q8_tree_workspace_bytes bytes for okvq_q8_tree_attention (no contents needed)."""
    return torch.empty(max(okvq_q8_tree_workspace_bytes(dims, n_max) + 15, 16) // 16 * 4, dtype=torch.float32, device=device)


def q8_tree_visible(parents: Sequence[Sequence[int]], n_max: int, device="cuda") -> torch.Tensor:
    """Masks int32 [batch][n_max][ceil(n_max / 32)] for okvq_q8_tree_attention: of each slot, the parent of every draft, an
    earlier draft or -1 for one that follows the cache."""
    words = -(-n_max // 32)
    flat = []
    for b, slot in enumerate(parents):
        if len(slot) > n_max:
            raise ValueError(f"parents[{b}]: {len(slot)} drafts, at most {n_max}")
        masks = []
        for i, parent in enumerate(slot):
            if not -1 <= parent < i:
                raise ValueError(f"parents[{b}][{i}]: {parent}, expected -1 or an earlier draft")
            masks.append((masks[parent] if parent >= 0 else 0) | 1 << i)
        for mask in masks + [0] * (n_max - len(slot)):
            for w in range(words):
                bits = mask >> 32 * w & 0xffffffff
                flat.append(bits - (1 << 32) if bits >> 31 else bits)
    return torch.tensor(flat, dtype=torch.int32).view(len(parents), n_max, words).to(device)


def okvq_q8_tree_attention(cache: Q8Cache, layer, lens, q, k_draft, v_draft, visible, n_draft, n_draft_dev, n_max, sm_scale, out,
                           workspace, window=0, sinks=0, stream=None, check=True) -> int:
    """Attention of drafts that are not in the cache: rows q, out [B][Hq][n_max][128] and k_draft, v_draft [B][H][n_max][128]
    (contiguous); visible int32 [B][n_max][ceil(n_max / 32)], the drafts that each one sees (q8_tree_visible); lens: tokens
    in the cache. window 0: all of them."""
    B, H, Hq = cache._sizes
    dev, dt, n_max = _device(), cache.row_dtype, _int(n_max, "n_max")
    shape, drafts = (B, Hq, n_max, 128), (B, H, n_max, 128)
    st = lib().okvq_q8_tree_attention(
        _cache_ref(cache, dev), _int(layer, "layer"), _ints(lens, B, "lens"), _need_rows(q, shape, dt, "q", dev),
        _need_rows(k_draft, drafts, dt, "k_draft", dev), _need_rows(v_draft, drafts, dt, "v_draft", dev),
        _need_rows(visible, (B, n_max, -(-n_max // 32)), torch.int32, "visible", dev), _ints(n_draft, B, "n_draft"),
        _need(n_draft_dev, B * 4, torch.int32, "n_draft_dev", dev), n_max, _int(window, "window"), _int(sinks, "sinks"), float(sm_scale),
        _need_rows(out, shape, dt, "out", dev), _need(workspace, 0, None, "workspace", dev), workspace.nbytes, _stream(stream))
    if check and st:
        _check(st, "okvq_q8_tree_attention")
    return st


def okvq_q8_page_workspace_bytes(dims: Q8Dims) -> int:
    return lib().okvq_q8_page_workspace_bytes(ctypes.byref(dims))


def q8_page_workspace(dims: Q8Dims, device="cuda") -> torch.Tensor:
    """A workspace of okvq_q8_page_workspace_bytes bytes for okvq_q8_extend and okvq_q8_compact (no contents needed)."""
    return torch.empty(max(okvq_q8_page_workspace_bytes(dims) + 15, 16) // 16 * 4, dtype=torch.int32, device=device)


def okvq_q8_extend(cache: Q8Cache, n_new_dev, granted, workspace, stream=None, check=True) -> int:
    """Pages for n_new_dev[b] more tokens in every slot and the lengths advanced by them; granted (int32 [B], device):
    the same counts, or 0 for all where pages are short."""
    dev, nbytes = _device(), cache._sizes[0] * 4
    st = lib().okvq_q8_extend(_cache_ref(cache, dev), _need(n_new_dev, nbytes, torch.int32, "n_new_dev", dev),
                              _need(granted, nbytes, torch.int32, "granted", dev), _need(workspace, 0, None, "workspace", dev),
                              workspace.nbytes, _stream(stream))
    if check and st:
        _check(st, "okvq_q8_extend")
    return st


def okvq_q8_fork(cache: Q8Cache, src, dst, stream=None, check=True) -> int:
    """Slot dst[i] becomes a copy of slot src[i] that shares its pages."""
    n = len(src)
    st = lib().okvq_q8_fork(_cache_ref(cache, _device()), _ints(src, n, "src"), _ints(dst, n, "dst"), n, _stream(stream))
    if check and st:
        _check(st, "okvq_q8_fork")
    return st


def okvq_q8_free(cache: Q8Cache, slots, stream=None, check=True) -> int:
    """Empty slots; pages without another holder are free."""
    n = len(slots)
    st = lib().okvq_q8_free(_cache_ref(cache, _device()), _ints(slots, n, "slots"), n, _stream(stream))
    if check and st:
        _check(st, "okvq_q8_free")
    return st


def okvq_q8_compact(cache: Q8Cache, workspace, stream=None, check=True) -> int:
    """Move the pages in use to the front of the pool."""
    dev = _device()
    st = lib().okvq_q8_compact(_cache_ref(cache, dev), _need(workspace, 0, None, "workspace", dev), workspace.nbytes,
                               _stream(stream))
    if check and st:
        _check(st, "okvq_q8_compact")
    return st


def okvq_q8_status(cache: Q8Cache, stream=None):
    """(1 once an extend was short of pages, pages in use after the last compaction). Synchronizes `stream`."""
    words = (ctypes.c_int32 * 2)()
    _check(lib().okvq_q8_status(_cache_ref(cache, _device()), words, _stream(stream)), "okvq_q8_status")
    return int(words[0]), int(words[1])
