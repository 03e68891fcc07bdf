"""Refusals of the head norm's calls that need no GPU: nothing here could reach the device."""

import ctypes
import math

import pytest
import torch

from paper_2609_11582_amd import q8

FAKE = ctypes.c_void_p(4096)  # aligned, never dereferenced: validation fails first
OFF = ctypes.c_void_p(4104)
PAR = q8.make_rotary([0.5] * 64, [0] * 64)
WS = q8.okvq_norm_rotary_workspace_bytes(2, 4)


def rows(data=4096, b=2048, h=512, t=128):
    return ctypes.byref(q8.Rows(data, b, h, t))


def forward(par=ctypes.byref(PAR), batch=2, hq=4, hk=4, n=4, q=rows(), k=rows(), qw=FAKE, kw=FAKE, eps=1e-6, pos=FAKE, lens=(0, 0),
            qo=rows(), ko=rows(), dtype=0, flags=0):
    lens = None if lens is None else (ctypes.c_int32 * 2)(*lens)
    return q8.lib().okvq_norm_rotary(par, batch, hq, hk, n, q, k, qw, kw, ctypes.c_float(eps), pos, lens, qo, ko, dtype, flags, None)


def backward(par=ctypes.byref(PAR), batch=2, hq=4, hk=4, n=4, q=rows(), k=rows(), qw=FAKE, kw=FAKE, eps=1e-6, pos=FAKE, lens=(9, 9),
             qo=rows(), ko=rows(), dtype=0, flags=0, gq=rows(), gk=rows(), dqw=FAKE, dkw=ctypes.c_void_p(8192), ws=FAKE, nbytes=WS):
    lens = None if lens is None else (ctypes.c_int32 * 2)(*lens)
    return q8.lib().okvq_norm_rotary_backward(par, batch, hq, hk, n, q, k, qw, kw, ctypes.c_float(eps), pos, lens, gq, gk, qo, ko, dqw,
                                              dkw, dtype, ws, nbytes, flags, None)


BAD = [dict(par=None), dict(batch=0), dict(batch=65536), dict(n=-1), dict(pos=OFF), dict(pos=None), dict(dtype=2), dict(dtype=-1),
       dict(flags=1), dict(flags=4), dict(q=None), dict(qo=None), dict(ko=None), dict(hq=0), dict(hk=-1),
       dict(q=rows(4104)), dict(k=rows(0)), dict(qo=rows(t=130)), dict(ko=rows(h=-8)), dict(qw=None), dict(qw=OFF), dict(kw=None),
       dict(eps=0.0), dict(eps=-1e-6), dict(eps=1e-39), dict(eps=math.inf), dict(eps=math.nan), dict(lens=(-1, 0)), dict(lens=(0, 5)),
       dict(lens=(4, 4), qo=rows(t=64)), dict(lens=None, ko=rows(b=0)), dict(lens=(4, 4), qo=rows(h=128, t=128))]


@pytest.mark.parametrize("kw", BAD, ids=[f"{i}-{'-'.join(kw)}" for i, kw in enumerate(BAD)])
@pytest.mark.parametrize("call", [forward, backward])
def test_refused(call, kw):
    assert call(**kw) == -1


def test_accepted_without_rows():
    assert forward() == 0                                                  # no rows: nothing launched
    assert forward(n=0, lens=None, pos=None, q=rows(0), qo=rows(0)) == 0
    assert forward(q=None, qo=None, qw=None) == 0 and forward(k=None, ko=None, kw=None, hk=0) == 0
    assert forward(hq=65535, hk=1) == -2


def test_backward_refused():
    for kw in (dict(gq=None), dict(gk=None), dict(gq=rows(4104)), dict(gk=rows(t=4)), dict(dqw=None), dict(dkw=OFF), dict(dkw=FAKE)):
        assert backward(**dict(lens=(0, 0)) | kw) == -1
    assert backward(lens=(0, 0), k=None, ko=None, kw=None) == -1           # a gradient without its rows
    for kw in (dict(ws=None), dict(ws=OFF), dict(nbytes=WS - 1)):
        assert backward(**dict(lens=(0, 0)) | kw) == -4


def test_workspace():
    assert WS == 768 << 10 and q8.okvq_norm_rotary_workspace_bytes(65535, 1 << 20) == WS
    assert q8.okvq_norm_rotary_workspace_bytes(0, 4) == 0 and q8.okvq_norm_rotary_workspace_bytes(1, -1) == 0
    with pytest.raises(ValueError):
        q8.okvq_norm_rotary_workspace_bytes(1 << 32, 4)


def test_binding_refuses_host_tensors():
    x, w, pos = torch.zeros(1, 2, 4, 128, dtype=torch.float16), torch.zeros(128), torch.zeros(1, 3, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        q8.okvq_norm_rotary(PAR, x, None, w, None, 1e-6, pos, x, None)
    with pytest.raises(ValueError):
        q8.okvq_norm_rotary_backward(PAR, x, None, w, None, 1e-6, pos, x, None, x, None, w, None, w)
