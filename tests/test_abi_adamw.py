"""AdamW's C call refuses bad arguments on the host, before any CUDA call."""
import ctypes as C
import struct
from array import array

import pytest

from paper_2411_10764_gb300 import mlt


@pytest.fixture(scope="module")
def L():
    return mlt.lib()


def _rate(lr=0.1, decay=0.0):
    return struct.unpack("<q", struct.pack("<ff", lr, decay))[0]


def _call(L, tensors=None, count=None, m=1 << 20, v=1 << 21, ms=1 << 22, vs=1 << 23, rule=True, **kw):
    r = mlt.AdamWRule(0.9, 0.999, 1e-8, 1, None, None, None, 32, 0)
    for k, x in kw.items():
        setattr(r, k, x)
    t = array("q", sum(tensors if tensors is not None else [_tensor()], []))
    return L.mlt_adamw(None, t.buffer_info()[0], len(t) // 6 if count is None else count, C.byref(r) if rule else None, m, v,
                       ms, vs)


def _tensor(param=4096, grad=8192, copy=0, n=10, kinds=0, rate=_rate()):
    return [param, grad, copy, n, kinds, rate]


@pytest.mark.parametrize("bad", [
    dict(tensors=[_tensor(param=0)]), dict(tensors=[_tensor(param=4097)]), dict(tensors=[_tensor(grad=8194)]),
    dict(tensors=[_tensor(copy=12290)]), dict(tensors=[_tensor(n=-1)]), dict(tensors=[_tensor(n=(1 << 40) + 1)]),
    dict(tensors=[_tensor(kinds=3)]), dict(tensors=[_tensor(kinds=5 << 16)]), dict(tensors=[_tensor(kinds=9 << 32)]),
    dict(tensors=[_tensor(rate=_rate(float("nan")))]), dict(tensors=[_tensor(rate=_rate(0.1, float("inf")))]),
    dict(tensors=[_tensor(), _tensor(param=4096 + 36)]), dict(tensors=[_tensor(copy=4100)]),
    dict(tensors=[_tensor(param=(1 << 20) + 1020)]), dict(tensors=[_tensor(param=(1 << 22) + 0)], bits=8),
    dict(count=-1), dict(count=(1 << 20) + 1), dict(m=None), dict(v=None), dict(m=(1 << 20) + 4), dict(v=(1 << 20) + 512),
    dict(bits=8, ms=None), dict(bits=8, vs=None), dict(bits=8, vs=(1 << 23) + 2), dict(bits=16), dict(beta1=1.0),
    dict(beta1=-0.1), dict(beta2=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(step=0), dict(step=-3),
    dict(step_device=12), dict(lr=2), dict(grad_scale=6), dict(rule=False)])
def test_refused(L, bad):
    assert _call(L, **bad) == -1 and L.mlt_last_error()


def test_nothing_to_do(L):
    assert _call(L, []) == 0 and _call(L, [_tensor(n=0)], m=None) == 0 and _call(L, [_tensor(grad=0)], m=None) == 0
    assert L.mlt_adamw(None, None, 1, None, None, None, None, None) == -1


def test_blocks(L):
    n = C.c_int64()
    t = array("q", sum((_tensor(n=k) for k in (0, 1, 256, 257, 1 << 40)), []))
    assert L.mlt_adamw_blocks(t.buffer_info()[0], 5, C.byref(n)) == 0 and n.value == 4 + (1 << 32)
    assert L.mlt_adamw_blocks(t.buffer_info()[0], 5, None) == -1 and L.mlt_adamw_blocks(None, 1, C.byref(n)) == -1
