"""Layer norm's C calls refuse bad arguments on the host, before any CUDA call."""
import ctypes as C

import pytest

from paper_2411_10764_gb300 import mlt


@pytest.fixture(scope="module")
def L():
    return mlt.lib()


def _args(**kw):
    a = mlt.NormArgs(0, 0, 0, 8, 3, 256, None, 256, 256, 8, 0, 256, None, 8, 8, 256, 1e-5)
    for k, v in kw.items():
        setattr(a, k, v)
    return C.byref(a)


BOTH = [dict(dtype=3), dict(y_dtype=-1), dict(w_dtype=7), dict(dtype=1, y_dtype=0), dict(dtype=1, y_dtype=2),
        dict(rows=-1), dict(rows=1 << 31), dict(dim=0), dict(dim=(1 << 20) + 1), dict(x=None), dict(x=258),
        dict(weight=258), dict(bias=257), dict(stats=260), dict(x_stride=-8), dict(residual_stride=-1)]


@pytest.mark.parametrize("bad", BOTH + [dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(y=None),
                                        dict(y=258), dict(y_stride=7), dict(total=512, total_stride=7), dict(total=256),
                                        dict(total=514), dict(residual=258)])
def test_forward(L, bad):
    assert L.mlt_layer_norm(None, _args(**bad)) == -1 and L.mlt_last_error()


def test_gradient(L):
    size = C.c_size_t()
    assert L.mlt_layer_norm_grad_workspace(3, 8, C.byref(size)) == 0 and size.value > 0
    n = size.value

    def grad(args=None, ws=256, bytes_=n, **kw):
        g = mlt.NormGrads(256, None, 8, 8, 256, 8, 256, 256)
        for k, v in kw.items():
            setattr(g, k, v)
        return L.mlt_layer_norm_grad(None, args or _args(), C.byref(g), ws, bytes_)

    for bad in BOTH + [dict(residual=256), dict(stats=None)]:
        assert grad(_args(**bad)) == -1, bad
    for bad in (dict(gy=None), dict(gy=258), dict(gy_stride=-1), dict(g_total=258), dict(g_total_stride=-8),
                dict(gx_stride=7), dict(gx=258), dict(gweight=258), dict(gbias=257), dict(ws=None), dict(bytes_=n - 1),
                dict(ws=264)):
        assert grad(**bad) == -1, bad
    assert grad(gx=None, gweight=None, gbias=None, ws=None) == 0  # nothing wanted
    assert L.mlt_layer_norm(None, None) == -1 and L.mlt_layer_norm_grad(None, None, None, None, 0) == -1
    assert L.mlt_layer_norm_grad(None, _args(), None, None, 0) == -1
    assert L.mlt_layer_norm(None, _args(rows=0, x=None, y=None)) == 0
    assert L.mlt_layer_norm_grad_workspace(3, 8, None) == -1
    for rows, dim in ((-1, 8), (3, 0), (3, (1 << 20) + 1)):
        assert L.mlt_layer_norm_grad_workspace(rows, dim, C.byref(size)) == -1


def test_outputs_over_inputs(L):
    """Where an output begins at an input's address it has to be that input, or rows would be written before others
    have read theirs."""
    for bad in (dict(x_stride=0), dict(y_stride=16), dict(y_dtype=1), dict(rows=1, y_dtype=2),
                dict(y=512, residual=512), dict(y=512, total=256, total_stride=16), dict(y=512, total=1024, residual=1024),
                dict(y=512, residual=512, residual_stride=8, y_dtype=1)):
        assert L.mlt_layer_norm(None, _args(**bad)) == -1 and b"over an input" in L.mlt_last_error(), bad
    for bad, args in ((dict(gy=512, g_total=256, g_total_stride=0), {}), (dict(gy_stride=0), {}), (dict(gx_stride=16), {}),
                      (dict(), dict(y_dtype=1)), (dict(gy=512), dict(x_stride=0))):
        g = mlt.NormGrads(256, None, 8, 8, 256, 8, 256, 256)
        for k, v in bad.items():
            setattr(g, k, v)
        assert L.mlt_layer_norm_grad(None, _args(**args), C.byref(g), None, 0) == -1
        assert b"over an input" in L.mlt_last_error(), (bad, args)
