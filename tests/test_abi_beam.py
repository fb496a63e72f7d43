"""Beam search's C calls refuse bad arguments on the host, before any CUDA call."""
import ctypes as C

import pytest

from paper_2411_10764_gb300 import mlt


@pytest.fixture(scope="module")
def L():
    return mlt.lib()


def _args(**kw):
    a = mlt.BeamArgs(0, 2, 4, 50000, 8, 0, -1, 4096, 200000, 50000, 256, None, 512, 1024, 2048, 3000)
    for k, v in kw.items():
        setattr(a, k, v)
    return C.byref(a)


SIZES = [dict(dtype=3), dict(batch=-1), dict(batch=65536), dict(beams=0), dict(beams=1025), dict(n=0), dict(n=(1 << 22) + 1),
         dict(m=0), dict(m=1025), dict(beams=1024, m=9), dict(beams=9, m=1000)]


def test_step(L):
    size = C.c_size_t()
    assert L.mlt_beam_step_workspace(_args(), C.byref(size)) == 0 and size.value > 0
    n = size.value
    step = lambda ws=256, b=n, **kw: L.mlt_beam_step(None, _args(**kw), ws, b)  # noqa: E731
    for bad in SIZES:
        assert step(**bad) == -1 and L.mlt_beam_step_workspace(_args(**bad), C.byref(size)) == -1, bad
    for bad in (dict(scores=None), dict(logp=None), dict(out_parent=None), dict(out_token=None), dict(out_logp=None),
                dict(out_done=None), dict(batch_stride=-1), dict(beam_stride=-1), dict(eos=50000), dict(done=64),
                dict(scores=4098), dict(logp=258), dict(out_parent=516), dict(out_token=1028), dict(out_logp=2050),
                dict(ws=None), dict(b=n - 1), dict(ws=264)):
        assert step(**bad) == -1 and L.mlt_last_error(), bad
    assert step(batch=0, ws=None) == 0
    assert L.mlt_beam_step(None, None, None, 0) == -1 and L.mlt_beam_step_workspace(None, C.byref(size)) == -1
    assert L.mlt_beam_step_workspace(_args(), None) == -1
    assert L.mlt_beam_step_workspace(_args(n=8), C.byref(size)) == 0 and size.value == 0  # few scores: none needed


def test_reorder(L):
    def reorder(*states, parent=1 << 30, batch=2, beams=4, count=None, tensors=True):
        t = (mlt.BeamState * max(1, len(states)))(*[mlt.BeamState(*s) for s in states])
        return L.mlt_beam_reorder(None, parent, batch, beams, t if tensors else None, len(states) if count is None else count)

    one = (4096, 64, 64)
    for bad in (dict(batch=-1), dict(batch=65536), dict(beams=0), dict(beams=1025), dict(count=-1), dict(count=65),
                dict(tensors=False), dict(parent=None), dict(parent=(1 << 30) + 4), dict(parent=4096), dict(parent=4096 + 504)):
        assert reorder(one, **bad) == -1 and L.mlt_last_error(), bad
    for bad in ((None, 64, 64), (4096, -1, 64), (4096, 64, 63), (4096, 64, -64), (4096, (1 << 40) + 1, 1 << 41), (4096, 64, 0)):
        assert reorder(bad) == -1, bad
    assert reorder(one, (4096 + 448, 64, 64)) == -1  # the other's last row
    assert reorder() == 0 and reorder(one, batch=0) == 0 and reorder((4096, 0, 0), parent=None) == 0


def test_states_side_by_side(L):
    """Columns of one buffer that share a byte, or lie at different strides, are refused; so is what ends past 2^60 bytes."""
    def reorder(*states, parent=1 << 30, batch=2, beams=4):
        t = (mlt.BeamState * len(states))(*[mlt.BeamState(*s) for s in states])
        return L.mlt_beam_reorder(None, parent, batch, beams, t, len(states))

    one = (4096, 16, 64)
    for other in ((4096 + 15, 8, 64), (4096 + 48, 17, 64), (4096 + 64, 16, 64), (4096 - 8, 9, 64), (4096 - 64 + 8, 8, 64),
                  (4096 + 16, 16, 128), (4096, 16, 64), (4096 + 7 * 64 + 15, 1, 64), (4096 - 20, 30, 64)):
        assert reorder(one, other) == -1 and b"overlap" in L.mlt_last_error(), other
        assert reorder(other, one) == -1 and b"overlap" in L.mlt_last_error(), other
    assert reorder((4096, 1, 1 << 40), batch=65535, beams=1024) == -1 and b"2^60" in L.mlt_last_error()
