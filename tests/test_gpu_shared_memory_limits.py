"""Calls whose kernels take more shared memory than a kernel has unasked, from two host threads: what one call asks for
is not taken back by another of less."""
import ctypes as C
import threading

import pytest

from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu


class _Calls:
    """Pairs of C calls of one kernel, both with more than 40 KB: f(stream) and the tensor that receives its result."""

    def __init__(self):
        import torch

        self.L, self.torch = mlt.lib(), torch
        self.g = torch.Generator("cuda").manual_seed(1)
        self.kept = []

    def rnd(self, *shape, dtype=None):
        t = self.torch.randn(*shape, generator=self.g, device="cuda").to(dtype or self.torch.float32)
        self.kept.append(t)
        return t

    def args(self, x, dim, w, b, y, stats):
        code = mlt.MLT_F32 if x.dtype == self.torch.float32 else mlt.MLT_BF16
        return mlt.NormArgs(code, code, mlt.MLT_F32, dim, len(x), x.data_ptr(), None, w.data_ptr(), b.data_ptr(), dim, 0,
                            y.data_ptr(), None, dim, 0, stats.data_ptr(), 1e-5)

    def norm(self, dim, dtype):
        x, y, w, b, stats = self.rnd(2, dim, dtype=dtype), self.rnd(2, dim, dtype=dtype), self.rnd(dim), self.rnd(dim), self.rnd(2, 2)
        a = self.args(x, dim, w, b, y, stats)
        return lambda s: self.L.mlt_layer_norm(s, C.byref(a)), y

    def grad(self, dim):
        x, gy, gx, w, gw = self.rnd(2, dim), self.rnd(2, dim), self.rnd(2, dim), self.rnd(dim), self.rnd(dim)
        a = self.args(x, dim, w, w, gx, mlt.layer_norm(x)[2])
        a.stats = self.rnd(2, 2).copy_(mlt.layer_norm(x)[2]).data_ptr()
        q = mlt.NormGrads(gy.data_ptr(), None, dim, 0, gx.data_ptr(), dim, gw.data_ptr(), None)
        n = C.c_size_t()
        assert self.L.mlt_layer_norm_grad_workspace(2, dim, C.byref(n)) == 0
        ws = self.rnd(n.value // 4 + 1)
        return lambda s: self.L.mlt_layer_norm_grad(s, C.byref(a), C.byref(q), ws.data_ptr(), n.value), gx

    def step(self, beams, n, dtype, k=8):
        m, t = 500 if beams > 100 else k, self.torch
        x, lp = self.rnd(1, beams, n, dtype=dtype), self.rnd(1, beams)
        parent, token, out, done = (t.zeros(1, m, dtype=d, device="cuda") for d in (t.int64, t.int64, t.float32, t.bool))
        self.kept += [parent, token, out, done]
        code = mlt.MLT_F32 if dtype == t.float32 else mlt.MLT_BF16
        a = mlt.BeamArgs(code, 1, beams, n, m, 0, -1, x.data_ptr(), beams * n, n, lp.data_ptr(), None, parent.data_ptr(),
                         token.data_ptr(), out.data_ptr(), done.data_ptr())
        size = C.c_size_t()
        assert self.L.mlt_beam_step_workspace(C.byref(a), C.byref(size)) == 0
        ws = self.rnd(size.value // 4 + 1)
        return lambda s: self.L.mlt_beam_step(s, C.byref(a), ws.data_ptr(), size.value), token

    def reorder(self, beams):
        t = self.torch.arange(beams * 997, device="cuda").view(beams, 997)
        parent = self.torch.zeros(beams, dtype=self.torch.int64, device="cuda")  # the same however often
        states = (mlt.BeamState * 1)(mlt.BeamState(t.data_ptr(), 997 * 8, 997 * 8))
        self.kept += [t, parent]
        return lambda s: self.L.mlt_beam_reorder(s, parent.data_ptr(), 1, beams, states, 1), t

    def pairs(self):
        bf16, f32 = self.torch.bfloat16, self.torch.float32
        return {"norm": (self.norm(8192, bf16), self.norm(6200, bf16)),
                "long norm": (self.norm(50001, f32), self.norm(12301, f32)),
                "grad": (self.grad(4096), self.grad(2048)),
                "step": (self.step(1000, 8, bf16), self.step(700, 5, bf16)),
                "step from lists": (self.step(7, 9000, bf16, 1000), self.step(5, 9000, bf16, 700)),
                "reorder": (self.reorder(1000), self.reorder(400))}


def test_captured_together():
    """A large and a small call in one graph, and the kernel called with less before it is replayed."""
    import torch

    calls = _Calls()
    for name, pair in calls.pairs().items():
        torch.cuda.synchronize()
        now = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
        assert all(call(now()) == 0 for call, _ in pair), name
        want = [t.clone() for _, t in pair]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            assert all(call(now()) == 0 for call, _ in pair), name
        if name != "reorder":
            for _, t in pair:
                t.zero_()
        assert pair[1][0](now()) == 0
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for (_, t), w in zip(pair, want)), name


def test_from_two_threads():
    """The host's parts of two calls overlap some thousand times."""
    import torch

    calls = _Calls()
    for name, pair in calls.pairs().items():
        streams = [torch.cuda.Stream() for _ in pair]
        torch.cuda.synchronize()
        for (call, _), s in zip(pair, streams):
            assert call(s.cuda_stream) == 0
        torch.cuda.synchronize()
        want = [t.clone() for _, t in pair]
        refused = [0, 0]

        def loop(i, call, stream):
            for _ in range(20):
                refused[i] += sum(call(stream.cuda_stream) != 0 for _ in range(500))
                stream.synchronize()

        threads = [threading.Thread(target=loop, args=(i, call, s)) for i, ((call, _), s) in enumerate(zip(pair, streams))]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert refused == [0, 0], name
        assert all(torch.equal(t, w) for (_, t), w in zip(pair, want)), name
