"""mlt_scan_grad against the chain rule on the recurrence in 64 bits, and against
differences of the recurrence; tolerances from the bound that sequence.Approx carries
along, plus half a unit of the output type."""
import numpy as np
import pytest

import sequence as S
from paper_2411_10764_gb300 import mlt
from test_gpu_scan import host, make, near

pytestmark = pytest.mark.gpu

WIDE = ("x", "dt", "B", "C", "z", "conv_state")


def grads_in(t, seed=5, state=True):
    import torch

    rng = np.random.default_rng(seed)
    b, L, d = t["x"].shape
    gy = torch.from_numpy(rng.standard_normal((b, L, d)).astype(np.float32)).cuda().to(t["x"].dtype)
    gs = torch.from_numpy(rng.standard_normal((b, d, t["A"].shape[1])).astype(np.float32)).cuda() if state else None
    return gy, gs


def call(t, gy, gs):
    a = {k: v for k, v in t.items() if k not in ("x", "dt", "B", "C", "A")}
    return mlt.scan_grad(gy, t["x"], t["dt"], t["B"], t["C"], t["A"], g_state=gs, **{
        k: v for k, v in a.items()})


def check(t, gy, gs, got, kind):
    want = S.scan(host(t), gy.float().cpu().numpy(), None if gs is None else gs.cpu().numpy())["grad"]
    assert {k for k, v in got.items() if v is not None and v.numel()} == set(want)
    for k, w in want.items():
        assert got[k].dtype == t[k].dtype
        try:
            near(got[k], w, kind if k in WIDE else "f32")
        except AssertionError as e:
            raise AssertionError(f"{k}: {e}") from None


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("b,L,d,n,g,taps", [
    (1, 1, 1, 1, 1, 4), (3, 1, 70, 16, 1, 4), (2, 2, 64, 16, 2, 2), (5, 3, 33, 13, 1, 3), (2, 9, 128, 32, 1, 0),
    (2, 7, 6, 5, 3, 1), (1, 63, 64, 16, 1, 4), (2, 64, 65, 4, 1, 4), (2, 65, 130, 8, 1, 3), (1, 66, 64, 16, 1, 0),
    (2, 67, 96, 16, 3, 4), (1, 131, 7, 32, 1, 2), (1, 200, 64, 16, 1, 4), (2, 333, 40, 9, 2, 4), (1, 500, 20, 1, 1, 1),
    (1, 129, 260, 32, 4, 4)])
def test_gradients(b, L, d, n, g, taps, kind):
    for ragged in (False, True):
        t = make(b, L, d, n, g, taps, kind, ragged=ragged)
        gy, gs = grads_in(t)
        check(t, gy, gs, call(t, gy, gs), kind)
    t = make(b, L, d, n, g, taps, kind, bare=True)
    gy, gs = grads_in(t, state=False)
    check(t, gy, None, call(t, gy, None), kind)


def test_differences():
    """Along a random direction in each input, the change of sum(y gy) + sum(state gs) by
    differences of the 64-bit recurrence (steps e and e / 2, extrapolated)."""
    t = make(2, 70, 24, 16, 2, 4, "f32", ragged=True)
    gy, gs = grads_in(t)
    got = call(t, gy, gs)
    p, gyn, gsn = host(t), gy.double().cpu().numpy(), gs.double().cpu().numpy()
    bound = S.scan(p, gy.cpu().numpy(), gs.cpu().numpy())["grad"]
    rng = np.random.default_rng(3)

    def loss(q):
        o = S.scan(q)
        return (o["y"].v * gyn).sum() + (o["state"].v * gsn).sum()

    for k, g in got.items():
        way = rng.standard_normal(p[k].shape)
        slope = []
        for e in (1e-4, 5e-5):
            up, down = (dict(p, **{k: p[k].astype(np.float64) + s * e * way}) for s in (1, -1))
            slope.append((loss(up) - loss(down)) / (2 * e))
        want = (4 * slope[1] - slope[0]) / 3
        have = (g.double().cpu().numpy() * way).sum()
        tol = (bound[k].e * np.abs(way)).sum() + 2.0 ** -24 * np.abs(bound[k].v * way).sum() + 1e-7 * (
            1 + abs(want)) + abs(slope[1] - slope[0])
        assert abs(have - want) <= tol, (k, have, want, tol)


def test_the_same_from_call_to_call_and_past_the_end_unused():
    import torch

    for L in (40, 400):
        t = make(3, L, 200, 16, 1, 4, "bf16", ragged=True)
        gy, gs = grads_in(t)
        want = call(t, gy, gs)
        q = {k: v.clone() for k, v in t.items()}
        gy2 = gy.clone()
        for i, n in enumerate(t["lengths"].tolist()):
            gy2[i, n:] = float("nan")
            for k in ("x", "dt", "B", "C", "z"):
                q[k][i, n:] = float("nan")
        streams = [torch.cuda.Stream() for _ in range(3)]
        torch.cuda.synchronize()
        for s in streams:
            with torch.cuda.stream(s):
                got = call(q, gy2, gs)
            torch.cuda.synchronize()
            for k in want:
                assert torch.equal(want[k], got[k]), k
        for i, n in enumerate(t["lengths"].tolist()):
            assert all((want[k][i, n:] == 0).all() for k in ("x", "dt", "z", "B", "C"))


def test_strides():
    import torch

    t = make(2, 70, 66, 16, 1, 4, "f16")
    gy, gs = grads_in(t)
    want = call(t, gy, gs)
    wide = torch.zeros((2, 70, 70 * 4), dtype=torch.float16, device="cuda")
    q = dict(t)
    for j, k in enumerate(("x", "dt", "z")):
        wide[..., 1 + 70 * j:67 + 70 * j] = t[k]
        q[k] = wide[..., 1 + 70 * j:67 + 70 * j]
    wide[..., 213:279] = gy
    got = call(q, wide[..., 213:279], gs)
    for k in want:
        assert torch.equal(want[k], got[k]), k


def test_no_positions():
    import torch

    t = make(2, 4, 64, 16, 1, 4, "bf16")
    t = dict(t, **{k: t[k][:, :0] for k in ("x", "dt", "B", "C", "z")})
    gs = torch.ones_like(t["state"])
    g = call(t, t["x"], gs)
    assert torch.equal(g["state"], gs)
    for k in ("A", "skip", "dt_bias", "conv_w", "conv_b", "conv_state"):
        assert (g[k] == 0).all(), k


def test_refusals():
    import ctypes as C

    import torch

    t = make(1, 5, 64, 16, 1, 4, "f32")
    gy, gs = grads_in(t)
    with pytest.raises(ValueError):
        call(t, gy[:, :3], gs)
    with pytest.raises(TypeError):
        call(t, gy.half(), gs)
    with pytest.raises(ValueError):
        call(t, gy, gs[..., :8])
    mlt._setup()
    a = mlt._scan_args(t["x"], t["dt"], t["B"], t["C"], t["A"], None, None, None, t["conv_w"], None, None, None, None)
    q = mlt.ScanGrads()
    q.gy, q.gy_step, q.gy_batch = gy.data_ptr(), 64, 320
    q.z = torch.empty_like(gy).data_ptr()  # there is no z
    L = mlt.lib()
    n = C.c_size_t()
    assert L.mlt_scan_grad_workspace(C.byref(a), C.byref(n)) == 0
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    assert L.mlt_scan_grad(None, C.byref(a), C.byref(q), ws.data_ptr(), n.value) == -1
    q.z = None
    assert L.mlt_scan_grad(None, C.byref(a), C.byref(q), ws.data_ptr(), n.value - 1) == -1
    assert b"workspace" in L.mlt_last_error()
    assert L.mlt_scan_grad(None, C.byref(a), C.byref(q), ws.data_ptr(), n.value) == 0
    mlt.sync_status()
