"""mlt_scan against the recurrence in 64 bits; tolerances from the bound that
sequence.Approx carries along, plus half a unit of the output type."""
import numpy as np
import pytest

import sequence as S
from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu

UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
NAMES = ("x", "dt", "B", "C", "A", "z", "skip", "dt_bias", "conv_w", "conv_b", "lengths", "state", "conv_state")


def _type(name):
    import torch

    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def make(b, L, d, n, g=1, taps=4, kind="f32", seed=0, ragged=False, bare=False):
    """CUDA tensors by name; `bare`: only what a call cannot do without."""
    import torch

    rng = np.random.default_rng(seed + 7 * L + d)
    r = lambda *s: rng.standard_normal(s)  # noqa: E731
    step = np.exp(rng.uniform(np.log(0.001), np.log(0.3), d))
    p = dict(x=r(b, L, d), dt=r(b, L, d) * 0.5 - (3.0 if bare else 0), B=r(b, L, g, n), C=r(b, L, g, n),
             A=-np.exp(rng.uniform(-1, 3, (d, n))))
    if taps:
        p["conv_w"] = r(d, taps) * 0.5
    if not bare:
        p.update(z=r(b, L, d), skip=r(d), dt_bias=np.log(np.expm1(step)), state=r(b, d, n))
        if taps:
            p["conv_b"] = r(d) * 0.2
        if taps > 1:
            p["conv_state"] = r(b, taps - 1, d)
    wide = ("x", "dt", "B", "C", "z", "conv_state")
    t = {k: torch.from_numpy(v.astype(np.float32)).cuda().to(_type(kind) if k in wide else torch.float32)
         for k, v in p.items()}
    if ragged:
        lens = rng.integers(0, L + 1, b)
        lens[0] = L
        if b > 1:
            lens[1] = 0
        t["lengths"] = torch.from_numpy(lens.astype(np.int32)).cuda()
    return t


def host(t):
    return {k: (v.float() if v.is_floating_point() else v).cpu().numpy() for k, v in t.items()}


def call(t, **more):
    a = {k: v for k, v in t.items() if k not in ("x", "dt", "B", "C", "A")}
    return mlt.scan(t["x"], t["dt"], t["B"], t["C"], t["A"], **a, **more)


def near(got, want, kind):
    """Within the bound, half a unit of the type, and (binary16) half a subnormal."""
    assert tuple(got.shape) == want.v.shape
    tol = want.e + UNIT[kind] * np.abs(want.v) + (2.0 ** -25 if kind == "f16" else 0)
    off = np.abs(got.double().cpu().numpy() - want.v)
    assert (off <= tol).all(), (off - tol).max()


def check(t, got, kind):
    ref = S.scan(host(t))
    y, state, conv = got
    near(y, ref["y"], kind)
    near(state, ref["state"], "f32")
    if "conv_state" in ref:
        assert np.array_equal(conv.float().cpu().numpy(), ref["conv_state"].v.astype(np.float32))
    else:
        assert conv is None


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("b,L,d,n,g,taps", [
    (1, 1, 1, 1, 1, 4), (3, 1, 70, 16, 1, 4), (2, 1, 64, 16, 2, 2), (5, 1, 33, 13, 1, 3), (2, 1, 128, 32, 1, 0),
    (2, 1, 6, 5, 3, 1), (1, 2, 64, 16, 1, 4), (2, 3, 65, 4, 1, 4), (2, 15, 130, 8, 1, 3), (1, 16, 64, 16, 1, 0),
    (2, 17, 96, 16, 3, 4), (1, 63, 7, 32, 1, 2), (1, 200, 64, 16, 1, 4), (2, 333, 40, 9, 2, 4), (1, 1025, 20, 1, 1, 1),
    (1, 700, 260, 16, 4, 4)])
def test_scan(b, L, d, n, g, taps, kind):
    for ragged in (False, True):
        t = make(b, L, d, n, g, taps, kind, ragged=ragged)
        check(t, call(t), kind)
    t = make(b, L, d, n, g, taps, kind, bare=True)
    check(t, call(t), kind)


def test_one_chunk_and_many_agree_with_the_recurrence():
    for b, L, d in ((40, 90, 512), (1, 3000, 64)):
        t = make(b, L, d, 16, 1, 4, "f32", ragged=b > 1)
        check(t, call(t), "f32")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_prompt_then_tokens_equal_the_whole(kind):
    """A prompt in two parts and single tokens in place continue where the whole sequence is."""
    import torch

    b, L, d, n = 3, 41, 100, 16
    t = make(b, L, d, n, 2, 4, kind)
    seq = ("x", "dt", "B", "C", "z")
    part = lambda i, j, **more: dict(t, **{k: t[k][:, i:j] for k in seq}, **more)  # noqa: E731
    y1, s, c = call(part(0, 25))
    y2, s, c = call(part(25, 38, state=s, conv_state=c))
    ys = [y1, y2]
    for i in range(38, L):
        y, s2, c2 = call(part(i, i + 1, state=s, conv_state=c), state_out=s, conv_state_out=c)
        assert s2 is s and c2 is c
        ys.append(y)
    check(t, (torch.cat(ys, 1), s, c), kind)


def test_what_lies_past_a_sequences_end_is_not_used():
    import torch

    for L in (1, 50, 900):
        t = make(3, L, 64, 16, 1, 4, "bf16", ragged=True)
        want = call(t)
        q = {k: v.clone() for k, v in t.items()}
        for i, n in enumerate(t["lengths"].tolist()):
            for k in ("x", "dt", "B", "C", "z"):
                q[k][i, n:] = float("nan")
        got = call(q)
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        assert (got[0][1] == 0).all()
        q["lengths"] = q["lengths"] + torch.tensor([5, -7, 0], dtype=torch.int32, device="cuda")  # clamped
        assert torch.equal(call(q)[0][:2], want[0][:2])


def test_strides_alignment_and_output_in_a_wider_buffer():
    import torch

    b, L, d, n = 2, 37, 66, 16
    t = make(b, L, d, n, 1, 4, "f16")
    want = call(t)
    for off in (0, 1, 4):
        wide = torch.zeros((b, L, 3 * d + 8), dtype=torch.float16, device="cuda")
        q = dict(t)
        for j, k in enumerate(("x", "dt", "z")):
            wide[..., off + j * d:off + (j + 1) * d] = t[k]
            q[k] = wide[..., off + j * d:off + (j + 1) * d]
        bc = torch.cat([t["B"], t["C"]], -1)
        q["B"], q["C"] = bc[..., :n], bc[..., n:]
        buf = torch.full((b, L, d + 10), 3.0, dtype=torch.float16, device="cuda")
        got = call(q, out=buf[..., off:off + d])
        for a, e in zip(want, got):
            assert torch.equal(a, e)
        assert (buf[..., :off] == 3).all() and (buf[..., off + d:] == 3).all()


def test_transposed_sequences_and_no_groups_dimension():
    import torch

    t = make(3, 20, 64, 16, 1, 4, "f32")
    want = call(t)
    q = dict(t)
    for k in ("x", "dt", "z", "B", "C"):
        q[k] = t[k].transpose(0, 1).contiguous().transpose(0, 1)
    q["B"], q["C"] = q["B"][:, :, 0], q["C"][:, :, 0]
    for a, e in zip(want, call(q)):
        assert torch.equal(a, e)


def test_large_steps_forget_and_tiny_steps_keep():
    import torch

    t = make(1, 40, 64, 16, 1, 0, "f32")
    t["dt"] = torch.full_like(t["dt"], 60.0)
    check(t, call(t), "f32")
    t["dt"] = torch.full_like(t["dt"], -60.0)
    t["dt_bias"] = torch.zeros_like(t["dt_bias"])
    check(t, call(t), "f32")


def test_no_positions_and_no_sequences():
    import torch

    t = make(2, 4, 64, 16, 1, 4, "bf16")
    q = dict(t, **{k: t[k][:, :0] for k in ("x", "dt", "B", "C", "z")})
    y, s, c = call(q)
    assert y.shape == (2, 0, 64) and torch.equal(s, t["state"]) and torch.equal(c, t["conv_state"])
    del q["state"], q["conv_state"]
    y, s, c = call(q)
    assert (s == 0).all() and (c == 0).all()
    q = {k: v[:0] if k in ("x", "dt", "B", "C", "z", "state", "conv_state") else v for k, v in t.items()}
    assert call(q)[0].shape == (0, 4, 64)


def test_streams_and_graph():
    import torch

    t = make(1, 2000, 128, 16, 1, 4, "bf16")
    want = call(t)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(5):
        got = []
        for s in streams:
            with torch.cuda.stream(s):
                got.append(call(t))
        torch.cuda.synchronize()
        for g in got:
            assert all(torch.equal(a, b) for a, b in zip(want, g))
    t = make(4, 1, 128, 16, 1, 4, "bf16")
    y = torch.empty_like(t["x"])
    s0, c0 = t["state"].clone(), t["conv_state"].clone()
    two = [call(dict(t, state=s0, conv_state=c0), state_out=s0, conv_state_out=c0)[0] for _ in range(2)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            call(t, out=y, state_out=t["state"], conv_state_out=t["conv_state"])
    for k in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, two[k])
    assert torch.equal(t["state"], s0) and torch.equal(t["conv_state"], c0)


def test_binding_refuses():
    import torch

    t = make(2, 5, 64, 16, 2, 4, "f32")
    for k, bad, err in (("dt", t["dt"].half(), TypeError), ("A", t["A"].half(), TypeError),
                        ("z", t["z"][:, :3], ValueError), ("B", t["B"][..., :8], ValueError),
                        ("state", t["state"][:, :10], ValueError), ("conv_w", t["conv_w"].t(), ValueError),
                        ("x", t["x"].cpu(), TypeError), ("lengths", torch.ones(2, device="cuda"), TypeError),
                        ("dt", t["dt"].transpose(1, 2).contiguous().transpose(1, 2), ValueError)):
        with pytest.raises(err):
            call(dict(t, **{k: bad}))
    big = make(1, 2, 4, 33, 1, 4, "f32")
    with pytest.raises(mlt.MltError) as e:
        call(big)
    assert e.value.code == -1
    five = make(1, 2, 4, 4, 1, 5, "f32")
    with pytest.raises(mlt.MltError):
        call(five)
