"""mlt_beam_step and mlt_beam_reorder against plain implementations.

A total in 64 bits is off by the normaliser alone: each of its terms exp(s - top) by 2^-22 of
itself (the approximate power) and by 2^-23 |s - top| (its argument), so ln of the sum by
the mean of these, weighted by the terms; one more rounding where the total is written.  Where neighbours
in the order are nearer than that, either may come first; equal totals have a rule and
are tested with totals that are equal exactly."""
import math

import numpy as np
import pytest

from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
FMAX = 3.4028234663852886e38


def _type(name):
    import torch

    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _best(scores, logp, done, eos, m, normalised):
    """One item: lists of (total, tolerance, beam, score, token), best first, m + 1 of them."""
    got = []
    for w in range(len(logp)):
        lp = float(logp[w])
        if not lp > -math.inf:
            continue
        if done is not None and done[w]:
            got.append((lp, 0.0, w, 0.0, eos))
            continue
        x = scores[w].astype(np.float64)
        ok = np.flatnonzero(x > -np.inf)
        if ok.size == 0:
            continue
        s = np.clip(x[ok], -FMAX, FMAX)
        top = s.max()
        e = np.exp(s - top)
        z, tol = 0.0, 0.0
        if not normalised:
            z = top + math.log(e.sum())
            tol = 2.0 ** -22 + 2.0 ** -23 * (e * np.where(e > 0, top - s, 0)).sum() / e.sum()
        order = np.lexsort((ok, -s))[:m + 1]
        got += [(lp + (s[i] - z), tol, w, s[i], int(ok[i])) for i in order]
    got.sort(key=lambda c: (-c[0], c[2], -c[3], c[4]))
    return got[:m + 1]


def _check(scores, logp, m, got, done=None, eos=-1, normalised=False):
    parent, token, out, ended = (t.cpu().numpy() for t in got)
    x, lp = scores.float().cpu().numpy(), logp.cpu().numpy()
    d = None if done is None else done.cpu().numpy()
    assert parent.shape == token.shape == out.shape == ended.shape == (x.shape[0], m)
    for b in range(x.shape[0]):
        want = _best(x[b], lp[b], None if d is None else d[b], eos, m, normalised)
        have = min(m, len(want))
        assert (parent[b, have:] == -1).all() and (token[b, have:] == -1).all()
        assert (out[b, have:] == -np.inf).all() and not ended[b, have:].any()
        for j in range(have):
            total, tol, w, s, t = want[j]
            tol = 2 * max(c[1] for c in want[max(0, j - 1):j + 2]) + 2.0 ** -50 * abs(total)
            # rounding to fp32 takes what lies below the lowest float to -infinity
            assert abs(out[b, j] - total) <= tol + U * abs(total) if total >= -FMAX else out[b, j] == -np.inf, (b, j)
            near = [c for c in want if abs(c[0] - total) <= tol]
            assert (parent[b, j], token[b, j]) in [(c[2], c[4]) for c in near], (b, j)
            over = d is not None and bool(d[b, parent[b, j]])
            assert ended[b, j] == (over or token[b, j] == eos)
        pairs = set(zip(parent[b, :have].tolist(), token[b, :have].tolist()))
        assert len(pairs) == have


def _make(rng, batch, beams, n, kind="f32", masked=0.0, done=None, start=False):
    import torch

    x = (rng.standard_normal((batch, beams, n)) * 2.5).astype(np.float32)
    if masked:
        x[rng.random(x.shape) < masked] = -np.inf
    scores = torch.from_numpy(x).cuda().to(_type(kind))
    lp = -np.abs(rng.standard_normal((batch, beams))) * 3 - 5
    if start:
        lp[:, 1:] = -np.inf
    logp = torch.from_numpy(lp.astype(np.float32)).cuda()
    d = None if done is None else torch.from_numpy(rng.random((batch, beams)) < done).cuda()
    return scores, logp, d


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("batch,beams,n,m", [
    (1, 1, 1, 1), (3, 4, 1, 4), (2, 3, 5, 7), (1, 256, 8, 256), (5, 16, 37, 16), (2, 1024, 8, 1024), (1, 1000, 3, 777),
    (4, 1, 8192, 10), (3, 2, 4097, 4), (2, 4, 50021, 8), (1, 1, 262147, 1), (1, 1, 20000, 1024), (2, 8, 9000, 1024),
    (1, 64, 5000, 128), (40, 8, 3001, 8), (7, 5, 12345, 33), (1, 900, 100, 9), (300, 3, 17, 3)])
def test_step(batch, beams, n, m, kind):
    rng = np.random.default_rng(n + beams + m)
    for masked, done, start in ((0.0, None, False), (0.5, 0.3, False), (0.9, None, True)):
        scores, logp, d = _make(rng, batch, beams, n, kind, masked, done, start)
        eos = -1 if d is None else min(2, n - 1)
        _check(scores, logp, m, mlt.beam_step(scores, logp, m, done=d, eos=eos), d, eos)
    got = mlt.beam_step(scores, logp, m, normalised=True)
    _check(scores, logp, m, got, normalised=True)


@pytest.mark.parametrize("beams", [950, 960, 970, 1000, 1024])
def test_lists_around_48_kb(beams):
    """2,048 candidates of 16 bytes and the beams' numbers in shared memory."""
    rng = np.random.default_rng(beams)
    for n in (2, 3):
        scores, logp, d = _make(rng, 2, beams, n, done=0.1)
        _check(scores, logp, 300, mlt.beam_step(scores, logp, 300, done=d, eos=0), d, 0)


def test_one_item_and_uint8():
    import torch

    rng = np.random.default_rng(0)
    scores, logp, d = _make(rng, 1, 6, 100, done=0.4)
    got = mlt.beam_step(scores[0], logp[0], 5, done=d[0].to(torch.uint8), eos=7)
    assert all(t.shape == (5,) for t in got)
    want = mlt.beam_step(scores, logp, 5, done=d, eos=7)
    assert all(torch.equal(a, b[0]) for a, b in zip(got, want))


@pytest.mark.parametrize("beams,n", [(4, 6), (4, 60), (4, 30011), (2, 100000)])
def test_ties(beams, n):
    """Equal totals: the lower beam, then the lower token; a longer row's equal scores overflow every
    list.  All beams alike, so their normalisers are equal to the bit."""
    import torch

    for fill, some in ((0.0, 0), (1.0, 3), (-2.0, 900)):
        x = np.full((beams, n), fill, np.float32)
        rng = np.random.default_rng(some)
        at = rng.choice(n, min(some, n // 2), replace=False)
        x[:, at] = fill + 1
        scores = torch.from_numpy(x)[None].cuda()
        logp = torch.full((1, beams), -3.0, device="cuda")
        for m in (1, 5, 64, 1000):
            parent, token, out, _ = (t[0].cpu().numpy() for t in mlt.beam_step(scores, logp, m))
            ranked = sorted(((w, t) for w in range(beams) for t in range(n) if n <= 60 or x[w, t] > fill or t < 1200),
                            key=lambda c: (-x[c], c))[:m]
            assert list(zip(parent.tolist(), token.tolist()))[:len(ranked)] == ranked, (fill, m)
            z = fill + math.log((x[0] > fill).sum() * math.e + (x[0] == fill).sum())
            for j, c in enumerate(ranked):
                assert abs(out[j] - (-3.0 + x[c] - z)) <= 2.0 ** -21 + U * abs(out[j])


@pytest.mark.parametrize("n", [3, 9000])
def test_rows_of_one_score(n):
    """A beam's only continuation has the beam's own log-probability exactly, whatever its score: equal ones tie."""
    import torch

    rng = np.random.default_rng(n)
    x = torch.full((4, 8, n), -math.inf, device="cuda")
    at = rng.integers(0, n, (4, 8))
    for b in range(4):
        for w in range(8):
            x[b, w, at[b, w]] = float(rng.standard_normal() * 10.0 ** rng.integers(-3, 4))
    logp = torch.full((4, 8), -11.3, device="cuda")
    parent, token, out, _ = mlt.beam_step(x, logp, 8)
    assert (out == logp[0, 0]).all()
    assert torch.equal(parent, torch.arange(8, device="cuda").expand(4, 8))
    assert torch.equal(token.cpu(), torch.from_numpy(at))


def test_scores_that_one_total_cannot_tell_apart():
    """Within a beam the scores decide even where totals are equal in 64 bits."""
    import torch

    x = torch.full((1, 2, 20000), -50.0, device="cuda")
    x[0, 0, 100], x[0, 0, 50], x[0, 0, 7] = 3e-30, 1e-30, 2e-30
    x[0, 1, 9], x[0, 1, 8] = 1e-38, 1e-38
    logp = torch.tensor([[0.0, -20.0]], device="cuda")
    for y in (x, x[:, :, :1000].contiguous()):
        parent, token, _, _ = mlt.beam_step(y, logp, 5)
        assert parent[0].tolist() == [0, 0, 0, 1, 1] and token[0].tolist() == [100, 7, 50, 8, 9]


@pytest.mark.parametrize("n", [12, 5000, 40000])
def test_special_scores(n):
    """NaN and -infinity are no continuations, +infinity counts as the largest float, the lowest float is
    one; beams without any, beams with logp NaN or -infinity."""
    import torch

    rng = np.random.default_rng(n)
    scores, logp, _ = _make(rng, 1, 8, n)
    scores[0, 0] = math.nan
    scores[0, 1] = -math.inf
    scores[0, 2, ::2] = math.nan
    scores[0, 3] = -FMAX
    scores[0, 4, 3] = math.inf
    scores[0, 5, 1], scores[0, 5, 2] = -FMAX, FMAX
    logp[0, 6], logp[0, 7] = math.nan, -math.inf
    got = mlt.beam_step(scores, logp, 100)
    _check(scores, logp, 100, got)
    assert not torch.isin(got[0], torch.tensor([0, 1, 6, 7], device="cuda")).any()
    none = mlt.beam_step(scores[:, :2].contiguous(), logp[:, :2].contiguous(), 3)
    assert (none[0] == -1).all() and (none[1] == -1).all() and (none[2] == -math.inf).all() and not none[3].any()
    logp[0] = -math.inf
    assert (mlt.beam_step(scores, logp, 3)[0] == -1).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n", [30, 9001])
def test_strides_and_alignment(n, kind):
    rng = np.random.default_rng(n)
    wide, logp, _ = _make(rng, 3, 6, n + 40, kind)
    for off in range(0, 9):
        x = wide[:, ::2, off:off + n]
        lp = logp[:, ::2].contiguous()
        _check(x, lp, 7, mlt.beam_step(x, lp, 7))
    x = wide[:1, :1, :n].expand(3, 6, n)  # one row for all
    _check(x, logp, 7, mlt.beam_step(x, logp, 7))


def test_normaliser_of_long_rows():
    """262,144 terms of which none dominates: the sum's error does not grow with their number."""
    import torch

    for n, scale in ((262144, 0.0), (262143, 0.1), (65536, 1.0)):
        rng = np.random.default_rng(n)
        x = torch.from_numpy((rng.standard_normal((1, 2, n)) * scale).astype(np.float32)).cuda()
        logp = torch.zeros(1, 2, device="cuda")
        out = mlt.beam_step(x, logp, 1)[2]
        s = x.double()
        want = (s.amax(2) - torch.logsumexp(s, 2)).max().item()
        assert abs(out.item() - want) <= 2.0 ** -22 * 1.5 + U * abs(want)


def test_captured_on_another_stream_and_side_by_side():
    import torch

    rng = np.random.default_rng(8)
    cases = [_make(rng, 3, 8, 20001, "bf16", 0.1, 0.2), _make(rng, 3, 8, 20001, "bf16", 0.3, 0.2)]
    want = [[t.clone() for t in mlt.beam_step(s, lp, 8, done=d, eos=3)] for s, lp, d in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [mlt.beam_step(s, lp, 8, done=d, eos=3, stream=q) for (s, lp, d), q in zip(cases, streams)]
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    graphs, outs = [], []
    for s, lp, d in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(mlt.beam_step(s, lp, 8, done=d, eos=3))
        graphs.append(g)
    for _ in range(2):
        for g, q in zip(graphs, streams):
            with torch.cuda.stream(q):
                g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, outs):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


# --- states ----------------------------------------------------------------------------------

def _moved(t, parent):
    import torch

    b, w = parent.shape
    place = torch.arange(b * w, device="cuda").view(b, w)
    source = torch.where(parent < 0, place, place[:, :1] + parent).view(-1)
    flat = t.reshape(b * w, -1)
    return flat[source].reshape(t.shape)


@pytest.mark.parametrize("batch,beams", [(1, 1), (1, 2), (3, 4), (64, 8), (1, 256), (2, 1000), (700, 3)])
def test_reorder(batch, beams):
    import torch

    g = torch.Generator("cuda").manual_seed(beams)
    rows = batch * beams
    tensors = [torch.randn(rows, 37, 5, device="cuda", generator=g), torch.randn(rows, 3, 40, device="cuda", generator=g).bfloat16(),
               torch.randint(0, 99, (rows, 11), device="cuda", generator=g),
               torch.randint(0, 255, (batch, beams, 13), device="cuda", generator=g, dtype=torch.uint8),
               torch.rand(rows, device="cuda", generator=g) < 0.5, torch.randn(rows, 7, device="cuda", generator=g).half(),
               torch.randn(rows, 4100, device="cuda", generator=g), torch.empty(rows, 0, device="cuda")]
    for kind in ("any", "same", "swap", "gaps"):
        parent = torch.randint(0, beams, (batch, beams), device="cuda", generator=g)
        if kind == "same":
            parent = torch.arange(beams, device="cuda").repeat(batch, 1)
        elif kind == "swap":
            parent = torch.arange(beams - 1, -1, -1, device="cuda").repeat(batch, 1)
        elif kind == "gaps":
            parent[torch.rand(batch, beams, device="cuda", generator=g) < 0.5] = -1
        want = [_moved(t, parent) for t in tensors]
        mlt.beam_reorder(parent, *tensors)
        assert all(torch.equal(a, b) for a, b in zip(tensors, want)), kind
    mlt.sync_status()


@pytest.mark.parametrize("beams", [9, 11, 12, 13, 100, 300, 350, 384, 400])
def test_reorder_around_48_kb(beams):
    """Slices of all beams in shared memory beside their parents."""
    import torch

    g = torch.Generator("cuda").manual_seed(beams)
    t = torch.randint(0, 1 << 40, (beams, 3001), device="cuda", generator=g)
    parent = torch.randint(0, beams, (1, beams), device="cuda", generator=g)
    want = _moved(t, parent)
    mlt.beam_reorder(parent, t)
    assert torch.equal(t, want)


def test_reorder_strides_and_bad_parents():
    import torch

    buf = torch.arange(24 * 50, device="cuda").view(24, 50)
    for a, b in ((0, 50), (3, 17), (8, 40)):
        parent = torch.randint(0, 6, (4, 6), device="cuda")
        want = buf.clone()
        want[:, a:b] = _moved(buf[:, a:b], parent)
        mlt.beam_reorder(parent, buf[:, a:b])
        assert torch.equal(buf, want)
    one = torch.arange(6.0, device="cuda")
    mlt.beam_reorder(torch.tensor([5, 5, 0, 1, 2, -7], device="cuda"), one)
    assert one.tolist() == [5, 5, 0, 1, 2, 5]
    mlt.sync_status()
    mlt.beam_reorder(torch.tensor([1, 6, 1 << 40, 0, 4, 5], device="cuda"), one)
    assert one.tolist() == [5, 5, 0, 5, 2, 5]
    with pytest.raises(mlt.MltError, match="parent"):
        mlt.sync_status()
    mlt.sync_status()


def test_reorder_of_long_rows():
    """Offsets past 32 bits: two rows of 5 GB."""
    import torch

    n = 5 * (1 << 30)
    t = torch.zeros(2, n, dtype=torch.uint8, device="cuda")
    t[0, n - 5:] = 7
    t[1, :3] = 9
    mlt.beam_reorder(torch.tensor([[1, 0]], device="cuda"), t)
    assert (t[1, n - 5:] == 7).all() and (t[0, :3] == 9).all() and t[1, :3].sum() == 0 and t[0, n - 5:].sum() == 0


def test_step_and_reorder_over_several_steps():
    """A search of five steps over 4 options equals the best of all 4^5 sequences where no beam is lost."""
    import torch

    rng = np.random.default_rng(5)
    beams, n, steps = 64, 4, 5
    tables = torch.from_numpy(rng.standard_normal((steps, 64, n)).astype(np.float32)).cuda()
    logp = torch.full((1, beams), -math.inf, device="cuda")
    logp[0, 0] = 0.0
    state = torch.zeros(beams, 1, dtype=torch.int64, device="cuda")  # the digits so far as one number
    for t in range(steps):
        scores = tables[t][state[:, 0] % 64]
        parent, token, logp, _ = mlt.beam_step(scores[None], logp, beams)
        mlt.beam_reorder(parent, state)
        state[:, 0] = state[:, 0] * n + token[0].clamp(min=0)
    lp, alive = {0: 0.0}, tables.double().cpu().numpy()
    for t in range(steps):
        row = alive[t]
        row = row - np.log(np.exp(row).sum(1, keepdims=True))
        new = {s * n + d: v + row[s % 64, d] for s, v in lp.items() for d in range(n)}
        lp = dict(sorted(new.items(), key=lambda c: -c[1])[:beams])
    assert set(state[:, 0].tolist()) == set(lp)
    for s, v in zip(state[:, 0].tolist(), logp[0].tolist()):
        assert abs(lp[s] - v) <= 1e-5


def test_refusals():
    import torch

    x, lp = torch.zeros(2, 3, 10, device="cuda"), torch.zeros(2, 3, device="cuda")
    d = torch.zeros(2, 3, dtype=torch.bool, device="cuda")
    p = torch.zeros(2, 3, dtype=torch.int64, device="cuda")
    t = torch.zeros(6, 4, device="cuda")
    bad = [lambda: mlt.beam_step(x.cpu(), lp, 3), lambda: mlt.beam_step(x.double(), lp, 3), lambda: mlt.beam_step(x, lp[:1], 3),
           lambda: mlt.beam_step(x, lp.double(), 3), lambda: mlt.beam_step(x, lp, 0), lambda: mlt.beam_step(x, lp, 1025),
           lambda: mlt.beam_step(x, lp, 3, done=d), lambda: mlt.beam_step(x, lp, 3, done=d, eos=10),
           lambda: mlt.beam_step(x, lp, 3, done=d.int(), eos=1), lambda: mlt.beam_step(x, lp, 3, done=d[:1], eos=1),
           lambda: mlt.beam_step(x.transpose(1, 2), lp, 3), lambda: mlt.beam_step(x[0, 0], lp, 3),
           lambda: mlt.beam_step(torch.zeros(1, 100, 1000, device="cuda"), torch.zeros(1, 100, device="cuda"), 100),
           lambda: mlt.beam_step(torch.zeros(1, 1025, 2, device="cuda"), torch.zeros(1, 1025, device="cuda"), 4),
           lambda: mlt.beam_step(x[:, :0], lp[:, :0], 3), lambda: mlt.beam_step(x[..., :0], lp, 3),
           lambda: mlt.beam_reorder(p.int(), t), lambda: mlt.beam_reorder(p, t[:5]), lambda: mlt.beam_reorder(p, t.cpu()),
           lambda: mlt.beam_reorder(p, t.t()), lambda: mlt.beam_reorder(p, t, t), lambda: mlt.beam_reorder(p, t[:1].expand(6, 4)),
           lambda: mlt.beam_reorder(p, p), lambda: mlt.beam_reorder(p, *[t] * 65), lambda: mlt.beam_reorder(p[:, ::2], t)]
    for call in bad:
        with pytest.raises((TypeError, ValueError, mlt.MltError)):
            call()
    assert mlt.beam_step(x[:0], lp[:0], 3)[0].shape == (0, 3)
    mlt.beam_reorder(p[:0], t[:0])
    mlt.beam_reorder(p)
