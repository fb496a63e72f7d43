"""mlt_sample against a plain 64-bit implementation.

The scaled score and the draw key are defined as 32-bit operations, so indices
have to be equal.  Log-probabilities: a lane adds at most a 256th of the row's
weights one after another, each sum off by 2^-24 of it, then up to 16 joins;
a weight is off by 2^-22; the difference s - max is rounded once and the result once."""
import math

import numpy as np
import pytest

import sequence as S
from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu

RULES = {
    "plain": dict(temperature=0.8),
    "greedy": dict(temperature=0.0, top_k=3, top_p=0.5),
    "top_k": dict(temperature=1.1, top_k=40),
    "top_k1": dict(temperature=0.7, top_k=1),
    "top_p": dict(temperature=0.9, top_p=0.9),
    "top_p0": dict(temperature=0.9, top_p=0.0),
    "min_p": dict(temperature=1.3, min_p=0.05),
    "min_p2": dict(temperature=1.3, min_p=2.0),
    "all": dict(temperature=1.5, top_k=30, top_p=0.8, min_p=0.01),
}


def _type(name):
    import torch

    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _check(scores, noise, got, m, rules):
    """rules: one dict for every row, or a list of them."""
    index, logp = (t.cpu().numpy() for t in got)
    x, g = scores.float().cpu().numpy(), noise.cpu().numpy()
    rows, n = x.shape
    assert index.shape == logp.shape == (rows, m)
    for r in range(rows):
        q = dict(dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **(rules[r] if isinstance(rules, list) else rules))
        q = {k: float(np.float32(v)) if k != "top_k" else v for k, v in q.items()}
        want, want_p = S.sample_row(x[r], g[r], m=m, **q)
        assert np.array_equal(index[r], want), (r, q, index[r][:8], want[:8])
        fine = np.isfinite(want_p)
        assert np.array_equal(np.isfinite(logp[r]), fine) and (logp[r][~fine] == -np.inf).all()
        tol = (n / 256 + 24) * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -22 * np.abs(want_p[fine])
        assert (np.abs(logp[r][fine] - want_p[fine]) <= tol).all(), (r, q)


def _inputs(rows, n, kind, seed, masked=0.0, steps=0):
    import torch

    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, n)).astype(np.float32) * 3
    if steps:
        x = np.round(x * steps) / steps  # many equal scores
    x[rng.random((rows, n)) < masked] = -np.inf
    g = -np.log(rng.exponential(size=(rows, n))).astype(np.float32)
    return torch.from_numpy(x).cuda().to(_type(kind)), torch.from_numpy(g).cuda()


@pytest.mark.parametrize("rule", list(RULES))
@pytest.mark.parametrize("n", [1, 2, 8, 31, 33, 200, 512, 513, 1999, 5003, 40009])
def test_one_draw(n, rule):
    for kind, masked, steps in (("f32", 0.0, 0), ("bf16", 0.3, 0), ("f16", 0.0, 2)):
        x, g = _inputs(3, n, kind, n + len(rule), masked, steps)
        _check(x, g, mlt.sample(x, g, **RULES[rule]), 1, RULES[rule])
    mlt.sync_status()


@pytest.mark.parametrize("rule", list(RULES))
@pytest.mark.parametrize("n,m", [(8, 8), (40, 64), (512, 32), (512, 33), (700, 700), (3001, 2048), (70001, 257)])
def test_draws_without_replacement(n, m, rule):
    for kind, masked, steps in (("f32", 0.5, 0), ("bf16", 0.0, 0), ("f32", 0.0, 1)):
        x, g = _inputs(2, n, kind, n + m, masked, steps)
        _check(x, g, mlt.sample(x, g, m=m, **RULES[rule]), m, RULES[rule])
    mlt.sync_status()


@pytest.mark.parametrize("m", [1, 5])
@pytest.mark.parametrize("rows,n", [(9, 64), (9, 6007), (200, 900), (77, 30011)])
def test_rules_of_their_own(rows, n, m):
    import torch

    names = list(RULES)
    each = [RULES[names[r % len(names)]] for r in range(rows)]
    full = [dict(dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **q) for q in each]
    rules = mlt.sample_rules(*(torch.tensor([q[k] for q in full]) for k in ("temperature", "top_k", "top_p", "min_p")))
    x, g = _inputs(rows, n, "bf16", rows, 0.1)
    _check(x, g, mlt.sample(x, g, rules=rules, m=m), m, each)


@pytest.mark.parametrize("n", [40, 3000, 100003])
def test_one_long_row_and_equal_scores(n):
    """A team of CTAs shares the row; equal scores are cut by index."""
    import torch

    for rule in (dict(top_k=n // 3), dict(top_p=0.4), dict(top_k=n // 2, top_p=0.5, min_p=0.2)):
        for steps in (1, 8):
            x, g = _inputs(1, n, "f32", n, 0.2, steps)
            for m in (1, 20):
                _check(x, g, mlt.sample(x, g, m=m, **rule), m, rule)
        x = torch.full((1, n), 1.25, device="cuda")
        for m in (1, 7):
            _check(x, g, mlt.sample(x, g, m=m, **rule), m, rule)


@pytest.mark.parametrize("n", [16, 600, 9001])
def test_values_that_mask(n):
    """Empty rows, NaN, infinities, the type's lowest value and noise out of the ordinary."""
    import torch

    for kind in ("f32", "bf16", "f16"):
        x, g = _inputs(8, n, kind, n)
        low = torch.finfo(x.dtype).min
        x[0] = -math.inf
        x[1] = math.nan
        x[2] = low
        x[3, ::2] = low
        x[3, 1::3] = math.nan
        x[4, n // 2] = math.inf
        x[5, :] = -math.inf
        x[5, n - 1] = -3.0
        g[6, ::2] = math.nan
        g[6, 1] = -math.inf
        g[7, n // 3] = math.inf
        for rule in (dict(), dict(top_k=4), dict(top_p=0.7), dict(temperature=0.25, min_p=0.1), dict(temperature=0.0)):
            for m in (1, 3):
                _check(x, g, mlt.sample(x, g, m=m, **rule), m, rule)
    mlt.sync_status()


@pytest.mark.parametrize("n", [37, 1301])
def test_strides_and_alignment(n):
    import torch

    x, g = _inputs(6, n + 40, "f16", 5)
    for a in range(0, 9):
        for rule in (dict(), dict(top_k=11, top_p=0.9)):
            xs, gs = x[::2, a:a + n], g[1::2, 9 - a:9 - a + n]
            _check(xs, gs, mlt.sample(xs, gs, m=2, **rule), 2, rule)
    xt = torch.arange(12.0, device="cuda")
    i, p = mlt.sample(xt, torch.zeros(12, device="cuda"), m=3)
    assert i.tolist() == [11, 10, 9] and p.shape == (3,)


def test_many_chains():
    x, g = _inputs(5000, 8, "f32", 1, 0.4)
    _check(x, g, mlt.sample(x, g, temperature=0.6, top_p=0.8), 1, dict(temperature=0.6, top_p=0.8))


def test_the_same_from_call_to_call_and_on_two_streams():
    import torch

    x, g = _inputs(4, 300007, "f32", 2, 0.3)
    calls = [dict(top_k=5000, top_p=0.7, m=300), dict(min_p=0.001, m=1000), dict(top_p=0.95)]
    want = [mlt.sample(x, g, **q) for q in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        got = []
        for s, q in zip(streams, calls):
            with torch.cuda.stream(s):
                got.append(mlt.sample(x, g, **q))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_graph_capture():
    import torch

    x, g = _inputs(2, 200003, "f32", 8)
    index = torch.empty((2, 4), dtype=torch.int64, device="cuda")
    logp = torch.empty((2, 4), device="cuda")
    mlt.sample(x, g, top_k=100, m=4, out=(index, logp))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            mlt.sample(x, g, top_k=100, m=4, out=(index, logp))
    torch.cuda.synchronize()
    for seed in (3, 4):
        x2, g2 = _inputs(2, 200003, "f32", seed)
        x.copy_(x2)
        g.copy_(g2)
        graph.replay()
        torch.cuda.synchronize()
        _check(x, g, (index, logp), 4, dict(top_k=100))


def test_shares_of_the_draws():
    """With Gumbel noise the first draw follows the kept entries' softmax: shares of 200,000
    draws lie within six standard deviations."""
    import torch

    p = torch.tensor([0.05, 0.2, 0.4, 0.25, 0.1])
    rows = 200000
    x = p.log().cuda().expand(rows, 5).contiguous()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    g = -torch.empty(rows, 5, device="cuda").exponential_(generator=gen).log()
    i, lp = mlt.sample(x, g, top_k=4)
    share = torch.bincount(i[:, 0], minlength=5).double().cpu() / rows
    want = torch.tensor([0, 0.2, 0.4, 0.25, 0.1], dtype=torch.float64) / 0.95
    assert ((share - want).abs() <= 6 * (want * (1 - want) / rows).sqrt()).all()


def test_rules_out_of_range_draw_nothing_and_are_reported():
    import torch

    for n in (30, 3000):
        x, g = _inputs(4, n, "f32", 3)
        rules = mlt.sample_rules(torch.tensor([1.0, -1.0, math.nan, 1.0]), 0, torch.tensor([1.0, 1.0, 1.0, math.nan]))
        mlt.sync_status()
        i, lp = mlt.sample(x, g, rules=rules, m=2)
        with pytest.raises(mlt.MltError) as e:
            mlt.sync_status()
        assert e.value.code == -1 and "rule" in str(e.value)
        assert (i[0] >= 0).all() and (i[1:] == -1).all() and torch.isinf(lp[1:]).all()
        mlt.sync_status()


def test_no_rows_and_no_entries():
    import torch

    e = torch.empty((0, 50), device="cuda")
    i, lp = mlt.sample(e, e, m=3)
    assert i.shape == (0, 3)
    e = torch.empty((5, 0), device="cuda")
    for m in (3, 100):
        i, lp = mlt.sample(e, e, m=m)
        assert (i == -1).all() and (lp == -math.inf).all() and i.shape == (5, m)


def test_binding_refuses():
    import torch

    x, g = _inputs(2, 16, "f32", 1)
    with pytest.raises(TypeError):
        mlt.sample(x.double(), g)
    with pytest.raises(TypeError):
        mlt.sample(x, g.half())
    with pytest.raises(TypeError):
        mlt.sample(x.cpu(), g)
    with pytest.raises(ValueError):
        mlt.sample(x, g[:, :8])
    with pytest.raises(ValueError):
        mlt.sample(x.t(), g.t())
    with pytest.raises(ValueError):
        mlt.sample(x, g, rules=torch.zeros((3, 4), dtype=torch.int32, device="cuda"))
    for bad in (dict(m=0), dict(m=2049), dict(temperature=-1.0), dict(temperature=math.nan), dict(top_p=math.nan)):
        with pytest.raises(mlt.MltError) as e:
            mlt.sample(x, g, **bad)
        assert e.value.code == -1
