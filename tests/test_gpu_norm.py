"""mlt_layer_norm and mlt_layer_norm_grad against the formulas in 64 bits.

u = 2^-24.  A sum over a row passes at most DEPTH = 26 + dim / 1024 roundings (8 values of a pack and 2 packs
in a thread, 5 shuffles, 6 over warps, 8 over CTAs where dim is above 2,048; long rows dim / 512 in a thread, 5
and 6), so it
is off by DEPTH u of the sum of magnitudes; what is made from it follows by
first-order propagation, written out in _forward and _backward."""
import math

import numpy as np
import pytest

from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}  # half a step of f16's subnormals


def _type(name):
    import torch

    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _rand(rng, shape, kind, scale=1.0, shift=0.0):
    import torch

    a = rng.standard_normal(shape) * scale + shift
    return torch.from_numpy(a.astype(np.float32)).cuda().to(_type(kind))


def _np(t):
    return t.double().cpu().numpy()


def _forward(t, w, b, eps):
    """y, mean, rstd of rows t in 64 bits and how far each may be off in 32 (y before its rounding)."""
    dim = t.shape[1]
    depth = 26 + dim / 1024
    mean = t.mean(1, keepdims=True)
    dm = (depth + 1) * U * np.abs(t).mean(1, keepdims=True)
    c = t - mean
    dc = dm + U * np.abs(c)
    var = (c * c).mean(1, keepdims=True)
    dv = (depth + 5) * U * var + dm ** 2 + U * eps
    rstd = 1 / np.sqrt(var + eps)
    dr = rstd * (dv / (2 * (var + eps)) + 4 * U)
    h = c * rstd
    dh = np.abs(c) * dr + rstd * dc + 2 * U * np.abs(h)
    y = h * w + b
    return y, mean, rstd, np.abs(w) * dh + U * np.abs(y), dm, dr


def _check_forward(x, residual, w, b, eps, got, kin, kout):
    import torch

    y, total, stats = got
    t = x.float() if residual is None else (x.float() + residual.float()).to(x.dtype).float()
    assert torch.equal(total.float(), t) and total.dtype == x.dtype
    t = _np(t).reshape(-1, x.shape[-1])
    one, zero = np.ones(t.shape[1]), np.zeros(t.shape[1])
    want, mean, rstd, err, dm, dr = _forward(t, one if w is None else _np(w), zero if b is None else _np(b),
                                             float(np.float32(eps)))
    assert y.dtype == _type(kout) and y.shape == x.shape and stats.shape == (*x.shape[:-1], 2)
    s = _np(stats).reshape(-1, 2)
    assert (np.abs(s[:, :1] - mean) <= dm + 2 * U * np.abs(mean)).all()
    assert (np.abs(s[:, 1:] - rstd) <= dr + 2 * U * rstd).all()
    off = np.abs(_np(y).reshape(want.shape) - want)
    assert (off <= err + UNIT[kout] * (np.abs(want) + err) + TINY[kout]).all()


SIZES = [(1, 1), (5, 2), (33, 7), (3, 8), (100, 61), (37, 64), (9, 128), (4, 250), (70, 256), (5, 257), (3, 264),
         (11, 1000), (7, 1024), (2, 4097), (3, 8192), (2, 8200), (1, 20001), (2, 32768), (1, 65536), (2, 65543)]


@pytest.mark.parametrize("kinds", ["f32 f32", "bf16 bf16", "f16 f16", "f32 bf16", "f32 f16"])
@pytest.mark.parametrize("rows,dim", SIZES)
def test_forward(rows, dim, kinds):
    kin, kout = kinds.split()
    rng = np.random.default_rng(rows * 7 + dim)
    x, r = _rand(rng, (rows, dim), kin, 1.5, 0.7), _rand(rng, (rows, dim), kin)
    for wk in ("f32", kin):
        w, b = _rand(rng, (dim,), wk, 0.1, 1.0), _rand(rng, (dim,), wk, 0.1)
        _check_forward(x, r, w, b, 1e-5, mlt.layer_norm(x, w, b, 1e-5, residual=r, out_dtype=_type(kout)), kin, kout)
    got = mlt.layer_norm(x, out_dtype=_type(kout))
    assert got[1] is x
    _check_forward(x, None, None, None, 1e-5, got, kin, kout)
    _check_forward(x, None, w, None, 0.25, mlt.layer_norm(x, w, eps=0.25, out_dtype=_type(kout)), kin, kout)
    _check_forward(x, None, None, b, 1e-5, mlt.layer_norm(x, None, b, out_dtype=_type(kout)), kin, kout)


@pytest.mark.parametrize("kind,dims", [("bf16", (6000, 6100, 6144, 8184, 8185, 16384, 114000, 114689)),
                                       ("f32", (3000, 3056, 4096, 4097, 12224, 12288, 57300, 57345))])
def test_sizes_of_shared_memory(kind, dims):
    """Weights, rows ahead and whole rows in shared memory: just below and above what fits unasked (48 KB with a
    kernel's own part) and at all (224 KB)."""
    rng = np.random.default_rng(0)
    for dim in dims:
        x, gy = _rand(rng, (3, dim), kind, 1.5, 0.7), _rand(rng, (3, dim), kind)
        w, b = _rand(rng, (dim,), "f32", 0.1, 1.0), _rand(rng, (dim,), "f32", 0.1)
        got = mlt.layer_norm(x, w, b, residual=gy)
        _check_forward(x, gy, w, b, 1e-5, got, kind, kind)
        g = mlt.layer_norm_grad(gy, got[1], got[2], w, b, g_total=gy)
        _check_backward(gy, got[1], got[2], w, gy, g, kind, "f32")


def test_many_rows_and_large_means():
    """More rows than all CTAs hold at once; a mean a thousand times the spread."""
    rng = np.random.default_rng(1)
    for rows, dim in ((200003, 5), (50001, 40), (5000, 1024)):
        x = _rand(rng, (rows, dim), "f32", 1.0, 1000.0)
        _check_forward(x, None, None, None, 1e-5, mlt.layer_norm(x), "f32", "f32")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [40, 61, 1000, 9000])
def test_strides_alignment_and_in_place(dim, kind):
    import torch

    rng = np.random.default_rng(dim)
    wide = _rand(rng, (20, dim + 16), kind)
    res = _rand(rng, (20, dim), kind)
    w, b = _rand(rng, (dim,), "f32"), _rand(rng, (dim,), "f32")
    for off in (0, 1, 2, 4, 8):
        x = wide[::2, off:off + dim]
        want = mlt.layer_norm(x.contiguous(), w, b, residual=res[::2].contiguous())
        buf = torch.full((10, dim + 16), 9.0, dtype=x.dtype, device="cuda")
        tot = torch.full((10, dim + 16), 9.0, dtype=x.dtype, device="cuda")
        y, t, s = mlt.layer_norm(x, w, b, residual=res[::2], out=buf[:, off:off + dim], total_out=tot[:, off:off + dim])
        # the split over threads goes by dim alone, but for packs: sums may differ by their order
        assert torch.equal(t, want[1]) and torch.allclose(y.float(), want[0].float(), rtol=2 ** -7, atol=1e-5)
        _check_forward(x, res[::2], w, b, 1e-5, (y, t, s), kind, kind)
        for q in (buf, tot):
            assert (q[:, :off] == 9).all() and (q[:, off + dim:] == 9).all()
    x, r = wide[:, :dim].contiguous(), res.clone()
    want = mlt.layer_norm(x, w, b, residual=r)
    a, c = x.clone(), r.clone()
    mlt.layer_norm(a, w, b, residual=c, out=a, total_out=c)  # y over x, the sum over the residual stream
    assert torch.equal(a, want[0]) and torch.equal(c, want[1])
    a, c = x.clone(), r.clone()
    mlt.layer_norm(a, w, b, residual=c, out=c, total_out=a)
    assert torch.equal(c, want[0]) and torch.equal(a, want[1])
    # leading dimensions, rows at no one distance (copied), one row read many times
    y, _, s = mlt.layer_norm(wide[:, :dim].reshape(4, 5, dim).transpose(0, 1), w, b)
    flat = mlt.layer_norm(wide[:, :dim].contiguous(), w, b)
    assert y.shape == (5, 4, dim) and s.shape == (5, 4, 2)
    again = x.reshape(4, 5, dim).transpose(0, 1).reshape(20, dim)
    _check_forward(again, None, w, b, 1e-5, (y.reshape(20, dim), again, s.reshape(20, 2)), kind, kind)
    if dim % 8 == 0:  # rows that lie alike towards 16-byte boundaries are summed in the same order
        assert torch.equal(y, flat[0].reshape(4, 5, dim).transpose(0, 1))
    y = mlt.layer_norm(x[:1].expand(33, dim), w, b)[0]
    assert torch.equal(y, flat[0][:1].expand(33, dim))


def test_rows_do_not_touch_each_other():
    """A NaN, an infinity and a row of equal values."""
    import torch

    rng = np.random.default_rng(4)
    for dim in (6, 64, 300, 9000, 70001):
        x = _rand(rng, (9, dim), "f32")
        want = mlt.layer_norm(x)[0]
        z = x.clone()
        z[2, 0], z[5, dim - 1], z[7] = math.nan, math.inf, 3.25
        y, _, s = mlt.layer_norm(z)
        assert y[2].isnan().all() and y[5].isnan().any() and (y[7] == 0).all()
        assert s[7, 0] == 3.25 and abs(s[7, 1].item() - 1e5 ** 0.5) <= 4 * U * 1e5 ** 0.5
        keep = [0, 1, 3, 4, 6, 8]
        assert torch.equal(y[keep], want[keep])


def _backward(gy, x, mean, rstd, w, gt, terms):
    """Gradients in 64 bits and how far they may be off before their rounding; `terms`: roundings on
    the way of a column's sum."""
    depth = 26 + x.shape[1] / 1024
    h = (x - mean) * rstd
    dh = 2 * U * np.abs(h)
    gw = gy * w
    m0, m1 = gw.mean(1, keepdims=True), (gw * h).mean(1, keepdims=True)
    dm0 = (depth + 2) * U * np.abs(gw).mean(1, keepdims=True)
    dm1 = (depth + 6) * U * np.abs(gw * h).mean(1, keepdims=True)
    inner = gw - m0 - h * m1
    de = U * np.abs(gw) + dm0 + U * np.abs(gw - m0) + dh * np.abs(m1) + np.abs(h) * dm1 + U * np.abs(inner)
    gx, dx = inner * rstd, (de + U * np.abs(inner)) * rstd
    if gt is not None:
        gx = gx + gt
        dx = dx + U * np.abs(gx)
    return {"x": (gx, dx), "weight": ((gy * h).sum(0), (terms + 4) * U * np.abs(gy * h).sum(0)),
            "bias": (gy.sum(0), terms * U * np.abs(gy).sum(0))}


# a thread's 64 rows in a plain sum (more are compensated: two roundings), 5 over the groups of a warp, 8 over
# warps, a compensated sum over teams, 5 over threads
TERMS = 64 + 5 + 8 + 2 + 5


def _check_backward(gy, x, stats, w, gt, got, kin, wk):
    s = _np(stats).reshape(-1, 2)
    flat = lambda t: None if t is None else _np(t).reshape(-1, x.shape[-1])  # noqa: E731
    want = _backward(flat(gy), flat(x), s[:, :1], s[:, 1:], 1.0 if w is None else _np(w), flat(gt), TERMS)
    for name, (v, e) in want.items():
        if got[name] is None:
            continue
        kind = kin if name == "x" else wk
        assert got[name].dtype == _type(kind)
        off = np.abs(_np(got[name]).reshape(v.shape) - v)
        assert (off <= e + UNIT[kind] * (np.abs(v) + e) + TINY[kind]).all(), name


@pytest.mark.parametrize("kinds", ["f32 f32", "bf16 bf16", "f16 f16", "f32 bf16", "f32 f16"])
@pytest.mark.parametrize("rows,dim", SIZES + [(1500, 33), (40000, 24), (700, 300), (20000, 260), (300, 5000)])
def test_backward(rows, dim, kinds):
    kin, kout = kinds.split()
    rng = np.random.default_rng(rows * 5 + dim)
    x, gy, gt = _rand(rng, (rows, dim), kin, 1.5, 0.7), _rand(rng, (rows, dim), kout), _rand(rng, (rows, dim), kin)
    stats = mlt.layer_norm(x)[2]
    for wk, more in (("f32", None), (kin, gt)):
        w, b = _rand(rng, (dim,), wk, 0.2, 1.0), _rand(rng, (dim,), wk)
        g = mlt.layer_norm_grad(gy, x, stats, w, b, g_total=more)
        _check_backward(gy, x, stats, w, more, g, kin, wk)
    g = mlt.layer_norm_grad(gy, x, stats, g_total=gt)
    assert g["weight"] is None and g["bias"] is None
    _check_backward(gy, x, stats, None, gt, g, kin, kin)
    g = mlt.layer_norm_grad(gy, x, stats, None, b)
    assert g["weight"] is None
    _check_backward(gy, x, stats, None, None, g, kin, kin)


def test_gradient_equals_differences():
    """Along a direction, by central differences of the 64-bit formula: their error is of the order of
    step^2 = 1e-8 of the third derivative; the kernel's fp32 gradients give 1e-6."""
    import torch

    rng = np.random.default_rng(9)
    x, gy = _rand(rng, (13, 77), "f32", 2.0, 0.5), _rand(rng, (13, 77), "f32")
    w, b = _rand(rng, (77,), "f32", 0.3, 1.0), _rand(rng, (77,), "f32")
    _, _, stats = mlt.layer_norm(x, w, b)
    g = mlt.layer_norm_grad(gy, x, stats, w, b)
    t = {"x": _np(x), "weight": _np(w), "bias": _np(b)}
    loss = lambda q: (_np(gy) * _forward(q["x"], q["weight"], q["bias"], 1e-5)[0]).sum()  # noqa: E731
    for name in t:
        d = rng.standard_normal(t[name].shape)
        up, down = dict(t), dict(t)
        up[name], down[name] = t[name] + 1e-4 * d, t[name] - 1e-4 * d
        want = (loss(up) - loss(down)) / 2e-4
        have = (_np(g[name]) * d).sum()
        assert abs(have - want) <= 2e-6 * np.abs(_np(g[name]) * d).sum()
    assert torch.isfinite(g["x"]).all()


def test_equal_terms_of_many_rows():
    """A plain sum of a million equal terms is off by its length; compensated ones by 2 u for each
    of two sums and u for each of 18 further additions."""
    import torch

    for rows, dim in ((1 << 20, 3), (300001, 300)):
        x = torch.zeros(rows, dim, device="cuda")
        x[:, 0] = 1.0
        stats = torch.stack([torch.full((rows,), -0.7, device="cuda"), torch.full((rows,), 1.3, device="cuda")], 1)
        gy = torch.full((rows, dim), 0.1, device="cuda")
        w = torch.ones(dim, device="cuda")
        g = mlt.layer_norm_grad(gy, x, stats.contiguous(), w, w)
        one = float(np.float32(0.1))
        assert np.abs(_np(g["bias"]) - rows * one).max() <= 22 * U * rows * one
        h = (_np(x[:1])[0] - float(np.float32(-0.7))) * float(np.float32(1.3))
        assert (np.abs(_np(g["weight"]) - rows * one * h) <= 26 * U * rows * one * h).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [40, 61, 1000, 9000, 33000])
def test_backward_strides_and_in_place(dim, kind):
    import torch

    rng = np.random.default_rng(dim + 1)
    wide, gwide = _rand(rng, (20, dim + 16), kind), _rand(rng, (20, dim + 16), kind)
    w, b = _rand(rng, (dim,), "f32"), _rand(rng, (dim,), "f32")
    for off in (0, 1, 2, 4, 8):
        x, gy = wide[::2, off:off + dim], gwide[::2, off:off + dim]
        stats = mlt.layer_norm(x)[2]
        buf = torch.full((10, dim + 16), 9.0, dtype=x.dtype, device="cuda")
        g = mlt.layer_norm_grad(gy, x, stats, w, b, g_total=gy, out=buf[:, off:off + dim])
        _check_backward(gy, x, stats, w, gy, g, kind, "f32")
        assert (buf[:, :off] == 9).all() and (buf[:, off + dim:] == 9).all()
    x, gy, gt = (t[:, :dim].contiguous() for t in (wide, gwide, gwide))
    stats = mlt.layer_norm(x)[2]
    want = mlt.layer_norm_grad(gy, x, stats, w, b, g_total=gt)
    over = gy.clone()
    g = mlt.layer_norm_grad(over, x, stats, w, b, g_total=gt, out=over)
    assert g["x"] is over and all(torch.equal(g[k], want[k]) for k in want)
    over = gt.clone()
    g = mlt.layer_norm_grad(gy, x, stats, w, b, g_total=over, out=over)
    assert all(torch.equal(g[k], want[k]) for k in want)
    # a gradient broadcast over the rows
    row = gy[:1].expand(20, dim)
    _check_backward(row, x, stats, w, None, mlt.layer_norm_grad(row, x, stats, w, b), kind, "f32")


def test_more_than_32_bits_of_values():
    """The last row of 4.6 billion values is normed, and its gradient lands there."""
    import torch

    rows, dim = 70001, 65536
    x = torch.zeros(rows, dim, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator("cuda").manual_seed(3)
    last = torch.randn(1, dim, device="cuda", generator=gen).bfloat16()
    x[-1:] = last
    want, _, stats = mlt.layer_norm(last)
    g = mlt.layer_norm_grad(last, last, stats)["x"]
    y, _, s = mlt.layer_norm(x)
    assert torch.equal(y[-1:], want) and torch.equal(s[-1:], stats) and (y[-2] == 0).all()
    out = mlt.layer_norm_grad(x, x, s, out=x)["x"]
    assert torch.equal(out[-1:], g) and (out[-2] == 0).all()


def test_no_rows():
    import torch

    x = torch.empty(0, 37, device="cuda")
    w = torch.ones(37, device="cuda")
    y, total, stats = mlt.layer_norm(x, w, w, residual=x)
    assert y.shape == (0, 37) and total.shape == (0, 37) and stats.shape == (0, 2)
    g = mlt.layer_norm_grad(x, x, stats, w, w)
    assert g["x"].shape == (0, 37) and (g["weight"] == 0).all() and (g["bias"] == 0).all()
    y = mlt.layer_norm(torch.empty(3, 0, 8, device="cuda", dtype=torch.bfloat16))[0]
    assert y.shape == (3, 0, 8)


def test_refusals():
    import torch

    x, w = torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda")
    s = torch.zeros(4, 2, device="cuda")
    bad = [lambda: mlt.layer_norm(x.cpu()), lambda: mlt.layer_norm(x.double()), lambda: mlt.layer_norm(x, w[:4]),
           lambda: mlt.layer_norm(x, w, w.bfloat16()), lambda: mlt.layer_norm(x, residual=x[:2]),
           lambda: mlt.layer_norm(x, residual=x.bfloat16()), lambda: mlt.layer_norm(x, out=x[:2]),
           lambda: mlt.layer_norm(x, total_out=x), lambda: mlt.layer_norm(x.t()),
           lambda: mlt.layer_norm(x, w.repeat(2)[::2]), lambda: mlt.layer_norm(x, eps=-1.0),
           lambda: mlt.layer_norm(x, eps=math.nan), lambda: mlt.layer_norm(x.bfloat16(), out_dtype=torch.float32),
           lambda: mlt.layer_norm(x, residual=x, out=x, total_out=x),
           lambda: mlt.layer_norm(torch.zeros(4, 0, device="cuda")),
           lambda: mlt.layer_norm_grad(x[:2], x, s), lambda: mlt.layer_norm_grad(x, x, s[:2]),
           lambda: mlt.layer_norm_grad(x, x, s.double()), lambda: mlt.layer_norm_grad(x, x, s, g_total=x.half()),
           lambda: mlt.layer_norm_grad(x, x, s, out=x[:2])]
    for call in bad:
        with pytest.raises((TypeError, ValueError, mlt.MltError)):
            call()


def test_captured_and_on_another_stream():
    import torch

    rng = np.random.default_rng(2)
    x, r, gy = (_rand(rng, (777, 520), "bf16") for _ in range(3))
    w, b = _rand(rng, (520,), "f32"), _rand(rng, (520,), "f32")

    def both(**kw):
        y, t, s = mlt.layer_norm(x, w, b, residual=r, **kw)
        if "stream" in kw:
            kw["stream"].synchronize()
        g = mlt.layer_norm_grad(gy, t, s, w, b, g_total=gy, **kw)
        return [y, t, s, *g.values()]

    want = [v.clone() for v in both()]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = both(stream=s)
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(2):
        for v in got:
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, got))
