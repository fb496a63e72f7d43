"""mlt_embed and mlt_embed_grad against plain 64-bit implementations.

Lookup: one 32-bit product and one rounding, so 2^-24 of the value for the
product and half a unit of the output type.  Gradient: a row's sum of k terms
in 32 bits is off by at most k 2^-24 of the sum of magnitudes, plus the scale's
product and the rounding."""
import math

import numpy as np
import pytest

import sequence as S
from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu

UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _type(name):
    import torch

    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _rand(rng, shape, kind):
    import torch

    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda().to(_type(kind))


def _check_embed(ids, table, scale, out, kind):
    want = S.embed(ids.cpu().numpy(), table.float().cpu().numpy(), scale)
    tol = np.abs(want) * (2.0 ** -24 + UNIT[kind]) + (2.0 ** -25 if kind == "f16" else 0)  # f16: subnormals
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("kinds", ["f32 f32", "bf16 bf16", "f16 f16", "f32 bf16", "bf16 f32", "f32 f16"])
@pytest.mark.parametrize("tokens,vocab,dim", [(1, 1, 1), (3, 5, 7), (64, 100, 24), (17, 1000, 130), (1000, 33, 1024),
                                              (5, 64, 4100), (257, 50, 16)])
def test_lookup(tokens, vocab, dim, kinds):
    import torch

    kin, kout = kinds.split()
    rng = np.random.default_rng(tokens + dim)
    table = _rand(rng, (vocab, dim), kin)
    for idt in (torch.int64, torch.int32):
        ids = torch.from_numpy(rng.integers(-1, vocab, tokens)).cuda().to(idt)
        out = mlt.embed(ids, table, scale=1.7, out_dtype=_type(kout))
        assert out.dtype == _type(kout) and out.shape == (tokens, dim)
        _check_embed(ids, table, 1.7, out, kout)
    mlt.sync_status()


def test_lookup_shapes_strides_and_alignment():
    import torch

    rng = np.random.default_rng(0)
    wide = _rand(rng, (40, 70), "bf16")
    ids = torch.from_numpy(rng.integers(0, 20, (3, 4, 5))).cuda()
    for a in range(0, 9):
        table = wide[::2, a:a + 61]
        out = mlt.embed(ids, table, scale=0.5)
        assert out.shape == (3, 4, 5, 61)
        _check_embed(ids.reshape(-1), table, 0.5, out.reshape(-1, 61), "bf16")
        buf = torch.full((60, 80), 9.0, dtype=torch.bfloat16, device="cuda")
        view = buf[:, a:a + 61]
        mlt.embed(ids.reshape(-1), table, scale=0.5, out=view)
        assert torch.equal(view, out.reshape(-1, 61))
        assert (buf[:, :a] == 9).all() and (buf[:, a + 61:] == 9).all()


def test_ids_out_of_range():
    import torch

    table = torch.ones((10, 6), device="cuda")
    ids = torch.tensor([3, -1, 10, -2 ** 40, 2 ** 40, 9], device="cuda")
    mlt.sync_status()
    out = mlt.embed(ids, table)
    with pytest.raises(mlt.MltError) as e:
        mlt.sync_status()
    assert e.value.code == -1 and "id" in str(e.value)
    assert out.sum(1).tolist() == [6, 0, 0, 0, 0, 6]
    g = mlt.embed_grad(ids, torch.ones((6, 6), device="cuda"), 10)
    with pytest.raises(mlt.MltError):
        mlt.sync_status()
    assert g.sum(1).tolist() == [0, 0, 0, 6, 0, 0, 0, 0, 0, 6]
    mlt.sync_status()


def _check_grad(ids, grad, vocab, scale, out, kind):
    i, g = ids.cpu().numpy().reshape(-1), grad.float().cpu().numpy().reshape(-1, grad.shape[-1])
    want, mag = S.embed_grad(i, g, vocab, scale)
    count = np.bincount(i[(i >= 0) & (i < vocab)], minlength=vocab)[:, None]
    tol = mag * (count + 2) * 2.0 ** -24 + np.abs(want) * UNIT[kind] + (2.0 ** -25 if kind == "f16" else 0)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("kinds", ["f32 f32", "bf16 bf16", "f16 f16", "bf16 f32"])
@pytest.mark.parametrize("tokens,vocab,dim,skew", [
    (1, 1, 1, 0), (1, 300, 5, 0), (7, 3, 33, 0), (1000, 2, 8, 0), (5000, 64, 128, 0), (5000, 70000, 40, 0),
    (40000, 900, 9, 1), (4097, 257, 1030, 1), (30000, 1, 4, 0), (20001, 300000, 3, 2)])
def test_gradient(tokens, vocab, dim, skew, kinds):
    import torch

    kin, kout = kinds.split()
    rng = np.random.default_rng(tokens + vocab)
    w = np.arange(1, vocab + 1) ** -float(skew)
    ids = rng.permutation(vocab)[np.searchsorted(np.cumsum(w), rng.random(tokens) * w.sum()).clip(max=vocab - 1)]
    ids[rng.random(tokens) < 0.05] = -1
    grad = _rand(rng, (tokens, dim), kin)
    for idt in (torch.int64, torch.int32):
        t = torch.from_numpy(ids).cuda().to(idt)
        out = mlt.embed_grad(t, grad, vocab, scale=3.0, out_dtype=_type(kout))
        assert out.shape == (vocab, dim) and out.dtype == _type(kout)
        _check_grad(t, grad, vocab, 3.0, out, kout)
        assert torch.equal(out, mlt.embed_grad(t, grad, vocab, scale=3.0, out_dtype=_type(kout)))
    mlt.sync_status()


def test_gradient_is_that_of_the_lookup():
    """Against differences: the lookup is linear in the table, so with L = sum(out * g) and a step e in one
    entry (a power of two, in f32, table zero elsewhere in that entry's column sums) L moves by grad * e."""
    import torch

    rng = np.random.default_rng(4)
    ids = torch.from_numpy(rng.integers(0, 6, 50)).cuda()
    g = _rand(rng, (50, 3), "f32")
    grad = mlt.embed_grad(ids, g, 6, scale=2.0).double().cpu()
    table = torch.zeros((6, 3), device="cuda")
    for v in range(6):
        for c in range(3):
            table[v, c] = 4.0
            moved = (mlt.embed(ids, table, scale=2.0).double() * g.double()).sum().item()
            table[v, c] = 0.0
            assert abs(moved / 4.0 - grad[v, c].item()) <= 60 * 2.0 ** -24 * 2 * g[:, c].abs().sum().item()


def test_gradient_strides_empty_and_streams():
    import torch

    rng = np.random.default_rng(9)
    ids = torch.from_numpy(rng.integers(0, 30, 200)).cuda()
    wide = _rand(rng, (200, 50), "bf16")
    for a in (0, 1, 4, 8):
        grad = wide[:, a:a + 41]
        buf = torch.full((30, 60), 7.0, device="cuda")
        mlt.embed_grad(ids, grad, 30, out=buf[:, a:a + 41])
        _check_grad(ids, grad, 30, 1.0, buf[:, a:a + 41], "f32")
        assert (buf[:, :a] == 7).all() and (buf[:, a + 41:] == 7).all()
    none = torch.empty((0,), dtype=torch.int64, device="cuda")
    assert (mlt.embed_grad(none, torch.empty((0, 5), device="cuda"), 12) == 0).all()
    assert (mlt.embed_grad(torch.full((9,), -1, device="cuda"), torch.ones((9, 5), device="cuda"), 12) == 0).all()
    assert mlt.embed(none, torch.ones((4, 5), device="cuda")).shape == (0, 5)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    want = mlt.embed_grad(ids, wide, 30)
    torch.cuda.synchronize()
    for _ in range(10):
        with torch.cuda.stream(a):
            p = mlt.embed_grad(ids, wide, 30)
        with torch.cuda.stream(b):
            q = mlt.embed_grad(ids, wide, 30)
        torch.cuda.synchronize()
        assert torch.equal(p, want) and torch.equal(q, want)


def test_binding_refuses():
    import torch

    t = torch.ones((4, 6), device="cuda")
    ids = torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(TypeError):
        mlt.embed(ids.float(), t)
    with pytest.raises(TypeError):
        mlt.embed(ids, t.double())
    with pytest.raises(ValueError):
        mlt.embed(ids, t.t())
    with pytest.raises(ValueError):
        mlt.embed(ids, t, out=torch.empty((3, 5), device="cuda"))
    with pytest.raises(ValueError):
        mlt.embed_grad(ids, t, 4)
    with pytest.raises(mlt.MltError):
        mlt.embed_grad(ids, t[:3], 0)


@pytest.mark.parametrize("kinds", ["f32 f32", "bf16 bf16", "f16 f32", "f32 bf16"])
@pytest.mark.parametrize("tokens,dim,stride", [(5, 269, 269), (20011, 131, 140), (39001, 174, 174), (80003, 269, 273),
                                               (100003, 140, 140)])
def test_many_rows_of_narrow_packs(tokens, dim, stride, kinds):
    """Rows that only narrow accesses fit, by one to four rows a warp."""
    import torch

    ti, to = ({"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[k] for k in kinds.split())
    rng = np.random.default_rng(tokens + dim)
    ids = torch.from_numpy(rng.integers(-3, 301, tokens)).cuda()
    table = torch.from_numpy(rng.standard_normal((301, stride)).astype(np.float32)).cuda().to(ti)[:, :dim]
    buf = torch.full((tokens, stride), 7.0, device="cuda", dtype=to)
    mlt.embed(ids, table, scale=1.7, out=buf[:, :dim])
    want = (table.float() * np.float32(1.7).item())[ids.clamp(min=0)] * (ids >= 0)[:, None]
    assert torch.equal(buf[:, :dim], want.to(to))
    assert (buf[:, dim:] == 7.0).all()
    mlt.sync_status()
