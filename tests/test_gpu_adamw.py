"""mlt_adamw against the formulas.

Moments are defined operation by operation in 32 bits, so they are compared bit for bit with the same
operations in numpy; 8-bit ones too, with the hash that places a value between two
codes.  A parameter is compared with 64 bits: of the step, its rate, two moments' roundings,
the root (two units), the quotient (two) and some single operations are off by at most 12 u of it,
u = 2^-24; the decayed value by 2 u of itself; then half a unit of the type."""
import math

import numpy as np
import pytest

from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
BLOCK = 256
F = np.float32


def _type(name):
    import torch

    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _mix(h):
    h = np.asarray(h, np.uint32)
    h = (h ^ (h >> np.uint32(16))) * np.uint32(0x9E3779B1)
    h = (h ^ (h >> np.uint32(15))) * np.uint32(0xB504F333)
    return h ^ (h >> np.uint32(16))


# the formats' values by code, from their definition
def _table(mantissa, bias, special):
    c = np.arange(256)
    e, f = (c & 127) >> mantissa, c & ((1 << mantissa) - 1)
    mag = np.where(e > 0, (1 + f / 2.0 ** mantissa) * 2.0 ** (e - bias), f / 2.0 ** mantissa * 2.0 ** (1 - bias))
    return np.where(special(c & 127), np.nan, np.where(c > 127, -mag, mag))


E4M3 = _table(3, 7, lambda c: c == 127)
E5M2 = np.where((np.arange(256) & 127) == 124, np.inf, _table(2, 15, lambda c: c > 124))


def _encode(x, first_block, key, which):
    """Codes and scales of a tensor's moment (fp32 array)."""
    n = x.size
    pad = np.zeros(-(-n // BLOCK) * BLOCK, F)
    pad[:n] = x
    pad = pad.reshape(-1, BLOCK)
    mag = np.abs(pad).view(np.uint32)
    e = np.maximum(mag.max(1) >> 23, 16).astype(np.int64)
    with np.errstate(over="ignore"):
        b = (first_block + np.arange(len(pad))).astype(np.uint32)
        h = _mix(_mix(b + key)[:, None] + np.arange(BLOCK, dtype=np.uint32) * np.uint32(0x9E3779B9))
    r = (h & 0xFFFF) if which == "m" else h >> 16
    bias, drop, low = (134, 20, -120) if which == "m" else (141, 21, -112)
    with np.errstate(all="ignore"):
        s = np.abs(pad) * ((127 + bias - e) << 23).astype(np.uint32).view(F)[:, None] * F(2.0 ** low)
    code = (s.view(np.uint32).astype(np.int64) + (r.astype(np.int64) << (drop - 16))) >> drop
    if which == "m":
        code |= (pad.view(np.uint32) >> 31).astype(np.int64) << 7
    else:
        code = np.where(pad > 0, np.maximum(code, 1), code)
    code[e == 255] = 127
    return code.reshape(-1)[:n].astype(np.uint8), ((127 - bias + e) << 23).astype(np.uint32).view(F)


def _decode(code, scale, which):
    t = (E4M3 if which == "m" else E5M2).astype(F)
    return t[code] * np.repeat(scale, BLOCK)[:code.size]


def _bytes(t):
    import torch

    return t.view(torch.uint8).cpu().numpy()


class Model:
    """Tensors on the GPU and the same in numpy."""

    def __init__(self, sizes, kinds=("f32", "f32", None), bits=32, seed=0, offset=0):
        import torch

        rng = np.random.default_rng(seed)
        self.kinds, self.bits, self.sizes = kinds, bits, sizes
        new = lambda n, dt: torch.empty(n + offset, dtype=_type(dt), device="cuda")[offset:]  # noqa: E731
        self.rng, self.new = rng, new
        self.params = [new(n, kinds[0]).copy_(torch.from_numpy(rng.standard_normal(n).astype(F))) for n in sizes]
        self.copies = None if kinds[2] is None else [new(n, kinds[2]).zero_() for n in sizes]
        self.state = mlt.adamw_state(self.params, bits)
        self.first = np.concatenate([[0], np.cumsum([-(-n // BLOCK) for n in sizes])])

    def grads(self, spread=2.0):
        import torch

        return [self.new(n, self.kinds[1]).copy_(torch.from_numpy(
            (self.rng.standard_normal(n) * np.exp(spread * self.rng.standard_normal(n)) * 0.01).astype(F)))
            for n in self.sizes]

    def moments(self, k):
        """m and v of tensor k as fp32 arrays."""
        at, n = self.first[k] * BLOCK, self.sizes[k]
        if self.bits == 32:
            return tuple(t[at:at + n].cpu().numpy() for t in self.state[:2])
        blocks = slice(self.first[k], self.first[k + 1])
        return tuple(_decode(_bytes(t)[at:at + n], s[blocks].cpu().numpy(), w)
                     for t, s, w in ((self.state.m, self.state.m_scale, "m"), (self.state.v, self.state.v_scale, "v")))

    def step(self, grads, t, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, decay=0.0, scale=None, seed=0, **kw):
        """One step, checked."""
        import torch

        before = [self.moments(k) for k in range(len(self.sizes))]
        old = [p.double().cpu().numpy() for p in self.params]
        gs = None if scale is None else torch.tensor([scale], device="cuda")
        mlt.adamw(self.params, grads, self.state, kw.pop("step", t), lr=kw.pop("rate", lr), betas=betas, eps=eps,
                  weight_decay=decay, copies=self.copies, grad_scale=gs, seed=seed, **kw)
        with np.errstate(over="ignore"):
            key = _mix(_mix(np.uint32(seed)) + np.uint32(t & 0xFFFFFFFF))
        lrs = lr if isinstance(lr, list) else [lr] * len(self.sizes)
        decays = decay if isinstance(decay, list) else [decay] * len(self.sizes)
        for k, (m, v) in enumerate(before):
            if grads[k] is None:
                assert np.array_equal(self.params[k].double().cpu().numpy(), old[k])
                continue
            with np.errstate(all="ignore"):
                g = grads[k].float().cpu().numpy() * F(1.0 if scale is None else scale)
                m = m * F(betas[0]) + g * F(1 - betas[0])
                v = v * F(betas[1]) + (g * g) * F(1 - betas[1])
            at, n = self.first[k] * BLOCK, self.sizes[k]
            if self.bits == 32:
                for have, want in zip(self.moments(k), (m, v)):
                    assert np.array_equal(have, want, equal_nan=True)
            else:
                for have, sc, want, w in ((self.state.m, self.state.m_scale, m, "m"), (self.state.v, self.state.v_scale, v, "v")):
                    code, scales = _encode(want, self.first[k], key, w)
                    assert np.array_equal(_bytes(have)[at:at + n], code), w
                    assert np.array_equal(sc[self.first[k]:self.first[k + 1]].cpu().numpy(), scales), w
            with np.errstate(all="ignore"):
                m, v = m.astype(np.float64), v.astype(np.float64)
                move = lrs[k] / (1 - betas[0] ** t) * m / (np.sqrt(v / (1 - betas[1] ** t)) + eps)
                want = old[k] * (1 - lrs[k] * decays[k]) - move
                err = 12 * U * np.abs(move) + 2 * U * np.abs(old[k]) + U * np.abs(want) + 2 * U * np.abs(
                    old[k] * lrs[k] * decays[k])
            for q, kind in ((self.params, self.kinds[0]), (self.copies, self.kinds[2])):
                if q is None:
                    continue
                have = q[k].double().cpu().numpy()
                assert q[k].dtype == _type(kind)
                fine = np.isfinite(want)
                assert np.array_equal(fine, np.isfinite(have))
                tol = err + UNIT[kind] * (np.abs(want) + err) + (2.0 ** -25 if kind == "f16" else 0)
                assert (np.abs(have - want)[fine] <= tol[fine]).all()


SIZES = [1, 255, 256, 257, 0, 3, 128, 5000, 4096, 70001, 12]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kinds", [("f32", "f32", None), ("f32", "bf16", "bf16"), ("bf16", "bf16", None), ("f16", "f32", None),
                                   ("f32", "f16", "f16"), ("bf16", "f32", "f32")])
def test_steps(kinds, bits):
    model = Model(SIZES, kinds, bits, seed=len(kinds[0]) + bits)
    for t in range(1, 5):
        model.step(model.grads(), t, lr=0.01, decay=0.1, seed=7)
    assert (model.state.m.float() != 0).any()
    model.step(model.grads(), 100000, lr=0.01, scale=0.37, seed=(1 << 32) - 5)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [1, 2, 3, 4, 8])
def test_alignment(offset, bits):
    for kinds in (("f32", "bf16", "f16"), ("bf16", "f32", None)):
        model = Model(SIZES, kinds, bits, offset=offset)
        for t in range(1, 3):
            model.step(model.grads(), t)


@pytest.mark.parametrize("bits", [32, 8])
def test_rates_of_their_own_missing_gradients_and_many_tensors(bits):
    rng = np.random.default_rng(3)
    sizes = [int(n) for n in rng.integers(0, 700, 1203)]  # three launches
    model = Model(sizes, ("f32", "f32", None), bits)
    lr, decay = [0.001 * (k % 7) for k in range(1203)], [0.1 * (k % 3) for k in range(1203)]
    g = model.grads()
    for k in (0, 5, 499, 500, 1202):
        g[k] = None
    keep = [t.clone() for t in model.state if t is not None]
    model.step(g, 3, lr=lr, decay=decay, betas=(0.0, 0.5), eps=0.0 if bits == 32 else 1e-8)
    for t, old in zip((t for t in model.state if t is not None), keep):
        per = 1 if t.numel() == model.first[-1] else BLOCK
        for k in (0, 5, 499, 500, 1202):
            part = slice(model.first[k] * per, model.first[k + 1] * per)
            assert (t[part].float() == old[part].float()).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_extreme_gradients(bits):
    """Zeros, subnormals, huge values, infinities and NaN, each in a block of its own and mixed."""
    import torch

    model = Model([256 * 9 + 7, 300], ("f32", "f32", None), bits)
    for t in range(1, 4):
        g = model.grads()
        a = g[0]
        a[:256] = 0.0
        a[256:512] *= 1e-36
        a[512:768] = torch.where(torch.arange(256, device="cuda") % 2 == 0, a[512:768] * 1e-18, a[512:768] * 1e15)
        a[768:1024] *= 1e18
        a[1024:1280] = 1e-45
        if t == 2:
            a[1280], a[1536 + 17], a[1800] = math.inf, math.nan, -math.inf
            a[2304:] = math.nan
        model.step(g, t)
    if bits == 8:
        m = torch.isnan(model.state.m.float())
        assert m[1280:2048].all() and not m[:1280].any() and not m[2048:2304].any()


def test_device_values_and_capture():
    """A captured step, replayed with another rate, step and gradient scale."""
    import torch

    for bits in (32, 8):
        a, b = (Model(SIZES, ("f32", "bf16", "bf16"), bits, seed=5) for _ in range(2))
        step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
        scale = torch.ones(1, device="cuda")
        g = a.grads()
        factors = [1.0 + 0.5 * (k % 2) for k in range(len(SIZES))]
        stage = [q.clone() for q in g]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            mlt.adamw(a.params, stage, a.state, step, lr=lr, weight_decay=0.1, copies=a.copies, grad_scale=scale, seed=3,
                      lr_scale=factors)
        for t in (1, 2, 50):
            step.fill_(t)
            lr.fill_(0.01 / t)
            scale.fill_(0.5 * t)
            graph.replay()
            torch.cuda.synchronize()
            rate = float(np.float32(0.01 / t))
            b.step(g, t, lr=[rate * f for f in factors], decay=0.1, scale=0.5 * t, seed=3)
            for x, y in zip(a.state, b.state):
                assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8))
            for x, y in zip(a.params + a.copies, b.params + b.copies):
                # the bias corrections are off by some 2^-23 of the step
                d = (x.float() - y.float()).abs()
                tol = 2.0 ** -8 if x.dtype == torch.bfloat16 else 2.0 ** -21
                assert (d <= tol * (y.float().abs() + 0.02 * t)).all()


def test_rounding_to_8_bits_has_no_bias():
    """A constant gradient for 300 steps: rounding to the nearest would leave v at its first values; on
    average over 65,536 elements it follows its formula.  A step's rounding error of v is at most
    2^-2 of it, so the mean's is below 300 / 65,536^0.5 / 4 = 0.3 of what one step adds if errors
    are independent; the bound allows five times as much."""
    import torch

    n = 65536
    model = Model([n], ("f32", "f32", None), 8)
    rng = np.random.default_rng(0)
    g = torch.from_numpy((0.5 + rng.random(n)).astype(F)).cuda()
    for t in range(1, 301):
        mlt.adamw(model.params, [g], model.state, t, lr=0.0, seed=11)
    m, v = model.moments(0)
    want_v = (g.double().cpu().numpy() ** 2) * (1 - 0.999 ** 300)
    one = 0.001 * (g.double() ** 2).mean().item()
    assert abs(v.mean() - want_v.mean()) <= 1.5 * one
    assert abs(m.mean() - g.mean().item()) <= 0.002  # beta1^300 is 0; a code's step is 2^-3, 65,536 of them
    assert np.corrcoef(v, want_v)[0, 1] > 0.8


def test_more_than_32_bits_of_values():
    """The second tensor's moments begin past 2^32 values; both tensors' ends get their step."""
    import torch

    n = (1 << 32) + 1000
    big, small = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(300, device="cuda")
    g, h = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.ones(300, device="cuda")
    g[-1000:] = 1.0
    state = mlt.adamw_state([big, small], 8)
    mlt.adamw([big, small], [g, h], state, 1, lr=0.5)
    # the first step of a gradient of 1 is lr, but for eps and some roundings
    assert (big[-1000:] == -0.5).all() and (big[-1256:-1000] == 0).all() and (big[:1000] == 0).all()
    assert ((small + 0.5).abs() <= 12 * U * 0.5 + 1e-8).all()
    first = -(-n // BLOCK)
    assert (state.m_scale[first:] == state.m_scale[first]).all() and state.m_scale[first] > 0
    assert (state.m[first * BLOCK:first * BLOCK + 300].float() > 0).all()


def test_another_stream_and_refusals():
    import torch

    a, b = (Model(SIZES, ("f32", "bf16", None), 8, seed=2) for _ in range(2))
    g = a.grads()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    mlt.adamw(a.params, g, a.state, 1, stream=s)
    mlt.adamw(b.params, g, b.state, 1)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.params, b.params))
    # a gradient that is not contiguous is copied
    p, q = torch.zeros(8, 6, device="cuda"), torch.zeros(8, 6, device="cuda")
    g6 = torch.arange(48.0, device="cuda").view(6, 8).t()
    mlt.adamw([p], [g6], mlt.adamw_state([p]), 1)
    mlt.adamw([q], [g6.contiguous()], mlt.adamw_state([q]), 1)
    assert torch.equal(p, q) and (p.view(-1)[1:] != 0).all()
    mlt.adamw([], [], mlt.adamw_state([]), 1)
    p, st = torch.zeros(10, device="cuda"), mlt.adamw_state([torch.zeros(10, device="cuda")])
    two = mlt.adamw_state([p, p])
    bad = [lambda: mlt.adamw([p], [], st, 1), lambda: mlt.adamw([p], [p.clone()], st, 0),
           lambda: mlt.adamw([p], [p[:5]], st, 1), lambda: mlt.adamw([p], [p.double()], st, 1),
           lambda: mlt.adamw([p], [p.cpu()], st, 1), lambda: mlt.adamw([p.double()], [p], st, 1),
           lambda: mlt.adamw([p[::2]], [p[::2]], st, 1), lambda: mlt.adamw([p], [p.clone()], two, 1),
           lambda: mlt.adamw([p, p], [p.clone()] * 2, two, 1),  # one parameter twice
           lambda: mlt.adamw([p], [p.clone()], mlt.AdamWState(st.m, st.m), 1),
           lambda: mlt.adamw([st.m[:10]], [p], st, 1),
           lambda: mlt.adamw([p], [p.clone()], st, 1, copies=[p]), lambda: mlt.adamw([p], [p.clone()], st, 1, copies=[p[:3]]),
           lambda: mlt.adamw([p], [p.clone()], st, 1, betas=(1.0, 0.9)),
           lambda: mlt.adamw([p], [p.clone()], st, 1, betas=(0.9, -0.1)), lambda: mlt.adamw([p], [p.clone()], st, 1, eps=-1.0),
           lambda: mlt.adamw([p], [p.clone()], st, 1, lr=math.inf), lambda: mlt.adamw([p], [p.clone()], st, 1, lr=[0.1, 0.2]),
           lambda: mlt.adamw([p], [p.clone()], st, 1, grad_scale=torch.ones(2, device="cuda")),
           lambda: mlt.adamw([p], [p.clone()], st, torch.ones(1, device="cuda")),
           lambda: mlt.adamw([p], [p.clone()], mlt.AdamWState(st.m, st.v, st.m[:1], None), 1),
           lambda: mlt.adamw_state([p], 16)]
    for call in bad:
        with pytest.raises((TypeError, ValueError, mlt.MltError)):
            call()
    assert (p == 0).all()
