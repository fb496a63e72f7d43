"""Plain 64-bit implementations of the sequence-model operators, for tests."""
import math

import numpy as np

FMAX = np.float32(3.4028234663852886e38)


def sample_row(x, noise, temperature, top_k, top_p, min_p, m):
    """(indices, log-probabilities) of one row; x and noise float32 arrays.

    The scaled score and its sum with the noise are defined as 32-bit
    operations; the cuts are taken in 64 bits."""
    n = x.size
    index, logp = np.full(m, -1, np.int64), np.full(m, -np.inf)
    with np.errstate(all="ignore"):
        raw = x * (np.float32(1) / np.float32(temperature if temperature > 0 else 1))
        s = np.clip(raw, -FMAX, FMAX) + np.float32(0)
        alive = np.flatnonzero(~np.isnan(raw) & (x != -np.inf))
        if alive.size == 0:
            return index, logp
        order = alive[np.argsort(-s[alive].astype(np.float64), kind="stable")]
        if temperature == 0:
            index[0], logp[0] = order[0], 0.0
            return index, logp
        top = float(s[order[0]])
        total = np.exp(s[alive].astype(np.float64) - top).sum()
        if 0 < top_k < n:
            order = order[:top_k]
        w = np.exp(s[order].astype(np.float64) - top)
        if top_p < 1:
            order = order[np.maximum.accumulate(np.r_[True, (np.cumsum(w) < top_p * w.sum())[:-1]][::-1])[::-1]]
        if min_p > 0:
            order = order[s[order].astype(np.float64) - top >= min(math.log(min_p), 0.0)]
        kept = np.sort(order)
        key = s[kept] + noise[kept]
        key = np.where(np.isnan(key), -FMAX, np.clip(key, -FMAX, FMAX))
        drawn = kept[np.argsort(-key.astype(np.float64), kind="stable")[:m]]
    index[:drawn.size] = drawn
    logp[:drawn.size] = s[drawn].astype(np.float64) - top - math.log(total)
    return index, logp


def embed(ids, table, scale):
    """ids any shape; rows of negative and too large ids are zero."""
    ids = np.asarray(ids)
    ok = (ids >= 0) & (ids < table.shape[0])
    out = table[np.where(ok, ids, 0)].astype(np.float64) * float(np.float32(scale))
    out[~ok] = 0
    return out


def embed_grad(ids, grad, vocab, scale):
    """(gradient, sum of magnitudes) of the table."""
    out, mag = np.zeros((vocab, grad.shape[1])), np.zeros((vocab, grad.shape[1]))
    ok = (ids >= 0) & (ids < vocab)
    np.add.at(out, ids[ok], grad[ok].astype(np.float64))
    np.add.at(mag, ids[ok], np.abs(grad[ok]).astype(np.float64))
    c = float(np.float32(scale))
    return out * c, mag * abs(c)


U = 2.0 ** -23  # an operation in 32 bits is off by at most half of U, an approximate one by a few


class Approx:
    """A 64-bit value with a bound on how far a 32-bit evaluation of the same formula may be off."""

    def __init__(self, v, e=None):
        self.v = np.asarray(v, np.float64)
        self.e = np.zeros_like(self.v) if e is None else e

    def __add__(self, o):
        o = o if isinstance(o, Approx) else Approx(o)
        v = self.v + o.v
        return Approx(v, self.e + o.e + U * np.abs(v))

    def __mul__(self, o):
        o = o if isinstance(o, Approx) else Approx(o)
        v = self.v * o.v
        return Approx(v, np.abs(self.v) * o.e + np.abs(o.v) * self.e + self.e * o.e + U * np.abs(v))

    def __getitem__(self, i):
        return Approx(self.v[i], self.e[i])

    def exp(self):  # 2^(x log2 e): the argument is off by U of itself, the power by a few U
        v = np.exp(self.v)
        return Approx(v, v * np.expm1(self.e + U * (4 + 2 * np.abs(self.v))))

    def sigmoid(self):  # slope at most a quarter and at most the value
        v = 0.5 * (1 + np.tanh(0.5 * self.v))
        return Approx(v, np.minimum(0.25, v) * (self.e + 2 * U * np.abs(self.v)) + 6 * U * v)

    def softplus(self):  # slope sigmoid(x) <= the value where x < 0
        v = np.logaddexp(0, self.v)
        return Approx(v, np.minimum(1.0, v) * (self.e + 2 * U * np.abs(self.v)) + 8 * U * v)

    def sum(self, axis):
        n = np.prod([self.v.shape[i] for i in np.atleast_1d(axis)])
        return Approx(self.v.sum(axis), self.e.sum(axis) + U * min(n, 64) * np.abs(self.v).sum(axis))

    def where(self, on):
        return Approx(np.where(on, self.v, 0), np.where(on, self.e, 0))

    def pick(self, on, other):
        return Approx(np.where(on, self.v, other.v), np.where(on, self.e, other.e))


def _cat(parts, axis):
    return Approx(np.concatenate([p.v for p in parts], axis), np.concatenate([p.e for p in parts], axis))


def scan(p, gy=None, g_state=None):
    """One call, position by position, as Approx values: y, state, conv_state; with gy also the
    gradients of every input, by the chain rule on the recurrence.  p: numpy arrays by name
    (absent ones missing)."""
    f = lambda k: Approx(p[k]) if p.get(k) is not None else None  # noqa: E731
    x, dt, B, C, A = (f(k) for k in ("x", "dt", "B", "C", "A"))
    nb, L, d = x.v.shape
    n, gr = A.v.shape[1], B.v.shape[2]
    group = np.arange(d) // (d // gr)
    taps = 0 if p.get("conv_w") is None else p["conv_w"].shape[1]
    z, w, skip, bias, cb = f("z"), f("conv_w"), f("skip"), f("dt_bias"), f("conv_b")
    lengths = np.full(nb, L) if p.get("lengths") is None else np.clip(p["lengths"], 0, L)
    live = (np.arange(L)[None] < lengths[:, None])[..., None]
    x, dt, B, C = x.where(live), dt.where(live), B.where(live[..., None]), C.where(live[..., None])
    k1 = max(0, taps - 1)
    old = Approx(np.zeros((nb, k1, d))) if p.get("conv_state") is None else f("conv_state")
    past = _cat([old, x], 1)
    if taps:
        v = Approx(np.zeros((nb, L, d))) if cb is None else cb + np.zeros((nb, L, d))
        for j in range(taps):
            v = v + past[:, j:j + L] * w[:, j]
        sv = v.sigmoid()
        u = v * sv
    else:
        u = x
    raw = dt if bias is None else dt + bias
    step, u = raw.softplus().where(live), u.where(live)
    push = step * u
    sk = skip if skip is not None else Approx(np.zeros(d))
    h = f("state") or Approx(np.zeros((nb, d, n)))
    hs, decay, core = [h], [], []
    for t in range(L):
        on = live[:, t][..., None]
        a = (step[:, t][..., None] * A).exp()
        new = a * h + push[:, t][..., None] * B[:, t][:, group]
        h = new.pick(on, h)
        core.append((h * C[:, t][:, group]).sum(-1) + sk * u[:, t])
        hs.append(h)
        decay.append(a)
    stack = lambda q: Approx(np.stack([i.v for i in q], 1), np.stack([i.e for i in q], 1))  # noqa: E731
    core = stack(core) if L else Approx(np.zeros((nb, 0, d)))
    out = {}
    if z is not None:
        z = z.where(live)
        sz = z.sigmoid()
        gate = z * sz
    else:
        gate = Approx(np.ones((nb, L, d)))
    out["y"] = (core * gate).where(live)
    out["state"] = h
    if k1:
        at = np.broadcast_to((lengths[:, None] + np.arange(k1))[..., None], (nb, k1, d))
        out["conv_state"] = Approx(np.take_along_axis(past.v, at, 1))
    if gy is None:
        return out
    go = Approx(gy).where(live)
    gc = go * gate
    g = Approx(np.zeros((nb, d, n)) if g_state is None else g_state)
    G = {}
    if z is not None:
        G["z"] = go * core * sz * (z * (sz * -1.0 + 1.0) + 1.0)
    gB, gC, gp, ga = [None] * L, [None] * L, [None] * L, [None] * L
    gA = Approx(np.zeros((nb, d, n)))
    per = (nb, gr, d // gr, n)
    shape = lambda q, s: Approx(q.v.reshape(s), q.e.reshape(s))  # noqa: E731
    for t in range(L - 1, -1, -1):
        on = live[:, t][..., None]
        gt = g + gc[:, t][..., None] * C[:, t][:, group]
        gC[t] = shape(gc[:, t][..., None] * hs[t + 1], per).sum(2)
        gB[t] = shape(gt * push[:, t][..., None], per).sum(2)
        gp[t] = (gt * B[:, t][:, group]).sum(-1)
        r = gt * decay[t]
        e = r * hs[t]
        ga[t] = (e * A).sum(-1)
        gA = (gA + e * step[:, t][..., None]).pick(on, gA)
        g = r.pick(on, g)
    gp, ga = stack(gp), stack(ga)
    G.update(state=g, A=gA.sum(0), B=stack(gB).where(live[..., None]), C=stack(gC).where(live[..., None]))
    if skip is not None:
        G["skip"] = (gc * u).sum((0, 1))
    graw = ((gp * u + ga) * raw.sigmoid()).where(live)
    G["dt"] = graw
    if bias is not None:
        G["dt_bias"] = graw.sum((0, 1))
    gu = (gp * step + gc * sk).where(live)
    if not taps:
        G["x"] = gu
    else:
        gv = gu * sv * (v * (sv * -1.0 + 1.0) + 1.0)
        gpast = Approx(np.zeros_like(past.v))
        cols = []
        for j in range(taps):
            part = gv * w[:, j]
            gpast = Approx(gpast.v.copy(), gpast.e.copy())
            new = gpast[:, j:j + L] + part
            gpast.v[:, j:j + L], gpast.e[:, j:j + L] = new.v, new.e
            cols.append((gv * past[:, j:j + L]).sum((0, 1)))
        G["conv_w"] = Approx(np.stack([c.v for c in cols], 1), np.stack([c.e for c in cols], 1))
        if cb is not None:
            G["conv_b"] = gv.sum((0, 1))
        if p.get("conv_state") is not None:
            G["conv_state"] = gpast[:, :k1]
        G["x"] = gpast[:, k1:].where(live)
    out["grad"] = {k: q for k, q in G.items() if p.get(k) is not None}
    return out
