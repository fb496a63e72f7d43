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


def sigmoid(v):
    return 0.5 * (1 + np.tanh(0.5 * v))


U = 2.0 ** -23  # an approximate operation in 32 bits: one unit in the last place


def scan(p):
    """The recurrence of one call in 64 bits, position by position, with a bound on what 32-bit
    arithmetic may add: every factor and term is off by a few units U of its magnitude, the
    exponential's argument by U of it.  p: dict of numpy arrays (None where absent); returns a
    dict with y, state, conv_state, their bounds y_tol, state_tol, and what the gradient needs."""
    f = lambda k: None if p.get(k) is None else p[k].astype(np.float64)  # noqa: E731
    x, dt, B, C, A = (f(k) for k in ("x", "dt", "B", "C", "A"))
    nb, L, d = x.shape
    n = A.shape[1]
    group = np.arange(d) // (d // B.shape[2])
    taps = 0 if p.get("conv_w") is None else p["conv_w"].shape[1]
    z, w, cb, skip, bias = f("z"), f("conv_w"), f("conv_b"), f("skip"), f("dt_bias")
    lengths = np.full(nb, L) if p.get("lengths") is None else np.clip(p["lengths"], 0, L)
    live = np.arange(L)[None] < lengths[:, None]
    x = np.where(live[..., None], x, 0)
    k1 = max(0, taps - 1)
    old = np.zeros((nb, k1, d)) if p.get("conv_state") is None else f("conv_state")
    past = np.concatenate([old, x], 1)
    if taps:
        v = sum(past[:, j:j + L] * w[:, j] for j in range(taps)) + (0 if cb is None else cb)
        vm = sum(np.abs(past[:, j:j + L] * w[:, j]) for j in range(taps)) + (0 if cb is None else np.abs(cb))
        u = v * sigmoid(v)
        um = np.abs(u) * (4 + np.abs(v)) + 1.1 * vm * (taps + 1)  # units of U; silu's slope is at most 1.1
    else:
        v, u, um = x, x, 0 * x
    raw = np.where(live[..., None], dt, 0) + (0 if bias is None else bias)
    step = np.logaddexp(0, raw)
    stepm = step * (8 + np.abs(raw))  # units
    h = np.zeros((nb, d, n)) if p.get("state") is None else f("state")
    mag, err = np.abs(h), np.zeros_like(h)
    hs, y, tol = [h], np.zeros((nb, L, d)), np.zeros((nb, L, d))
    for t in range(L):
        on = live[:, t][:, None, None]
        arg = step[:, t][..., None] * A
        a = np.exp(arg)
        Bt, Ct = np.where(on, B[:, t], 0)[:, group], np.where(on, C[:, t], 0)[:, group]
        push = (step[:, t] * u[:, t])[..., None] * Bt
        pm = np.abs(push) * 4 + (stepm[:, t] * np.abs(u[:, t]) + step[:, t] * um[:, t])[..., None] * np.abs(Bt)
        am = a * (4 + 2 * np.abs(arg) + np.abs(A) * stepm[:, t][..., None])
        h2 = np.where(on, a * h + push, h)
        err = np.where(on, a * err + U * (am * mag + pm), err)
        mag = np.where(on, a * mag + np.abs(push), mag)
        h = h2
        hs.append(h)
        su = (0 if skip is None else skip) * u[:, t]
        y[:, t] = (h * Ct).sum(-1) + su
        tol[:, t] = (np.abs(Ct) * (err + U * (n + 4) * mag)).sum(-1) + U * (
            np.abs(su) * 4 + (0 if skip is None else np.abs(skip)) * um[:, t])
    core, gate = y, 1.0
    if z is not None:
        zz = np.where(live[..., None], z, 0)
        gate = zz * sigmoid(zz)
        tol = tol * np.abs(gate) + U * np.abs(y * gate) * (6 + np.abs(zz))
    y = np.where(live[..., None], y * gate, 0)
    idx = lengths[:, None] + np.arange(k1)
    conv = np.take_along_axis(past, np.broadcast_to(idx[..., None], (nb, k1, d)), 1) if k1 else None
    return dict(y=y, y_tol=np.where(live[..., None], tol, 0), state=h, state_tol=err + U * 4 * mag, conv_state=conv,
                hs=hs, u=u, v=v, step=step, raw=raw, past=past, core=core, live=live, group=group, taps=taps)
