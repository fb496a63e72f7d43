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
