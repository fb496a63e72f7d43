"""Beam search over finite scores of any size: large ones, and finite masks over parts of rows, whole rows and whole
shares of a row.

A normaliser is a 64-bit number, ln sum exp s, here and in the kernel: of scores near T two roundings to its
spacing, 2^-52 |T|, are added to what the terms are off by.  These: 2^-22 of each term (the approximate power), 2^-23
|s - top| (its argument), and 2^-24 of the argument's distance from a whole number where a product by log2 e is
rounded to its spacing; a pack's up to eight terms pass four roundings in 32 bits, 2^-22 of them."""
import math

import numpy as np
import pytest

from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
FMAX = 3.4028234663852886e38
SIZES = [2.0 ** 24, 2.0 ** 28 + 64, 1e9, float(np.nextafter(np.float32(2.0 ** 30), np.float32(0))), 2.0 ** 30, 1.5e9, 3e9,
         2.0 ** 32, 5e9, 1e10, 1e20, 1e30, 9e36, 1.1e37, 1e38, FMAX]
# all scores are candidates; two lists of the rows' (few candidates, then many)
PATHS = {"all": (6, 700, 5), "few": (6, 50021, 2), "lists": (6, 50021, 8), "short lists": (60, 3001, 9)}


def _ranked(x, logp, m):
    """One item: (total, tolerance, beam, token), best first, m + 1 of them."""
    got = []
    for w in range(len(logp)):
        s = x[w].astype(np.float64)
        ok = np.flatnonzero(s > -np.inf)
        if ok.size == 0:
            continue
        s = np.clip(s[ok], -FMAX, FMAX)
        top = s.max()
        e = np.exp(s - top)
        z = top + math.log(e.sum())
        far = np.where(e > 0, top - s, 0.0)
        # a top of 2^30 and more counts exactly its equals; below, its product's spacing is 2^-23 of it at most
        part = 0.0 if abs(top) >= 2.0 ** 30 else min(2.0 ** -24 * abs(top) * 1.4427, 64.0)
        tol = 2 * 2.0 ** -22 + (e * (2.0 ** -23 * far + U * part * (far > 0))).sum() / e.sum() + 2.0 ** -52 * abs(top)
        order = np.lexsort((ok, -s))[:m + 1]
        got += [(float(logp[w]) + (s[i] - z), tol, w, -s[i], int(ok[i])) for i in order]
    got.sort(key=lambda c: (-c[0], c[2], c[3], c[4]))
    return got[:m + 1]


def _check(x, logp, m, got):
    parent, token, out, ended = (t.cpu().numpy() for t in got)
    rows, lp = x.float().cpu().numpy(), logp.cpu().numpy()
    assert not np.isnan(out).any() and not ended.any()
    for b in range(len(rows)):
        want = _ranked(rows[b], lp[b], m)
        have = min(m, len(want))
        assert (parent[b, have:] == -1).all() and (out[b, have:] == -np.inf).all()
        for j in range(have):
            total = want[j][0]
            tol = 2 * max(c[1] for c in want[max(0, j - 1):j + 2]) + 2.0 ** -50 * abs(total)
            # below the lowest float by half a step and more a total is -infinity
            lowest = total <= -(FMAX + 2.0 ** 103)
            assert out[b, j] == -np.inf if lowest else abs(out[b, j] - total) <= tol + U * abs(total), (b, j)
            near = [(c[2], c[4]) for c in want if abs(c[0] - total) <= tol]
            assert (parent[b, j], token[b, j]) in near, (b, j)
        assert len(set(zip(parent[b, :have].tolist(), token[b, :have].tolist()))) == have


def _ordinary(rng, beams, n, kind):
    import torch

    x = torch.from_numpy((rng.standard_normal((1, beams, n)) * 2.5).astype(np.float32)).cuda()
    logp = torch.from_numpy((-5 - 3 * rng.random((1, beams))).astype(np.float32)).cuda()
    return x.to({"f32": torch.float32, "bf16": torch.bfloat16}[kind]), logp


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("sign", [1, -1])
def test_rows_and_masks_of_one_size(path, kind, sign):
    """Beam 0 is ordinary; of the others one is all of a score, one has it in some places, one but in some
    places, one but in a window of 300 adjacent ones, one holds the score and several parts of it."""
    beams, n, m = PATHS[path]
    rng = np.random.default_rng(n + m)
    for size in SIZES:
        x, logp = _ordinary(rng, beams, n, kind)
        v = sign * size
        x[0, 1] = v
        x[0, 2, 7::max(1, n // 5)] = v
        some = x[0, 3, 5::n // 3].clone()
        x[0, 3] = v
        x[0, 3, 5::n // 3] = some
        at = n // 2
        window = x[0, 4, at:at + 300].clone()
        x[0, 4] = v
        x[0, 4, at:at + 300] = window
        x[0, 5] = v * 0.5
        x[0, 5, 11], x[0, 5, n - 2], x[0, 5, n // 3] = v, v * 0.99, v * 0.75
        _check(x, logp, m, mlt.beam_step(x, logp, m))


@pytest.mark.parametrize("value", [-5e9, -1e10, -1e20, -1e30, -9e36, -FMAX])
@pytest.mark.parametrize("first", [0, 3131, 25000, 49721])
def test_a_masked_vocabulary_keeps_its_beams(value, first):
    """300 adjacent tokens allowed of 50,021: what a finite mask leaves is what -infinity leaves, to the bit."""
    import torch

    rng = np.random.default_rng(first)
    for batch, beams, m in ((1, 4, 8), (1, 1, 1), (3, 8, 8), (1, 64, 128)):
        x = torch.full((batch, beams, 50021), value, device="cuda")
        x[:, :, first:first + 300] = torch.from_numpy(rng.standard_normal((batch, beams, 300)).astype(np.float32)).cuda()
        logp = torch.from_numpy((-5 - rng.random((batch, beams))).astype(np.float32)).cuda()
        want = mlt.beam_step(torch.where(x == value, -math.inf, x), logp, m)
        assert (want[0] >= 0).all()
        got = mlt.beam_step(x, logp, m)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("n", [9, 700, 9000, 50021])
def test_one_score_of_any_size(n):
    """A beam's only continuation has the beam's own log-probability exactly; equal beams tie."""
    import torch

    for size in SIZES:
        for v in (size, -size):
            x = torch.full((1, 4, n), -math.inf, device="cuda")
            x[0, :, n // 2] = v
            logp = torch.full((1, 4), -11.3, device="cuda")
            parent, token, out, _ = mlt.beam_step(x, logp, 4)
            assert (out == logp).all() and parent[0].tolist() == [0, 1, 2, 3] and (token == n // 2).all()
