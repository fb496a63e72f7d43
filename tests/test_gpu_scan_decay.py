"""Decays over many positions: their errors must not add up one way.

With no input a state is its first value times the product of exp(d_t A), against the exponential of the
64-bit sum.  A decay is off by up to two units of 2^-24, on average over steps of all sizes by at most 0.3
of one; the exponent's own error (step size 3 units, rate and product half a unit each) is one of
their sum.  The average over some ten thousand states has a hundredth of one state's scatter."""
import numpy as np
import pytest

from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
D, N = 512, 16


def _inputs(b, L, octave, seed=0):
    """Steps and rates whose product with log2 e is about -2^-octave; the expected logarithm of each state."""
    import torch

    rng = np.random.default_rng(seed + octave)
    A = -(1 + rng.random((D, N))).astype(np.float32)
    d = np.exp2(-octave + rng.uniform(-0.5, 0.5, (b, L, D))) / (1.5 * 1.4427)
    dt = np.log(np.expm1(d)).astype(np.float32)
    total = np.log1p(np.exp(dt.astype(np.float64))).sum(1)[..., None] * A.astype(np.float64)
    c = lambda v: torch.from_numpy(v).cuda()  # noqa: E731
    zero = torch.zeros((b, L, 1, N), device="cuda")
    t = dict(x=torch.zeros((b, L, D), device="cuda"), dt=c(dt), B=zero, C_=zero + 1, A=c(A),
             state=torch.ones((b, D, N), device="cuda"))
    return t, total


def _near(got, total, steps):
    off = np.log(got.double().cpu().numpy()) - total
    most = 0.3 * steps * U + 4 * U * np.abs(total).mean()
    assert abs(off.mean()) <= most, (off.mean() / U, most / U)


@pytest.mark.parametrize("octave", [2, 5, 6, 7, 9, 11])
@pytest.mark.parametrize("b", [1, 48])
def test_prompts(b, octave):
    L = min(2 << octave, 512)
    t, total = _inputs(b, L, octave)
    _near(mlt.scan(**t)[1], total, L)


@pytest.mark.parametrize("octave", [5, 7])
def test_tokens(octave):
    L = 2 << octave
    t, total = _inputs(2, L, octave)
    state = t.pop("state")
    A = t.pop("A")
    for i in range(L):
        mlt.scan(**{k: v[:, i:i + 1] for k, v in t.items()}, A=A, state=state, state_out=state)
    _near(state, total, L)


@pytest.mark.parametrize("octave", [5, 6, 7, 9])
def test_gradient_of_the_state(octave):
    import torch

    t, total = _inputs(4, 64, octave)
    g = mlt.scan_grad(torch.zeros_like(t["x"]), **t, g_state=t["state"])
    _near(g["state"], total, 64)
