"""The normaliser of long rows: a sum of up to 2^27 weights."""
import math

import pytest

from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,n", [(1, 1 << 24), (3, 9_000_001), (77, 1 << 21), (80, 1 << 24)])
@pytest.mark.parametrize("below", [1.2, 0.1, 3.7])
def test_log_probability_in_long_rows(rows, n, below):
    """Every eighth of the first entries at 0, so that every thread has the maximum, the others at -below.  A weight is
    off by at most 2 + 1.2 below units of 2^-23 (an approximate power of two of a rounded argument), a thread's compensated
    sum of sums of eight by 3 more, 20 joins of threads, warps and CTAs by 10; the logarithm by a unit of its own, the
    result by half of one."""
    import torch

    x = torch.full((1, n), -below, device="cuda")
    x[0, :1 << 20:8] = 0.0
    at_0 = 1 << 17
    below = -float(x[0, 1])
    g = torch.zeros((1, n), device="cuda")
    g[0, 5] = 50.0
    i, lp = mlt.sample(x.expand(rows, n), g.expand(rows, n), m=2)
    assert (i[:, 0] == 5).all() and (i[:, 1] == 0).all()
    logz = math.log(at_0 + (n - at_0) * math.exp(-below))
    for j, s in ((0, -below), (1, 0.0)):
        tol = 2.0 ** -23 * (15 + 1.2 * below) + 2.0 ** -23 * 1.5 * (abs(s) + logz)
        assert (lp[:, j].double() - (s - logz)).abs().max().item() <= tol
