"""Probability mass of long rows: tails of many improbable entries."""
import math

import numpy as np
import pytest

import sequence as S
from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu


def _tail(n, below):
    """One entry at 0, all others `below` under it; and noise by which one of the first thousand is drawn next."""
    import torch

    x = torch.full((1, n), -below, device="cuda")
    x[0, n // 2] = 0.0
    g = torch.zeros((1, n), device="cuda")
    g[0, 700] = 3.0
    g[0, n // 2] = 100.0
    return x, g


@pytest.mark.parametrize("rows", [1, 3, 77])
@pytest.mark.parametrize("n,below", [(1 << 20, 22.0), (1 << 20, 22.3), (1 << 20, 20.7), (1 << 20, 24.0), (60_001, 21.0),
                                     (1 << 24, 24.9)])
def test_improbable_tails(n, below, rows):
    """The one entry's share is 1 / (1 + (n - 1) e^-below).  A top-p below it by a fiftieth of the tail's mass keeps it
    alone; one above it by half of the tail's mass keeps a part of the tail."""
    import torch

    x, g = _tail(n, below)
    tail = (n - 1) * math.exp(-below)
    share = 1.0 / (1.0 + tail)
    alone, part = share - tail / 50, share + tail / 2
    # the rule holds a share in 32 bits
    assert float(np.float32(alone)) < share - tail / 100 and abs(float(np.float32(part)) - part) < tail / 4
    x, g = x.expand(rows, n), g.expand(rows, n)
    i, _ = mlt.sample(x, g, top_p=alone, m=2)
    assert (i[:, 0] == n // 2).all() and (i[:, 1] == -1).all()
    i, _ = mlt.sample(x, g, top_p=part, m=2)
    assert (i[:, 0] == n // 2).all() and (i[:, 1] == 700).all()


def test_a_flat_tail_of_the_longest_row():
    """2^27 entries 22 nats below one: a mass of 0.0374 beside it."""
    import torch

    x, g = _tail(1 << 27, 22.0)
    for p, second in ((0.955, -1), (0.975, 700)):
        i, _ = mlt.sample(x, g, top_p=p, m=2)
        assert i.tolist() == [[1 << 26, second]], p


def test_random_rows_of_their_own_rules():
    """Rows whose scores span 60 nats, against 64 bits."""
    import torch

    rng = np.random.default_rng(8)
    n = 200_003
    x = torch.from_numpy((rng.standard_normal((4, n)) * 12).astype(np.float32)).cuda()
    g = torch.from_numpy(-np.log(rng.exponential(size=(4, n))).astype(np.float32)).cuda()
    for p in (0.5, 0.9, 0.999):
        i, _ = mlt.sample(x, g, top_p=p, m=7)
        for r in range(4):
            want, _ = S.sample_row(x[r].cpu().numpy(), g[r].cpu().numpy(), 1.0, 0, float(np.float32(p)), 0.0, 7)
            assert i[r].tolist() == want.tolist()
