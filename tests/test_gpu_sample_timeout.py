"""Draws whose CTAs do not meet: nothing is drawn, the status says so, the next call is exact."""
import math

import pytest

from paper_2411_10764_gb300 import mlt
from test_gpu_sample import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,n", [(1, 1 << 20), (3, 400_003)])
@pytest.mark.parametrize("rule", [dict(), dict(top_k=50), dict(top_p=0.9, m=5), dict(min_p=0.01, m=300),
                                  dict(temperature=0.0), dict(top_k=4000, top_p=0.7, m=40)])
def test_a_wait_that_gives_up_draws_nothing(rows, n, rule):
    import torch

    x, g = _inputs(rows, n, "f32", 5)
    m = rule.get("m", 1)
    out = (torch.full((rows, m), 123456789, device="cuda"), torch.full((rows, m), 7.0, device="cuda"))
    mlt.sync_status()
    mlt.selftest_sample_timeout(20_000_000)  # 20 ms
    mlt.sample(x, g, **rule, out=out)
    with pytest.raises(mlt.MltError) as e:
        mlt.sync_status()
    assert e.value.code == -5  # MLT_ETIMEOUT
    assert (out[0] == -1).all() and (out[1] == -math.inf).all()
    mlt.sample(x, g, **rule, out=out)
    mlt.sync_status()
    _check(x, g, out, m, {k: v for k, v in rule.items() if k != "m"})


def test_short_rows_use_the_one_shot_up():
    x, g = _inputs(2, 300, "f32", 5)
    mlt.selftest_sample_timeout(20_000_000)
    _check(x, g, mlt.sample(x, g), 1, dict())
    x, g = _inputs(1, 1 << 20, "f32", 6)
    _check(x, g, mlt.sample(x, g), 1, dict())
    mlt.sync_status()


@pytest.mark.parametrize("limit", [0, 999_999, 2_000_000_001])
def test_limits(limit):
    with pytest.raises(mlt.MltError) as e:
        mlt.selftest_sample_timeout(limit)
    assert e.value.code == -1
