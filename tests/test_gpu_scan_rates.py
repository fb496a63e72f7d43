"""Rates of -infinity forget at once, and neither they nor NaN reach the state of a sequence
that has ended."""
import pytest

from test_gpu_scan import call
from test_gpu_scan_past_end import SHAPES, _ragged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,L,d", SHAPES)
def test_ended_sequences_keep_their_state(b, L, d):
    import torch

    t = _ragged(b, L, d)
    for rate in (float("-inf"), -3.3e38, float("nan")):
        q = dict(t, A=torch.full_like(t["A"], rate))
        _, state, _ = call(q)
        assert torch.equal(state[1::3], t["state"][1::3]), rate
        if rate != rate:
            continue
        # what is left is the last position's own push, whether or not positions follow in its tile
        for i in (0, 2):
            n = int(t["lengths"][i])
            short = {k: v[i:i + 1, :n] if k in ("x", "dt", "B", "C", "z") else
                     v[i:i + 1] if k in ("state", "conv_state") else v for k, v in q.items() if k != "lengths"}
            alone = call(short)[1]
            assert torch.isfinite(alone).all() and torch.equal(state[i], alone[0]), (rate, i)
