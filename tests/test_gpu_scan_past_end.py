"""Positions past a sequence's end: y is 0 there and the state stays as it is, whatever the
state and the rates hold."""
import pytest

from test_gpu_scan import call, make

pytestmark = pytest.mark.gpu

# single tokens, one chunk, several chunks, and enough sequences for one chunk each
SHAPES = [(3, 1, 64), (3, 50, 64), (3, 900, 64), (48, 90, 512)]


def _ragged(b, L, d, **kw):
    """Every third sequence full, one empty, one that ends inside a tile."""
    import torch

    t = make(b, L, d, 16, 1, 4, **kw)
    t["lengths"] = torch.tensor([(L, 0, (L + 1) // 2)[i % 3] for i in range(b)], dtype=torch.int32, device="cuda")
    return t


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("b,L,d", SHAPES)
def test_outputs_are_zero_whatever_the_state(b, L, d, kind, gated):
    import torch

    t = _ragged(b, L, d, kind=kind)
    if not gated:
        del t["z"]
    want = call(t)
    for bad in (float("inf"), float("nan")):
        q = dict(t, state=t["state"].clone())
        q["state"][1::3] = bad
        q["state"][2::3, ::2] = bad
        y, state, conv = call(q)
        for i, n in enumerate(t["lengths"].tolist()):
            assert (y[i, n:] == 0).all(), (bad, i)
        assert torch.equal(y[0::3], want[0][0::3]) and torch.equal(state[0::3], want[1][0::3])
        assert torch.equal(torch.nan_to_num(state[1::3], 1.0, 2.0), torch.nan_to_num(q["state"][1::3], 1.0, 2.0))
        assert torch.equal(y[2::3, :, 1::2], want[0][2::3, :, 1::2]) and torch.equal(conv, want[2])
