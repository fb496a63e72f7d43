"""Gradients of many short sequences: sums over up to 65,535 of them.

A sum over sequences and positions is taken as off by at most 64 units of 2^-23 of the sum of
magnitudes, whatever their number (sequence.Approx.sum)."""
import pytest

from test_gpu_scan import make
from test_gpu_scan_grad import call, check, grads_in

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("b,L,d,n,taps", [(600, 1, 20, 16, 4), (513, 8, 12, 5, 3), (777, 33, 3, 20, 2), (517, 64, 4, 16, 4),
                                          (515, 65, 2, 3, 0)])
def test_hundreds_of_sequences(b, L, d, n, taps, kind):
    for ragged in (False, True):
        t = make(b, L, d, n, 1, taps, kind, ragged=ragged)
        gy, gs = grads_in(t)
        check(t, gy, gs, call(t, gy, gs), kind)


@pytest.mark.parametrize("ragged", [False, True])
def test_equal_terms_of_65535_sequences(ragged):
    """Terms of one sign and size, whose running sum in 32 bits drifts by a thousandth."""
    import torch

    t = make(65535, 1, 3, 2, 1, 4, "f32", ragged=ragged)
    for k, v in (("x", 0.1), ("dt", 0.37), ("B", 0.7), ("C", 0.3), ("z", 0.9), ("state", 0.21), ("conv_state", 0.13)):
        t[k].fill_(v)
    t["skip"].fill_(1.1)
    t["conv_w"].fill_(0.4)
    gy, gs = grads_in(t)
    gy.fill_(0.1)
    gs.fill_(0.3)
    if ragged:
        t["lengths"].fill_(1)
        t["lengths"][torch.arange(1, 65535, 7, device="cuda")] = 0
    check(t, gy, gs, call(t, gy, gs), "f32")


def test_an_infinite_term_leaves_an_infinite_sum():
    import torch

    t = make(600, 1, 3, 2, 1, 0, "f32")
    gy, gs = grads_in(t)
    del t["z"]
    gy[5, 0, 1] = float("inf")
    t["x"].abs_()
    g = call(t, gy, gs)
    assert g["skip"][1].item() == float("inf") and torch.isfinite(g["skip"][[0, 2]]).all()
