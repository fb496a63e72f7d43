"""The sequence operators together: a proposer over knob digits trains, proposes and feeds the
annealing step."""
import math

import numpy as np
import pytest

from paper_2411_10764_gb300 import mlt
from paper_2411_10764_gb300 import workloads as W
from paper_2411_10764_gb300.proposer import TAPS, Proposer, explore

pytestmark = pytest.mark.gpu


def _plain_loss(model, p, index):
    """The model in elementary 64-bit operations, differentiable."""
    import torch

    tokens = model.tokens_of(index).cpu()
    inp, i, n = tokens[:, :-1], model.inner, model.states
    e = p["table"][inp] * math.sqrt(model.dim)
    proj = e @ p["w_in"]
    x, z, dt, B, C = (proj[..., :i], proj[..., i:2 * i], proj[..., 2 * i:3 * i], proj[..., 3 * i:3 * i + n],
                      proj[..., 3 * i + n:])
    m, L = inp.shape
    past = torch.cat([torch.zeros(m, TAPS - 1, i, dtype=torch.float64), x], 1)
    v = sum(past[:, j:j + L] * p["conv_w"][:, j] for j in range(TAPS)) + p["conv_b"]
    u = v * torch.sigmoid(v)
    d = torch.nn.functional.softplus(dt + p["dt_bias"])
    h, ys = torch.zeros(m, i, n, dtype=torch.float64), []
    for t in range(L):
        h = torch.exp(d[:, t, :, None] * p["A"]) * h + (d[:, t] * u[:, t])[..., None] * B[:, t, None]
        ys.append((h * C[:, t, None]).sum(-1) + p["skip"] * u[:, t])
    y = torch.stack(ys, 1) * z * torch.sigmoid(z)
    scores = (e + y @ p["w_out"]) @ p["head"]
    loss = 0.0
    for j in range(L):
        a, b = model.offsets[j], model.offsets[j + 1]
        loss = loss - scores[:, j, a:b].log_softmax(-1)[torch.arange(m), tokens[:, j + 1] - a].mean() / L
    return loss


def test_gradients_of_the_whole_model():
    """Against the same model in 64 bits.  Products of at most 160 terms in fp32 and some thirty
    operations in a row: 1e-4 of the largest entry is a hundred times their rounding."""
    import torch

    torch.backends.cuda.matmul.allow_tf32 = False
    model = Proposer([4, 7, 3, 8, 2], dim=24, inner=40, states=13, seed=3)
    index = torch.randint(0, 4 * 7 * 3 * 8 * 2, (50,), device="cuda")
    loss, grads = model.loss_and_grads(index)
    p = {k: v.double().cpu().requires_grad_() for k, v in model.params.items()}
    want = _plain_loss(model, p, index)
    want.backward()
    assert abs(loss.item() - want.item()) <= 1e-5 * abs(want.item())
    assert set(grads) == set(p)
    for k, g in grads.items():
        w = p[k].grad
        assert (g.double().cpu() - w).abs().max() <= 1e-4 * w.abs().max(), k


def test_single_tokens_equal_the_sequence():
    import torch

    model = Proposer([5, 6, 7], dim=32, inner=48, states=16, seed=1)
    tokens = model.tokens_of(torch.randint(0, 210, (9,), device="cuda"))
    whole = model.forward(tokens)[0]
    state = torch.zeros((9, 48, 16), device="cuda")
    conv = torch.zeros((9, TAPS - 1, 48), device="cuda")
    for t in range(4):
        one = model.forward(tokens[:, t:t + 1].contiguous(), state, conv, in_place=True)[0]
        assert torch.allclose(one[:, 0], whole[:, t], rtol=1e-4, atol=1e-4)


def test_training_raises_the_likelihood_and_proposals_follow():
    import torch

    radices = [8, 8, 8]
    model = Proposer(radices, dim=32, inner=48, states=16, seed=2)
    good = torch.tensor([3 + 8 * 5 + 64 * 1, 3 + 8 * 5 + 64 * 2, 7 + 8 * 0 + 64 * 6], device="cuda").repeat(20)
    losses = model.train(good, steps=60)
    assert losses[-1] < 0.5 * losses[0]
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    index, logp = model.propose(500, g, temperature=0.5)
    assert ((index >= 0) & (index < 512)).all() and (logp <= 0).all()
    assert torch.isin(index, good).float().mean() > 0.5


def test_a_round_of_exploration():
    import torch

    w = W.make_workload(4, seed=1, n=20000)
    mlt.load_workload_models(w)
    out = explore(w.decoder, w.thr, 100, 20000, keep=64, chains=300, steps=10)
    perf = out["perf"]
    assert out["drawn"].numel() == 64 and out["drawn"].unique().numel() == 64
    assert torch.isfinite(perf[out["drawn"]]).all()  # none that V rejects
    space = int(np.prod(w.decoder.radices.astype(np.int64)))
    assert ((out["next"] >= 0) & (out["next"] < space)).all()
    assert out["losses"][-1] < out["losses"][0]
    ok = out["accepted"].bool()
    assert ok.any() and torch.isfinite(out["score"][ok]).all()
