"""Layer norm, AdamW and beam search together with the other sequence operators: a proposer with a norm is
trained with AdamW and searched with a beam."""
import math

import pytest

from paper_2411_10764_gb300 import mlt
from paper_2411_10764_gb300 import proposer
from paper_2411_10764_gb300 import workloads as W
from paper_2411_10764_gb300.proposer import TAPS, Proposer, explore

pytestmark = pytest.mark.gpu


def _plain_scores(model, p, tokens):
    """The model in elementary 64-bit operations, differentiable."""
    import torch

    i, n = model.inner, model.states
    e = p["table"][tokens] * math.sqrt(model.dim)
    proj = e @ p["w_in"]
    x, z, dt, B, C = (proj[..., :i], proj[..., i:2 * i], proj[..., 2 * i:3 * i], proj[..., 3 * i:3 * i + n],
                      proj[..., 3 * i + n:])
    m, L = tokens.shape
    past = torch.cat([torch.zeros(m, TAPS - 1, i, dtype=torch.float64), x], 1)
    v = sum(past[:, j:j + L] * p["conv_w"][:, j] for j in range(TAPS)) + p["conv_b"]
    u = v * torch.sigmoid(v)
    d = torch.nn.functional.softplus(dt + p["dt_bias"])
    h, ys = torch.zeros(m, i, n, dtype=torch.float64), []
    for t in range(L):
        h = torch.exp(d[:, t, :, None] * p["A"]) * h + (d[:, t] * u[:, t])[..., None] * B[:, t, None]
        ys.append((h * C[:, t, None]).sum(-1) + p["skip"] * u[:, t])
    o = e + (torch.stack(ys, 1) * z * torch.sigmoid(z)) @ p["w_out"]
    c = o - o.mean(-1, keepdim=True)
    o = c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-5) * p["norm_w"] + p["norm_b"]
    return o @ p["head"]


def _logp(model, p, index):
    import torch

    tokens = model.tokens_of(index.cpu()).cpu()
    scores, got = _plain_scores(model, p, tokens[:, :-1]), 0.0
    for j in range(len(model.radices)):
        a, b = model.offsets[j], model.offsets[j + 1]
        got = got + scores[:, j, a:b].log_softmax(-1)[torch.arange(len(tokens)), tokens[:, j + 1] - a]
    return got


def _wide(model, grad=False):
    return {k: v.double().cpu().requires_grad_(grad) for k, v in model.params.items()}


def test_gradients_of_the_model_with_a_norm():
    """Products of at most 160 terms in fp32 and some forty operations in a row: 1e-4 of the largest
    entry is a hundred times their rounding."""
    import torch

    torch.backends.cuda.matmul.allow_tf32 = False
    model = Proposer([4, 7, 3, 8, 2], dim=24, inner=40, states=13, seed=3, norm=True)
    model.params["norm_w"] += 0.1 * torch.randn(24, device="cuda")
    model.params["norm_b"] += 0.1 * torch.randn(24, device="cuda")
    index = torch.randint(0, 4 * 7 * 3 * 8 * 2, (50,), device="cuda")
    loss, grads = model.loss_and_grads(index)
    p = _wide(model, True)
    want = -_logp(model, p, index).mean() / 5
    want.backward()
    assert abs(loss.item() - want.item()) <= 1e-5 * abs(want.item())
    assert set(grads) == set(p)
    for k, g in grads.items():
        w = p[k].grad
        assert (g.double().cpu() - w).abs().max() <= 1e-4 * w.abs().max(), k


@pytest.mark.parametrize("bits", [32, 8])
def test_training_with_adamw_is_its_steps(bits):
    """train() does what its loop of calls does, and the whole runs."""
    import torch

    index = torch.randint(0, 8 * 9 * 10, (64,), device="cuda")
    model = Proposer([8, 9, 10], dim=32, inner=48, seed=2, norm=True)
    same = Proposer([8, 9, 10], dim=32, inner=48, seed=2, norm=True)
    losses = model.train(index, steps=3, optimizer="adamw", bits=bits)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)
    names = list(same.params)
    state = mlt.adamw_state([same.params[k] for k in names], bits)
    assert state.bits == bits
    for t in range(3):
        _, g = same.loss_and_grads(index)
        mlt.adamw([same.params[k] for k in names], [g[k] for k in names], state, t + 1,
                  lr=[0.005 * (0.1 if k in ("A", "dt_bias") else 1.0) for k in names],
                  weight_decay=[0.01 if k in ("table", "w_in", "w_out", "head") else 0.0 for k in names], seed=t)
        same.params["A"].clamp_(max=-1e-3)
    for k in names:
        assert torch.allclose(model.params[k], same.params[k], rtol=1e-4, atol=1e-6), k
    with pytest.raises(ValueError):
        model.train(index, optimizer="sgd")


@pytest.mark.parametrize("norm", [False, True])
def test_search_finds_the_most_probable_candidates(norm):
    """With a beam for every candidate, none is lost: the order is that of all log-probabilities."""
    import torch

    torch.backends.cuda.matmul.allow_tf32 = False
    model = Proposer([4, 5, 6], dim=32, inner=48, seed=4, norm=norm)
    if not norm:
        model.params.update(norm_w=torch.ones(32, device="cuda"), norm_b=torch.zeros(32, device="cuda"))
    index, logp = model.search(200, beams=200)
    assert (index[120:] == -1).all() and (logp[120:] == -math.inf).all()
    assert index[:120].unique().numel() == 120 and ((index[:120] >= 0) & (index[:120] < 120)).all()
    want = _logp(model, _wide(model), index[:120])
    assert (logp[:120].double().cpu() - want).abs().max() <= 1e-4
    assert (want[:-1] - want[1:]).min() >= -2e-4
    few, lp = model.search(7, beams=30)
    assert few.shape == (7,) and torch.allclose(lp[0], logp[0], atol=1e-4) and few[0] == index[0]


def test_a_round_with_everything():
    import torch

    w = W.make_workload(4, seed=1, n=20000)
    mlt.load_workload_models(w)
    out = explore(w.decoder, w.thr, 0, 20000, keep=64, chains=300, steps=5, beams=100, norm=True, optimizer="adamw")
    assert out["proposed"].shape == (300,) and out["proposed"][:100].unique().numel() >= 99
    assert (out["proposed"] >= 0).all() and torch.isfinite(out["score"][out["accepted"].bool()]).all()


def test_command(capsys):
    proposer.main(["--norm", "--adamw", "--beams", "64"])
    assert "annealed proposals valid" in capsys.readouterr().out


def test_search_keeps_as_many_beams_as_may_be():
    import torch

    for radices in ([9, 16, 9], [91, 3], [2, 3]):
        model = Proposer(radices, dim=16, inner=16, seed=6)
        most = proposer.most_beams(radices)
        index, logp = model.search(most)
        found, count = index[index >= 0], min(most, math.prod(radices))
        assert found.numel() == count and found.unique().numel() == count
        assert (logp[1:count] <= logp[:count - 1]).all() and (logp[count:] == -math.inf).all()
        assert torch.equal(model.search(3, 0)[0], model.search(3)[0])
