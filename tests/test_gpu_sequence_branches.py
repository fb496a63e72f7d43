"""Forms that only large or crowded inputs reach: more positions than one cluster sorts, in tiles of either size,
and a top-k whose candidates overflow a team's list."""
import numpy as np
import pytest

from paper_2411_10764_gb300 import mlt
from test_gpu_embed import _check_grad, _rand, _type
from test_gpu_sample import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [65536, 65537, 262144, 262145, 400003])
@pytest.mark.parametrize("vocab", [200, 70001, 1 << 24])
def test_gradient_of_many_positions(tokens, vocab):
    import torch

    rng = np.random.default_rng(tokens)
    ids = rng.integers(-1, vocab, tokens)
    ids[rng.random(tokens) < 0.1] = vocab - 1
    for kind, dim in (("f32", 3), ("bf16", 8)):
        if vocab * dim > 1 << 26:
            dim = 1
        grad = _rand(rng, (tokens, dim), kind)
        t = torch.from_numpy(ids).cuda()
        out = mlt.embed_grad(t, grad, vocab, scale=0.75)
        _check_grad(t, grad, vocab, 0.75, out, kind)
        assert torch.equal(out, mlt.embed_grad(t.int(), grad, vocab, scale=0.75, out_dtype=_type(kind)))
    mlt.sync_status()


@pytest.mark.parametrize("rows,n", [(1, 100_003), (1, 300_007), (5, 100_003), (40, 33_001)])
@pytest.mark.parametrize("top_k", [4, 1000])
def test_equal_scores_overflow_the_candidates(rows, n, top_k):
    import torch

    rng = np.random.default_rng(n)
    g = torch.from_numpy(-np.log(rng.exponential(size=(1, n))).astype(np.float32)).cuda().expand(rows, n)
    x = torch.full((rows, n), 0.75, device="cuda")
    x[:, ::9] = -1.0
    for more in (dict(), dict(top_p=0.5)):
        for m in (1, 20):
            rule = dict(top_k=top_k, **more)
            _check(x[:1], g[:1], tuple(v[:1] for v in mlt.sample(x, g, m=m, **rule)), m, rule)
            got = mlt.sample(x, g, m=m, **rule)
            assert (got[0] == got[0][:1]).all() and (got[1] == got[1][:1]).all()
    mlt.sync_status()
