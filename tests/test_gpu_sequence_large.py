"""The sequence operators where element offsets pass 32 bits, and tables too large to be cleared
beside the sort."""
import numpy as np
import pytest

import sequence as S
from paper_2411_10764_gb300 import mlt
from test_gpu_scan import call, make, near

pytestmark = pytest.mark.gpu


def test_embedding_rows_past_2_31_elements():
    import torch

    vocab, dim = 2_200_001, 1024
    table = torch.empty((vocab, dim), dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([0, vocab - 1, vocab - 2, 1, vocab - 1], device="cuda")
    table[ids] = torch.randn(5, dim, device="cuda").bfloat16()
    assert torch.equal(mlt.embed(ids, table, scale=2.0), (table[ids].float() * 2).bfloat16())
    g = torch.randn(5, dim, device="cuda").bfloat16()
    table.fill_(7.0)
    out = mlt.embed_grad(ids, g, vocab, out=table)
    want = torch.stack([g[0].float(), g[1].float() + g[4].float(), g[2].float(), g[3].float()]).bfloat16()
    assert torch.equal(out[torch.tensor([0, vocab - 1, vocab - 2, 1], device="cuda")], want)
    named = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    named[ids] = True
    for a in range(0, vocab, 1 << 18):
        part = out[a:a + (1 << 18)]
        assert (part[~named[a:a + (1 << 18)]] == 0).all()


@pytest.mark.parametrize("tokens", [3000, 70000])
def test_gradient_of_a_table_over_160_mb(tokens):
    """Rows are flagged in the sort and the others cleared: against an fp64 sum on the GPU."""
    import torch

    vocab, dim = 330001, 131
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    ids = torch.randint(0, vocab, (tokens,), device="cuda", generator=g)
    ids[::7] = ids[3]
    grad = torch.randn(tokens, dim, device="cuda", generator=g)
    out = torch.full((vocab, dim), float("nan"), device="cuda")
    mlt.embed_grad(ids, grad, vocab, scale=0.5, out=out)
    want = torch.zeros((vocab, dim), dtype=torch.float64, device="cuda").index_add_(0, ids, grad.double()) * 0.5
    mag = torch.zeros((vocab, dim), dtype=torch.float64, device="cuda").index_add_(0, ids, grad.double().abs()) * 0.5
    most = int(torch.bincount(ids, minlength=vocab).max())
    assert ((out.double() - want).abs() <= mag * (most + 2) * 2.0 ** -24).all()


def test_sampled_rows_past_2_31_scores():
    import torch

    rows, n = 20, 1 << 27
    x = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
    noise = torch.zeros((1, n), device="cuda").expand(rows, n)
    best = torch.tensor([n - 1 - 977 * r for r in range(rows)], device="cuda")
    x.scatter_(1, best[:, None], 9.0)
    noise2 = torch.zeros((2, n), device="cuda")
    i, lp = mlt.sample(x[18:], noise2, temperature=0.0)
    assert i[:, 0].tolist() == best[18:].tolist()
    i, lp = mlt.sample(x[18:], noise2, top_k=3, m=3)  # the best, then the first two of equal ones
    assert i.tolist() == [[int(b), 0, 1] for b in best[18:]]
    with pytest.raises(ValueError):
        mlt.sample(x, noise.t())
    del noise2
    full = torch.zeros((rows, n), device="cuda")
    i, _ = mlt.sample(x, full, min_p=0.5)
    assert i[:, 0].tolist() == best.tolist()


def test_scan_positions_past_2_31_elements():
    """The end of a long sequence equals that of a short one from the state in between."""
    import torch

    b, L, d, n = 1, 1_100_000, 2048, 4
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    one = r(1, 1, d).bfloat16()
    x = torch.empty((b, L, d), dtype=torch.bfloat16, device="cuda")
    for a in range(0, L, 100_000):
        x[:, a:a + 100_000] = r(b, 100_000, d).bfloat16()
    t = dict(x=x, dt=one.expand(b, L, d), B=r(1, 1, 1, n).bfloat16().expand(b, L, 1, n),
             C=r(1, 1, 1, n).bfloat16().expand(b, L, 1, n), A=-torch.ones(d, n, device="cuda"),
             conv_w=r(d, 4))
    y, s, c = call(t)
    at = L - 64
    h = dict(t, **{k: t[k][:, :at] for k in ("x", "dt", "B", "C")})
    _, s1, c1 = call(h)
    tail = {k: (t[k][:, at:].contiguous() if k in ("x", "dt", "B", "C") else t[k]) for k in t}
    tail.update(state=s1, conv_state=c1)
    ref = S.scan({k: (v.float() if v.is_floating_point() else v).cpu().numpy() for k, v in tail.items()})
    near(y[:, at:], ref["y"], "bf16")
    near(s, ref["state"], "f32")
    assert np.array_equal(c.float().cpu().numpy(), x[:, -3:].float().cpu().numpy())
