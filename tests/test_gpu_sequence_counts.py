"""Counts past 32 bits are refused or mean all, never cut to their low bits."""
import pytest

from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu


def test_top_k_past_32_bits_keeps_all():
    import torch

    x = torch.arange(100.0, device="cuda")[None]
    g = torch.zeros_like(x)
    for k in (2 ** 31, 2 ** 32 + 1, 2 ** 40 + 3):
        i, _ = mlt.sample(x, g, top_k=k, m=8)
        assert i[0].tolist() == list(range(99, 91, -1)), k
    many = torch.tensor([2 ** 32 + 1, 3, -2 ** 32 + 2], device="cuda")
    i, _ = mlt.sample(x.expand(3, 100), g.expand(3, 100), rules=mlt.sample_rules(1.0, many), m=8)
    assert i[0].tolist() == i[2].tolist() == list(range(99, 91, -1)) and i[1].tolist() == [99, 98, 97] + [-1] * 5
    for k in (-1, -2 ** 31 - 5, -2 ** 32 + 2):
        i, _ = mlt.sample(x, g, top_k=k, m=8)
        assert i[0].tolist() == list(range(99, 91, -1)), k


def test_counts_past_32_bits_are_refused():
    import torch

    x = torch.zeros((1, 10), device="cuda")
    with pytest.raises(ValueError):
        mlt.sample(x, x, m=2 ** 32 + 1)
    wide = torch.empty((1, 2 ** 32 + 3), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(1, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        mlt.embed(ids, wide, out=wide)
    with pytest.raises(ValueError):
        mlt.embed_grad(ids, wide, 1, out=wide)
    x = wide[None]
    s = torch.zeros((1, 1, 1), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        mlt.scan(x, x, s, s, torch.empty((2 ** 32 + 3, 1), device="cuda"), out=x)
