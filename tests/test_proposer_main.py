"""The proposer's command where no candidate is valid: nothing drawn, nothing to anneal to."""
import pytest

from paper_2411_10764_gb300 import mlt, proposer


@pytest.mark.parametrize("drawn,valid", [(0, 0), (0, 2), (3, 0), (3, 2)])
def test_main_prints_what_there_is(monkeypatch, capsys, drawn, valid):
    import torch

    score = torch.full((4,), -float("inf"))
    score[:valid] = torch.arange(1.0, valid + 1)
    out = dict(drawn=torch.arange(drawn), losses=[2.0, 1.0] if drawn else [], score=score, accepted=score > 0,
               perf=torch.tensor([0.5, 0.25]) if drawn else torch.full((2,), -float("inf")))
    monkeypatch.setattr(mlt, "load_workload_models", lambda w: None)
    monkeypatch.setattr(proposer, "explore", lambda *a, **k: out)
    proposer.main()
    said = capsys.readouterr().out
    assert f"drew {drawn}" in said and f"{valid} of 4 annealed proposals valid" in said
    assert ("loss 2.000 -> 1.000" in said) == (drawn > 0) and ("best score 2.0000" in said) == (valid > 0)
    assert "(screened: 0.5000)" in said if drawn else "screened: none valid" in said
