"""What Proposer.search and explore refuse, before any work on a GPU."""
import types

import pytest

from paper_2411_10764_gb300 import proposer
from paper_2411_10764_gb300.proposer import Proposer


@pytest.mark.parametrize("radices,m,beams", [([8, 8], 1025, None), ([8, 9], 1024, None), ([16, 4], 5, 513), ([4], 0, None),
                                             ([4], -3, None), ([9000], 8, 91), ([5, 9], 1, 2000)])
def test_search_refuses(radices, m, beams):
    with pytest.raises(ValueError, match="beams"):
        Proposer(radices, dim=8, inner=8, device="cpu").search(m, beams)


@pytest.mark.parametrize("radices,beams", [([8, 9], 1024), ([8, 8], -1), ([16], 513), ([8], 1025)])
def test_explore_refuses_first(radices, beams, monkeypatch):
    monkeypatch.setattr(proposer.mlt, "screen_decoded", lambda *a: pytest.fail("screened"))
    with pytest.raises(ValueError, match="beams"):
        proposer.explore(types.SimpleNamespace(radices=radices, option_values=None, program=None), 0.5, 0, 100, chains=4096,
                         beams=beams)


@pytest.mark.parametrize("radices,most", [([8, 8], 1024), ([9, 2], 910), ([16], 512), ([90], 91), ([91], 90), ([9000, 2], 90), ([1], 1024)])
def test_most_beams(radices, most):
    assert proposer.most_beams(radices) == most
