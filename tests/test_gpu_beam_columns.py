"""mlt_beam_reorder over states that are columns of one buffer."""
import pytest

from paper_2411_10764_gb300 import mlt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,beams", [(1, 2), (3, 5), (2, 300)])
@pytest.mark.parametrize("cuts", [(0, 16, 50), (0, 1, 2, 33, 50), (3, 17, 17, 40)])
def test_columns_of_one_buffer(batch, beams, cuts):
    import torch

    g = torch.Generator("cuda").manual_seed(beams)
    buf = torch.randint(0, 1 << 40, (batch * beams, 50), device="cuda", generator=g)
    parent = torch.randint(-1, beams, (batch, beams), device="cuda", generator=g)
    place = torch.arange(batch * beams, device="cuda").view(batch, beams)
    source = torch.where(parent < 0, place, place[:, :1] + parent).view(-1)
    want = buf.clone()
    want[:, cuts[0]:cuts[-1]] = buf[source, cuts[0]:cuts[-1]]
    states = [buf[:, a:b] for a, b in zip(cuts, cuts[1:])]
    mlt.beam_reorder(parent, *states[::-1])
    assert torch.equal(buf, want)
    for bad in ((buf[:, :10], buf[:, 9:20]), (buf[:, 4:9], buf), (buf[:, :3], buf[:, 40:41], buf[:, 2:3])):
        with pytest.raises(mlt.MltError, match="overlap"):
            mlt.beam_reorder(parent, *bad)
    assert torch.equal(buf, want)
