"""Far losses of preferences, whose other test compares them only in part."""
import math

import pytest
import torch

import paper_2510_26709_amd as arc

pytestmark = pytest.mark.gpu
INF = math.inf


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_far_losses():
    """Where a sigmoid is 0 or 1 in binary32: e^-200 is 0 there, and 200 + e^-200 is 200."""
    l = torch.tensor([0.0, -200.0, 300.0, -INF, -200.0, 0.0, 0.0, 0.0]).cuda()
    y = torch.zeros(8, dtype=torch.int64).cuda()
    head = arc.TokenLogProbs(V=10, rows=8, dtype="f32")
    got = head.preference(l, y, torch.arange(9).cuda(), beta=1.0)
    assert got.loss.tolist() == [0.0, 200.0, 0.0, INF]
    assert got.rewards.tolist() == l.tolist()
    assert got.totals.tolist() == [INF, -INF, 2.0]
    assert got.d_logp.tolist() == [0.0, -1.0, 0.0, -1.0, 0.0, 1.0, 0.0, 1.0]
    keep = [0, 1, 2, 4, 5, 6]
    got = head.preference(l[keep], y[:6], torch.arange(7).cuda(), beta=1.0)
    assert got.loss.tolist() == [0.0, 200.0, 0.0] and got.totals.tolist() == [200.0, 300.0, 2.0]
