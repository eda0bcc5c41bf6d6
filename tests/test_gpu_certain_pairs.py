"""Pairs whose preferred answer is certain: a rejected answer with a masked token has
the reward -infinity, z is +infinity, and a sigmoid loss whose coefficient there is 0
is 0, in its pair and in the batch's total."""
import math

import pytest
import torch

import paper_2510_26709_amd as arc

pytestmark = pytest.mark.gpu
INF = math.inf
EPS = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def answers(length, seed=1):
    """Two pairs of sequences of `length` tokens; the first pair's rejected one has a
    masked token."""
    gen = torch.Generator().manual_seed(seed)
    l = (-3 * torch.rand(4 * length, generator=gen)).cuda()
    masked = l.clone()
    masked[2 * length + length // 2] = -INF
    y = torch.zeros(4 * length, dtype=torch.int64).cuda()
    return l, masked, y, (torch.arange(5) * length).cuda()


# 1 and 700 tokens: a workgroup for each pair; 1500 and 5000: parts of sequences
@pytest.mark.parametrize("average", [False, True])
@pytest.mark.parametrize("length", [1, 700, 1500, 5000])
def test_certain_without_smoothing(length, average):
    l, masked, y, o = answers(length)
    head = arc.TokenLogProbs(V=10, rows=4 * length, dtype="f32")
    kw = dict(beta=0.25, average=average, weights=torch.tensor([0.5, 2.0]).cuda())
    clean = head.preference(l, y, o, **kw)
    got = head.preference(masked, y, o, **kw)
    assert got.loss[0] == 0.0 and got.rewards[2] == -INF
    # the other pair as it is without the mask, alone in the total of the losses
    assert got.loss[1] == clean.loss[1]
    s = masked.double().view(4, length).cpu()
    h = (s.mean(1) if average else s.sum(1)) * 0.25
    want = 2.0 * float(-torch.nn.functional.logsigmoid(h[1] - h[3]))
    # binary64 until the total's one rounding
    assert abs(float(got.totals[0]) - want) <= EPS * want + 1e-12 * (1 + float(h[1].abs()
                                                                            + h[3].abs()))
    assert got.totals[1] == INF
    d = got.d_logp.view(4, length)
    assert bool((d[0] == 0).all()) and bool((d[2] == 0).all())
    assert torch.equal(d[1::2], clean.d_logp.view(4, length)[1::2])
    assert float(d[1, 0]) != 0.0


@pytest.mark.parametrize("length", [3, 1500])
def test_certain_with_smoothing(length):
    """The smoothed loss takes the other answer to be right now and then, at any price."""
    l, masked, y, o = answers(length)
    head = arc.TokenLogProbs(V=10, rows=4 * length, dtype="f32")
    got = head.preference(masked, y, o, beta=0.25, smoothing=0.25)
    assert got.loss[0] == INF and got.totals[0] == INF
    d = got.d_logp.view(4, length)
    # 0.25 sigmoid(z) beta, both of which are exact here
    assert bool((d[0] == 0.0625).all()) and bool((d[2] == -0.0625).all())


def test_certainly_wrong():
    l, masked, y, o = answers(4)
    head = arc.TokenLogProbs(V=10, rows=16, dtype="f32")
    swap = torch.cat([masked[8:], masked[:8]])
    for e in (0.0, 0.25):
        got = head.preference(swap, y, o, beta=1.0, smoothing=e)
        assert got.loss[0] == INF
        d = got.d_logp.view(4, 4)
        assert bool((d[0] == e - 1).all()) and bool((d[2] == 1 - e).all())


@pytest.mark.parametrize("V,dtype", [(33, "f32"), (1001, "bf16"), (50_257, "bf16")])
def test_certain_from_logits(V, dtype):
    gen = torch.Generator().manual_seed(V)
    x = torch.randn(12, V, generator=gen).to(torch.float32 if dtype == "f32" else
                                             torch.bfloat16).cuda()
    y = torch.randint(0, V, (12,), generator=gen).cuda()
    o = torch.tensor([0, 3, 6, 9, 12]).cuda()
    head = arc.TokenLogProbs(V=V, rows=12, dtype=dtype)
    clean = head.preference_loss(x, y, o)
    x[7, y[7]] = -INF
    got = head.preference_loss(x, y, o)
    assert got.loss[0] == 0.0 and got.loss[1] == clean.loss[1]
    assert got.totals[0] == got.loss[1]  # the sum of one number and 0, rounded once
    assert bool((got.grad[0:3] == 0).all()) and bool((got.grad[6:9] == 0).all())
    assert torch.equal(got.grad[3:6], clean.grad[3:6])
    assert torch.equal(got.grad[9:], clean.grad[9:])
