"""Far losses, rows outside all sequences, and masked tokens that count: what the
objectives' other tests compare only in part."""
import math

import pytest
import torch

import paper_2510_26709_amd as arc
from test_gpu_objectives import (LOGITS, check_policy_grad, pair_formulas, policy_formulas,
                                 policy_inputs)
from test_gpu_tokens import formulas, near, place

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


# of 60 rows, and a hundred times that, where sequences are taken in parts: each row's
# sequence, -1 for none
@pytest.mark.parametrize("times", [1, 100])
@pytest.mark.parametrize("offsets,runs", [
    ([20, 20, 30, 30, 40], [(20, 30), (30, 40)]), ([70, 80, 90, 100, 110], []),
    ([-9, -8, -7, -6, -5], []), ([60, 60, 60, 60, 60], []), ([0, 0, 0, 0, 0], []),
    ([10, 2**40, 2**41, 2**42, 2**43], [(10, 60)]), ([-2**40, 7, 8, 9, 50], [(0, 50)])])
def test_rows_outside_all_sequences_have_no_gradient(offsets, runs, times):
    T = 60 * times
    gen = torch.Generator().manual_seed(3)
    l = -torch.rand(T, generator=gen).cuda()
    y = torch.zeros(T, dtype=torch.int64).cuda()
    o = torch.tensor([v * times if abs(v) < 2**30 else v for v in offsets]).cuda()
    buf = torch.full((T + 200,), 7.0, device="cuda")
    head = arc.TokenLogProbs(V=10, rows=T, dtype="f32")
    cfg = arc.arc_preference_config(0, 0, 0.1, 0.0, 0.0, 1.0)
    totals = torch.zeros(3).cuda()
    arc.arc_tokens_preference_terms(head.ctx, cfg, T, l, y, 2, o, None, None, None, None, totals,
                                    buf[100:100 + T])
    got = buf.cpu()
    assert bool((got[:100] == 7.0).all()) and bool((got[100 + T:] == 7.0).all())
    inside = torch.zeros(T, dtype=torch.bool)
    for first, last in runs:
        inside[first * times:last * times] = True
    d = got[100:100 + T]
    assert bool((d[~inside] == 0).all())
    want = pair_formulas(l, y, torch.tensor(offsets).mul(times).clamp(0, T))["d_logp"]
    near("d_logp", d, *want)


WITH_MASKS = [c for c in LOGITS if c[1] > 7]


@pytest.mark.parametrize("entropy", [0.0, 0.05])
@pytest.mark.parametrize("T,V,dtype,pad", WITH_MASKS)
def test_masked_tokens_that_count(T, V, dtype, pad, entropy):
    """Every row's given token is masked and has a weight.  Its ratio is 0 (1 without old
    log probabilities) and without a KL term all is finite."""
    gen = torch.Generator().manual_seed(V)
    x = place(torch.randn(T, V, generator=gen) * 2, dtype, pad)
    y = torch.randint(0, V, (T,), generator=gen)
    other = (y + 1 + torch.randint(0, V - 1, (T,), generator=gen)) % V  # masked, and not given
    rows = torch.arange(T)
    x[rows.cuda(), y.cuda()] = -INF
    x[rows.cuda(), other.cuda()] = -INF
    want = formulas(x, y, 1.0, 0)
    s = policy_inputs(T, V, torch.full((T,), -1.0, dtype=torch.float64))
    w = 0.25 + s["w"]
    A = torch.where(s["A"] == 0, 1.0, s["A"])
    head = arc.TokenLogProbs(V=V, rows=T, dtype=dtype)
    for kw in (dict(old_logp=s["old"]), dict()):
        kw = dict(kw, weights=w, entropy_coef=entropy)
        got = head.policy_loss(x, y.cuda(), A, **kw)
        assert bool((got.logp == -INF).all())
        assert bool((got.ratio == (0.0 if "old_logp" in kw else 1.0)).all())
        assert bool(torch.isfinite(got.totals).all())
        terms = policy_formulas(got.logp, got.entropy, y, A, **kw)
        for name in ("loss", "ratio", "kl", "totals"):
            near(name, getattr(got, name), *terms[name])
        up = (terms["d_logp"][0].float().cuda(), terms["d_entropy"][0].float().cuda(), None)
        if "old_logp" in kw:
            assert bool((terms["d_logp"][0] == 0).all())
            if not entropy:
                assert not bool(got.grad.any())
        check_policy_grad(x, y, 1.0, dtype, want, up, terms, got.grad)
    # with one, d loss / d l is -infinity, and so the row's gradient is infinite where p is
    # not 0, and 0 times infinity where it is
    got = head.policy_loss(x, y.cuda(), A, old_logp=s["old"], ref_logp=s["ref"], kl_coef=0.1,
                           weights=w, entropy_coef=entropy)
    assert bool((got.kl == INF).all()) and bool((got.loss == INF).all())
    assert got.totals[0] == INF and got.totals[2] == INF and got.totals[1] == 0.0
    g = got.grad.float().cpu()
    masked = torch.zeros(T, V, dtype=torch.bool)
    masked[rows, y] = masked[rows, other] = True
    assert bool((g[~masked] == INF).all()) and bool(torch.isnan(g[masked]).all())
