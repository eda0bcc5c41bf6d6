"""The policy and preference losses against the formulas in 64 bits: sizes from no
token up, every kernel that takes them, borders, tokens without a part, sequences
without tokens, and the gradients against differences."""
import ctypes
import math

import pytest
import torch

import paper_2510_26709_amd as arc
from paper_2510_26709_amd import _lib
from test_gpu_tokens import EPS, formulas, lse_slack, near, place, slack, tokens

pytestmark = pytest.mark.gpu
NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def f32(v):
    return ctypes.c_float(v).value


def opt(x, T):
    return torch.zeros(T, dtype=torch.float64) if x is None else x.double().cpu()


# ---------------------------------------------------------------- policy

def policy_formulas(logp, H, y, A, *, old_logp=None, ref_logp=None, weights=None, clip_low=0.2,
                    clip_high=0.2, dual=0.0, kl_coef=0.0, entropy_coef=0.0, scale=1.0, off=0.0):
    """Terms, totals and gradients in 64 bits with their tolerances; `off`: the
    absolute error [T] of the log probabilities."""
    T = y.numel()
    y, A, l, H = y.cpu(), A.double().cpu(), logp.double().cpu(), opt(H, T)
    live = y >= 0
    w = (torch.ones(T, dtype=torch.float64) if weights is None else weights.double().cpu())
    w = torch.where(live, w * f32(scale), 0.0)
    d = torch.zeros(T, dtype=torch.float64) if old_logp is None else l - old_logp.double().cpu()
    d = torch.where(live & torch.isnan(l), NAN, torch.where(live, d, 0.0))
    r = torch.exp(d)
    low, high, dual = 1.0 - f32(clip_low), 1.0 + f32(clip_high), f32(dual)
    A = torch.where(live, A, 0.0)
    held = r.clamp(low, high) * A
    plain = r * A
    clipped = plain > held
    gain = torch.where(clipped, held, plain)
    if dual:
        beyond = (A < 0) & (gain < dual * A)
        gain = torch.where(beyond, dual * A, gain)
        clipped |= beyond
    e = torch.zeros(T, dtype=torch.float64)
    if ref_logp is not None:
        e = torch.where(live, ref_logp.double().cpu() - l, 0.0)
    kl = torch.expm1(e) - e
    near_0 = e.abs() < 1e-3  # (64 bits cancel there too)
    kl = torch.where(near_0, e * e * (0.5 + e / 6 + e * e / 24), kl)
    kl = torch.where(e == INF, INF, kl)  # the exponential's
    kc, ec = f32(kl_coef), f32(entropy_coef)
    loss = -gain + (kc * kl if kc else 0.0) - (ec * H if ec else 0.0)
    loss = torch.where(live, loss, 0.0)
    g = torch.where(clipped, 0.0, -plain) - (kc * torch.expm1(e) if kc else 0.0)
    has = w != 0
    dl = torch.where(has, w * g, 0.0)
    dh = torch.where(has, -ec * w, 0.0)
    parts = [loss, r, kl, torch.where(live, H, 0.0), clipped.double()]
    totals = torch.stack([torch.where(has, w * x, 0.0).sum() for x in parts])
    # a difference of binary32 numbers, an exponential within 2 ulp, one product more
    # (an infinite difference is exact, and so is its exponential, 0 or infinity)
    rel = (d.abs().nan_to_num(posinf=0.0) * EPS + off) + 8 * EPS
    rel_e = e.abs().nan_to_num(posinf=0.0) * EPS + off
    tol_kl = torch.expm1(e).abs() * (rel_e + 4 * EPS) + 8 * EPS * kl
    tol_loss = plain.abs() * rel + (kc * tol_kl + 4 * EPS * kc * kl) + 4 * EPS * (
        gain.abs() + abs(ec) * H.abs()) + abs(ec) * off * 30
    tol_g = plain.abs() * rel + kc * ((e.exp() * rel_e) + 6 * EPS * torch.expm1(e).abs())
    tols = [tol_loss, r * rel, tol_kl, off * 30 + 0 * r, 0 * r]
    tol_totals = torch.stack([(w.abs() * t).nan_to_num().sum() + 4 * EPS * (w * x).abs()
                              .nan_to_num().sum() for t, x in zip(tols, parts)])
    far = torch.minimum((r - low).abs(), (r - high).abs())
    if dual:
        far = torch.minimum(far, (r - dual).abs())
    border = (far < r * rel * 2) & (r != low) & (r != high)
    assert not bool((live & border).any()), "inputs on a border"
    return {"loss": (loss, tol_loss + 1e-37), "ratio": (torch.where(live, r, 0.0), r * rel + 1e-37),
            "kl": (torch.where(live, kl, 0.0), tol_kl + 1e-37), "totals": (totals, tol_totals),
            "d_logp": (dl, w.abs() * tol_g + 4 * EPS * dl.abs() + 1e-37),
            "d_entropy": (dh, 4 * EPS * dh.abs())}


def policy_inputs(T, seed, logp=None):
    gen = torch.Generator().manual_seed(seed)
    rn = lambda: torch.randn(T, generator=gen, dtype=torch.float64)  # noqa: E731
    l = -torch.rand(T, generator=gen, dtype=torch.float64) * 8 if logp is None else logp
    d = rn() * torch.where(torch.rand(T, generator=gen) < 0.2, 1.0, 0.15)
    for b in (0.8, 1.2, 1.28, 3.0, 0.5):  # off the borders
        d = torch.where((d - math.log(b)).abs() < 1e-3, math.log(b) + 1e-3, d)
    y = torch.randint(0, 1000, (T,), generator=gen)
    y = torch.where(torch.rand(T, generator=gen) < 0.15, -1, y)
    s = {"logp": l.float().cuda(), "H": (torch.rand(T, generator=gen) * 3).cuda(), "y": y.cuda(),
         "A": rn().float().cuda(), "old": (l - d).float().cuda(),
         "ref": (l + 0.5 * rn()).float().cuda(), "w": torch.rand(T, generator=gen).cuda()}
    if T > 6:
        s["w"][3] = 0.0
        s["ref"][5] = s["logp"][5]
        s["A"][6] = 0.0
    return s


OPTIONS = [
    dict(old=True), dict(old=False, kl=True, kl_coef=0.1),
    dict(old=True, kl=True, kl_coef=0.05, dual=3.0, weights=True, clip_high=0.28, scale=0.25),
    dict(old=True, entropy_coef=0.01, weights=True, clip_low=0.5, scale=-2.0),
    dict(old=True, kl=True, kl_coef=0.0, clip_high=INF, clip_low=1.0, dual=0.0),
    dict(old=True, kl=True, kl_coef=1.0, entropy_coef=-0.5, dual=3.0),
]


def keywords(o, s):
    kw = {k: v for k, v in o.items() if k not in ("old", "kl", "weights")}
    return dict(kw, old_logp=s["old"] if o.get("old") else None,
                ref_logp=s["ref"] if o.get("kl") else None,
                weights=s["w"] if o.get("weights") else None)


@pytest.mark.parametrize("o", OPTIONS)
@pytest.mark.parametrize("T", [0, 1, 2, 63, 257, 1000, 4099, 262_145, 1_000_003])
def test_policy_terms(T, o):
    s = policy_inputs(T, T + 7)
    kw = keywords(o, s)
    head = arc.TokenLogProbs(V=10, rows=max(T, 1), dtype="f32")
    got = head.policy(s["logp"], s["y"], s["A"], entropy=s["H"], **kw)
    again = head.policy(s["logp"], s["y"], s["A"], entropy=s["H"], **kw)
    for a, b in zip(got, again):
        assert a is None or torch.equal(a, b), "a call repeats its bits"
    want = policy_formulas(s["logp"], s["H"], s["y"], s["A"], **kw)
    assert (got.d_entropy is None) == (not kw.get("entropy_coef"))
    for name, x in got._asdict().items():
        if x is not None:
            near(name, x, *want[name])


def test_small_differences_have_a_kl_of_their_own():
    e = torch.logspace(-8, 0.3, 500, dtype=torch.float64)
    e = torch.cat([e, -e, torch.zeros(1, dtype=torch.float64)])
    l = torch.zeros(e.numel())
    ref = e.float()
    head = arc.TokenLogProbs(V=10, rows=e.numel(), dtype="f32")
    got = head.policy(l.cuda(), torch.zeros(e.numel(), dtype=torch.int64).cuda(),
                      torch.zeros(e.numel()).cuda(), ref_logp=ref.cuda(), kl_coef=1.0)
    x = ref.double()
    # by its series where 64 bits cancel too
    want = torch.where(x.abs() < 0.01, x * x * (0.5 + x * (1 / 6 + x * (1 / 24 + x / 120))),
                       torch.expm1(x) - x)
    near("kl", got.kl, want, (8 * EPS + 1e-10) * want.abs() + torch.where(
        x.abs() >= 0.5, 4 * EPS * torch.expm1(x).abs(), 0.0) + 1e-40)


def test_policy_on_the_borders():
    """gain is ratio A on a border itself: the gradient is there."""
    T = 6
    l = torch.zeros(T).cuda()
    A = torch.tensor([1.0, -1.0, 0.0, 1.0, -1.0, 2.0]).cuda()
    y = torch.zeros(T, dtype=torch.int64).cuda()
    head = arc.TokenLogProbs(V=10, rows=T, dtype="f32")
    got = head.policy(l, y, A, clip_low=0.0, clip_high=0.0)
    assert torch.equal(got.d_logp, -A) and float(got.totals[4]) == 0.0
    assert torch.equal(got.ratio, torch.ones(T).cuda())
    # the bound for negative advantages, at ratio e
    got = head.policy(l, y, A, old_logp=l - 1.0, dual=1.0, clip_low=0.2, clip_high=0.2)
    assert torch.equal(got.d_logp, torch.zeros(T).cuda())
    assert torch.equal(got.loss[[1, 4]], torch.ones(2).cuda())


def test_policy_leaves_out_what_has_no_part():
    T = 1000
    s = policy_inputs(T, 3)
    kw = dict(old_logp=s["old"], ref_logp=s["ref"], weights=s["w"], kl_coef=0.1, dual=3.0,
              entropy_coef=0.01)
    head = arc.TokenLogProbs(V=10, rows=T, dtype="f32")
    want = head.policy(s["logp"], s["y"], s["A"], entropy=s["H"], **kw)
    none = s["y"] < 0
    bad = dict(kw)
    for k, v in (("old_logp", NAN), ("ref_logp", INF), ("weights", NAN)):
        bad[k] = torch.where(none, v, kw[k])
    got = head.policy(torch.where(none, -INF, s["logp"]), s["y"], torch.where(none, NAN, s["A"]),
                      entropy=torch.where(none, NAN, s["H"]), **bad)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    # weight 0: terms, but no part in sums and gradients
    zero = torch.zeros(T, device="cuda", dtype=torch.bool)
    zero[5:50] = True
    kw["weights"] = torch.where(zero, 0.0, s["w"])
    want = head.policy(s["logp"], s["y"], s["A"], entropy=s["H"], **kw)
    got = head.policy(torch.where(zero, -INF, s["logp"]), s["y"], s["A"], entropy=s["H"], **kw)
    for k in ("totals", "d_logp", "d_entropy"):
        assert torch.equal(getattr(got, k), getattr(want, k))
    assert bool((got.d_logp[zero] == 0).all()) and bool((got.d_entropy[zero] == 0).all())


def test_policy_follows_the_formulas_into_infinity():
    y = torch.zeros(4, dtype=torch.int64).cuda()
    A = torch.tensor([1.0, -1.0, 1.0, 1.0]).cuda()
    l = torch.tensor([-INF, -INF, -1.0, NAN]).cuda()
    old = torch.full((4,), -1.0).cuda()
    ref = torch.tensor([-1.0, -1.0, -INF, -1.0]).cuda()
    head = arc.TokenLogProbs(V=10, rows=4, dtype="f32")
    got = head.policy(l, y, A, old_logp=old)
    assert got.ratio.tolist()[:3] == [0.0, 0.0, 1.0] and math.isnan(got.ratio[3])
    assert got.d_logp.tolist()[:3] == [0.0, 0.0, -1.0] and math.isnan(got.d_logp[3])
    got = head.policy(l, y, A, old_logp=old, ref_logp=ref, kl_coef=0.5)
    assert got.kl.tolist()[:3] == [INF, INF, INF] and math.isnan(got.kl[3])
    assert got.d_logp.tolist()[:3] == [-INF, -INF, -0.5] and math.isnan(got.loss[3])


LOGITS = [  # rows, V, dtype, pad: a row in registers of each kernel, and rows read twice
    (1, 1, "f32", 0), (1, 7, "bf16", 1), (5, 33, "bf16", 0), (40, 1001, "bf16", 3),
    (64, 5000, "f32", 0), (70, 9001, "bf16", 0), (33, 12_001, "f32", 1), (60, 32_000, "bf16", 0),
    (40, 40_000, "f32", 0), (40, 50_257, "bf16", 47), (3, 50_257, "bf16", 0),
    (140, 100_003, "bf16", 0), (36, 98_000, "f32", 0), (2, 131_077, "f32", 5),
    (9, 200_003, "bf16", 0), (128, 700, "bf16", 1), (129, 701, "f32", 0), (300, 12_001, "bf16", 0)]


@pytest.mark.parametrize("o", [OPTIONS[0], OPTIONS[2], OPTIONS[5]])
@pytest.mark.parametrize("T,V,dtype,pad", LOGITS)
def test_policy_from_logits(T, V, dtype, pad, o):
    gen = torch.Generator().manual_seed(T + V)
    x = place(torch.randn(T, V, generator=gen) * 2, dtype, pad)
    y = torch.randint(0, V, (T,), generator=gen)
    if T > 4:
        y[2] = -1
    want = formulas(x, y, 0.8, 0)
    s = policy_inputs(T, V, want["logp"])
    if T > 4:
        x[4, :] = -INF  # a masked row: its ratio is 0
        x[4, 0] = 1.0
        y[4] = V - 1
        s["A"][4], s["ref"][4], s["w"][4] = -1.0, -1.0, 0.0
        o = dict(o, weights=True)
        want = formulas(x, y, 0.8, 0)
    scale = f32(0.8)
    want = formulas(x, y, scale, 0)
    kw = keywords(o, s)
    head = arc.TokenLogProbs(V=V, rows=T + 3, dtype=dtype, scale=0.8)
    got = head.policy_loss(x, y.cuda(), s["A"], **kw)
    off = slack(x, scale)
    near("lse", got.lse, want["lse"], lse_slack(x, scale, want["lse"]))
    tol = off + 4 * EPS * want["logp"].abs().nan_to_num(posinf=0.0)
    near("logp", got.logp, want["logp"], tol)
    H_tol = off * (2 + 2 * math.log(V + 1))
    near("entropy", got.entropy, want["entropy"], H_tol)
    # the terms from the log probabilities that the call gave, held to the formulas
    terms = policy_formulas(got.logp, got.entropy, y, s["A"], **kw)
    for name in ("loss", "ratio", "kl", "totals"):
        near(name, getattr(got, name), *terms[name])
    # and the gradient of the logits from those upstream
    up = (terms["d_logp"][0].float().cuda(), terms["d_entropy"][0].float().cuda(), None)
    check_policy_grad(x, y, scale, dtype, want, up, terms, got.grad)
    # scored, weighed and differentiated one after the other
    scores = head.score(x, y.cuda())
    parts = head.policy(scores.logp, y.cuda(), s["A"], entropy=scores.entropy, **kw)
    near("chain: loss", parts.loss, got.loss.cpu(), 4 * terms["loss"][1] + 30 * tol.nan_to_num() *
         (terms["ratio"][0] * s["A"].cpu().abs() + 2))
    # in place of the logits
    stored = x.clone()
    wide = place(stored.float(), dtype, pad)
    inside = head.policy_loss(wide, y.cuda(), s["A"], **kw, out=wide)
    assert inside.grad.data_ptr() == wide.data_ptr()
    assert torch.equal(wide, got.grad)
    for a, b in zip(inside[:-1], got[:-1]):
        assert torch.equal(a, b)
    head.close()


def check_policy_grad(x, y, scale, dtype, want, up, terms, grad):
    """check_grad() with the upstream gradients' own tolerances on top: they go
    into an element through dl (1 + p) and dh p (|log p| + H)."""
    T, V = x.shape
    dl, dh = up[0].double().cpu(), up[1].double().cpu()
    q, logq, H = want["q"], want["logq"], want["entropy"]
    safe = torch.where(q > 0, logq, 0.0)
    g = -q * dl[:, None] - dh[:, None] * q * (safe + H[:, None])
    live = y >= 0
    g[torch.arange(T)[live], y[live]] += dl[live]
    g *= scale
    g[((dl == 0) & (dh == 0)) | want["empty"]] = 0.0
    tol = lse_slack(x, scale, want["lse"])[:, None]
    rel = 4 * tol + 8 * EPS + 8 * EPS * safe.abs().nan_to_num()
    size = (dl.abs() + dh.abs() * (H.abs() + 2))[:, None] + dh.abs()[:, None] * safe.abs()
    bound = scale * q * size * rel + scale * dl.abs()[:, None] * 4 * EPS
    bound += scale * dh.abs()[:, None] * q * tol * (4 + 2 * math.log(V + 1))
    given = torch.zeros_like(q)
    given[torch.arange(T)[live], y[live]] = 1.0
    bound += scale * (q + given) * (terms["d_logp"][1] + EPS * dl.abs())[:, None]
    if dtype == "bf16":
        bound = bound + (g.abs() + bound) * 2.0 ** -8
    near("grad", grad, g, bound + 1e-37)


def test_policy_gradient_against_differences():
    T, V, h = 6, 11, 1e-5
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(T, V, generator=gen).float()
    y = torch.tensor([3, 0, -1, 10, 5, 7])
    s = policy_inputs(T, 9, torch.log_softmax(x.double() * 1.5, 1)[torch.arange(T),
                                                                  y.clamp(min=0)])
    kw = dict(old_logp=s["old"], ref_logp=s["ref"], weights=s["w"], kl_coef=0.3,
              entropy_coef=0.2, clip_low=0.2, clip_high=0.3, dual=3.0, scale=2.0)
    head = arc.TokenLogProbs(V=V, rows=T, dtype="f32", scale=1.5)
    got = head.policy_loss(x.cuda(), y.cuda(), s["A"], **kw).grad.double().cpu()

    def total(z):
        q = torch.log_softmax(z * 1.5, 1)
        l, H = q[torch.arange(T), y.clamp(min=0)], -(q.exp() * q).sum(1)
        return float(policy_formulas(l, H, y, s["A"], **kw)["totals"][0][0])

    for i in range(T):
        for j in range(V):
            up, down = x.double().clone(), x.double().clone()
            up[i, j] += h
            down[i, j] -= h
            want = (total(up) - total(down)) / (2 * h)
            # the third derivative times h^2 / 6, 64 bits over 2 h, binary32 of the kernel
            assert abs(float(got[i, j]) - want) < 1e-7 + 1e-9 + 2e-6 * (1 + abs(want))


# ---------------------------------------------------------------- preference

def pair_formulas(logp, y, offsets, *, ref_logp=None, weights=None, kind="sigmoid", beta=0.1,
                  margin=0.0, smoothing=0.0, average=False, scale=1.0, off=0.0):
    T = y.numel()
    off_t = torch.as_tensor(off, dtype=torch.float64).expand(T)
    y, o = y.cpu(), offsets.cpu().tolist()
    P = (len(o) - 1) // 2
    live = y >= 0
    d = logp.double().cpu() - opt(ref_logp, T)
    beta, margin, e = f32(beta), f32(margin), f32(smoothing)
    reward, share, slack_ = [], [], []
    for k in range(2 * P):
        part = d[o[k]:o[k + 1]][live[o[k]:o[k + 1]]]
        share.append(beta / max(1, part.numel()) if average else beta)
        reward.append(part.sum() * share[-1])
        slack_.append(off_t[o[k]:o[k + 1]].sum() * share[-1])
    reward = torch.stack(reward) if P else torch.zeros(0, dtype=torch.float64)
    share = torch.tensor(share, dtype=torch.float64)
    slack_ = torch.tensor([float(x) for x in slack_], dtype=torch.float64)
    gap = reward[:P] - reward[P:]
    z = gap - margin
    tol_z = slack_[:P] + slack_[P:] + 1e-12 * (1 + reward[:P].abs() + reward[P:].abs())
    if kind == "sigmoid":
        ls = torch.nn.functional.logsigmoid
        loss = -(1 - e) * ls(z) - e * ls(-z)
        dz = e * torch.sigmoid(z) - (1 - e) * torch.sigmoid(-z)
        slope, bend = dz.abs(), torch.sigmoid(z) * torch.sigmoid(-z)
    elif kind == "hinge":
        loss, dz = (1 - z).clamp(min=0), -(z < 1).double()
        slope, bend = dz.abs(), 0 * z
        assert not bool(((z - 1).abs() < 2 * tol_z).any()), "inputs on the border"
    else:
        loss, dz = ((z - 0.5) / beta) ** 2, 2 * (z - 0.5) / beta ** 2
        slope, bend = dz.abs(), 2 / beta ** 2 + 0 * z
    w = torch.ones(P, dtype=torch.float64) if weights is None else weights.double().cpu()
    w = w * f32(scale)
    has = w != 0
    by = torch.cat([torch.where(has, w * dz, 0.0), torch.where(has, -w * dz, 0.0)]) * share
    tol_by = torch.cat([w.abs() * bend * tol_z] * 2) * share + EPS * by.abs()
    g, tol_g = torch.zeros(T, dtype=torch.float64), torch.zeros(T, dtype=torch.float64)
    for k in range(2 * P):
        g[o[k]:o[k + 1]] = by[k]
        tol_g[o[k]:o[k + 1]] = tol_by[k]
    parts = [loss, gap, (reward[:P] > reward[P:]).double()]
    totals = torch.stack([torch.where(has, w * x, 0.0).sum() for x in parts])
    tols = [slope * tol_z, tol_z, 0 * z]
    tol_totals = torch.stack([(w.abs() * t).nan_to_num().sum() + EPS * abs(float(x))
                              + 1e-12 * (w * p).abs().nan_to_num().sum()
                              for t, x, p in zip(tols, totals.nan_to_num(), parts)])
    return {"loss": (loss, slope * tol_z + 1e-12 + EPS * loss.abs()),
            "rewards": (reward, slack_ + 1e-12 * (1 + reward.abs()) + EPS * reward.abs()),
            "totals": (totals, tol_totals + 1e-37),
            "d_logp": (torch.where(live, g, 0.0), tol_g + 1e-37)}


def pair_inputs(lengths, seed, head=0, tail=0, logp=None):
    gen = torch.Generator().manual_seed(seed)
    T = head + sum(lengths) + tail
    l = -torch.rand(T, generator=gen, dtype=torch.float64) * 5 if logp is None else logp
    offsets = torch.tensor([head] + [head + sum(lengths[:k + 1]) for k in range(len(lengths))])
    y = torch.randint(0, 100, (T,), generator=gen)
    y = torch.where(torch.rand(T, generator=gen) < 0.3, -1, y)
    ref = l + 0.2 * torch.randn(T, generator=gen, dtype=torch.float64)
    return {"logp": l.float().cuda(), "y": y.cuda(), "offsets": offsets.cuda(),
            "ref": ref.float().cuda(),
            "w": torch.rand(len(lengths) // 2, generator=gen).cuda()}


KINDS = [dict(), dict(smoothing=0.1, margin=0.3, ref=True, weights=True, scale=0.5),
         dict(kind="hinge", beta=0.5, ref=True), dict(kind="squared", average=True, beta=1.0,
                                                      ref=True, weights=True),
         dict(average=True, beta=2.0, margin=1.0), dict(kind="hinge", average=True, beta=8.0)]

LENGTHS = [[], [1, 1], [0, 3], [0, 0], [5, 0], [64, 65], [3, 1, 0, 7, 255, 2], [300, 200, 1000, 257],
           [1, 2] * 700, [9] * 2600, [70_000, 3000], [4100, 0, 2, 9000], [0, 200_001],
           [6000] * 120]


def pair_keywords(o, s):
    kw = {k: v for k, v in o.items() if k not in ("ref", "weights")}
    return dict(kw, ref_logp=s["ref"] if o.get("ref") else None,
                weights=s["w"] if o.get("weights") else None)


@pytest.mark.parametrize("o", KINDS)
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda x: f"{len(x)}x{max(x, default=0)}")
@pytest.mark.parametrize("outside", [(0, 0), (3, 70)])
def test_preference_terms(lengths, o, outside):
    s = pair_inputs(lengths, len(lengths) + 3, *outside)
    T, P = s["y"].numel(), len(lengths) // 2
    kw = pair_keywords(o, s)
    head = arc.TokenLogProbs(V=10, rows=max(T, 1), dtype="f32")
    got = head.preference(s["logp"], s["y"], s["offsets"], **kw)
    again = head.preference(s["logp"], s["y"], s["offsets"], **kw)
    for a, b in zip(got, again):
        assert torch.equal(a, b), "a call repeats its bits"
    assert got.loss.shape == (P,) and got.rewards.shape == (2 * P,) and got.d_logp.shape == (T,)
    want = pair_formulas(s["logp"], s["y"], s["offsets"], **kw)
    for name, x in got._asdict().items():
        near(name, x, *want[name])
    d = got.d_logp.cpu()
    assert bool((d[:outside[0]] == 0).all()) and bool((d[T - outside[1]:] == 0).all())


@pytest.mark.parametrize("lengths", [[], [1, 1]])
def test_many_rows_outside_all_sequences(lengths):
    s = pair_inputs(lengths, 2, 50, 100_003)
    T = s["y"].numel()
    head = arc.TokenLogProbs(V=10, rows=T, dtype="f32")
    got = head.preference(s["logp"], s["y"], s["offsets"])
    want = pair_formulas(s["logp"], s["y"], s["offsets"])
    for name, x in got._asdict().items():
        near(name, x, *want[name])
    d = got.d_logp
    assert bool((d[:50] == 0).all()) and bool((d[50 + sum(lengths):] == 0).all())


def test_preference_leaves_out_what_has_no_part():
    s = pair_inputs([100, 50, 0, 2000, 30, 4], 8, 5, 9)
    head = arc.TokenLogProbs(V=10, rows=3000, dtype="f32")
    kw = dict(ref_logp=s["ref"], weights=s["w"], beta=0.1)
    want = head.preference(s["logp"], s["y"], s["offsets"], **kw)
    none = s["y"] < 0
    got = head.preference(torch.where(none, NAN, s["logp"]), s["y"], s["offsets"],
                          **dict(kw, ref_logp=torch.where(none, INF, s["ref"])))
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    # a pair of weight 0 whose answer has a masked token: its loss, and nothing else
    w = s["w"].clone()
    w[1] = 0.0
    at = torch.arange(s["y"].numel(), device="cuda")
    o = s["offsets"].tolist()
    second = ((at >= o[1]) & (at < o[2])) | ((at >= o[4]) & (at < o[5]))
    want = head.preference(s["logp"], s["y"], s["offsets"], **dict(kw, weights=w))
    got = head.preference(torch.where(second, -INF, s["logp"]), s["y"], s["offsets"],
                          **dict(kw, weights=w))
    assert torch.equal(got.totals, want.totals) and torch.equal(got.d_logp, want.d_logp)
    assert bool((got.d_logp[second] == 0).all())


def test_far_rewards():
    """Losses and gradients where a sigmoid is 0 or 1 in binary32, and infinities."""
    l = torch.tensor([0.0, -200.0, 300.0, -INF, -200.0, 0.0, 0.0, 0.0]).cuda()
    y = torch.zeros(8, dtype=torch.int64).cuda()
    o = torch.arange(9).cuda()
    head = arc.TokenLogProbs(V=10, rows=8, dtype="f32")
    got = head.preference(l, y, o, beta=1.0)
    assert got.loss.tolist()[1:] == [200.0, 0.0, INF] and 0 < float(got.loss[0]) < 1e-80 or \
        float(got.loss[0]) == 0.0
    assert got.d_logp.tolist()[1] == -1.0 and got.d_logp.tolist()[3] == -1.0
    assert got.d_logp.tolist()[2] == 0.0 and got.d_logp.tolist()[5] == 1.0


@pytest.mark.parametrize("offsets", [
    [0, 5, 3, 100, 7], [-9, 2, 4, 6, 8], [0, 2**40, 3, -2**62, 5], [100, 90, 80, 70, 60],
    [50, 50, 50, 50, 50]])
def test_offsets_stay_inside_the_rows(offsets):
    """Whatever they hold, nothing outside the rows is touched (the values behind
    them are compared) and tokens outside all sequences have no gradient."""
    T = 60
    s = pair_inputs([30, 30], 4)
    buf = torch.full((T + 200,), 7.0, device="cuda")
    head = arc.TokenLogProbs(V=10, rows=T, dtype="f32")
    cfg = arc.arc_preference_config(0, 0, 0.1, 0.0, 0.0, 1.0)
    o = torch.tensor(offsets).cuda()
    loss, rewards, totals = torch.zeros(2).cuda(), torch.zeros(4).cuda(), torch.zeros(3).cuda()
    arc.arc_tokens_preference_terms(head.ctx, cfg, T, s["logp"], s["y"], 2, o, None, None, loss,
                                    rewards, totals, buf[100:100 + T])
    torch.cuda.synchronize()
    assert bool((buf[:100] == 7.0).all()) and bool((buf[100 + T:] == 7.0).all())


PAIR_LOGITS = [([3, 2], 33, "f32", 0), ([1, 0], 7, "bf16", 1), ([9, 20, 0, 15], 1001, "bf16", 3),
               ([40, 30, 20, 25], 9001, "f32", 0), ([10, 12], 50_257, "bf16", 47),
               ([2, 1], 131_077, "f32", 0), ([300, 340], 2000, "bf16", 0)]


@pytest.mark.parametrize("o", [KINDS[1], KINDS[3], KINDS[4]])
@pytest.mark.parametrize("lengths,V,dtype,pad", PAIR_LOGITS)
def test_preference_from_logits(lengths, V, dtype, pad, o):
    T = sum(lengths) + 4
    gen = torch.Generator().manual_seed(V)
    x = place(torch.randn(T, V, generator=gen) * 2, dtype, pad)
    y = torch.randint(0, V, (T,), generator=gen)
    y[1] = -1
    want = formulas(x, y, 1.0, 0)
    s = pair_inputs(lengths, V, 1, 3, want["logp"])
    kw = pair_keywords(o, s)
    head = arc.TokenLogProbs(V=V, rows=T, dtype=dtype)
    got = head.preference_loss(x, y.cuda(), s["offsets"], **kw)
    off = slack(x, 1.0)
    near("lse", got.lse, want["lse"], lse_slack(x, 1.0, want["lse"]))
    near("logp", got.logp, want["logp"], off + 4 * EPS * want["logp"].abs())
    near("entropy", got.entropy, want["entropy"], off * (2 + 2 * math.log(V + 1)))
    terms = pair_formulas(got.logp, y, s["offsets"], **kw)
    for name in ("loss", "rewards", "totals"):
        near(name, getattr(got, name), *terms[name])
    up = (terms["d_logp"][0].float().cuda(), torch.zeros(T).cuda())
    check_policy_grad(x, y, 1.0, dtype, want, up, terms, got.grad)
    scores = head.score(x, y.cuda())
    parts = head.preference(scores.logp, y.cuda(), s["offsets"], **kw)
    near("chain: rewards", parts.rewards, got.rewards.cpu(),
         2 * terms["rewards"][1] + 8 * float(off.max()) * T)
    stored = place(x.float(), dtype, pad)
    inside = head.preference_loss(stored, y.cuda(), s["offsets"], **kw, out=stored)
    assert torch.equal(stored, got.grad) and torch.equal(inside.totals, got.totals)
    head.close()


@pytest.mark.parametrize("o", KINDS)
def test_preference_gradient_against_differences(o):
    V, h, lengths = 9, 1e-5, [3, 2, 2, 1]
    T = sum(lengths)
    gen = torch.Generator().manual_seed(2)
    x = torch.randn(T, V, generator=gen).float()
    y = torch.randint(0, V, (T,), generator=gen)
    y[1] = -1
    s = pair_inputs(lengths, 21, logp=torch.log_softmax(x.double(), 1)[
        torch.arange(T), y.clamp(min=0)])
    kw = pair_keywords(o, s)
    head = arc.TokenLogProbs(V=V, rows=T, dtype="f32")
    got = head.preference_loss(x.cuda(), y.cuda(), s["offsets"], **kw).grad.double().cpu()

    def total(z):
        l = torch.log_softmax(z, 1)[torch.arange(T), y.clamp(min=0)]
        return float(pair_formulas(l, y, s["offsets"], **kw)["totals"][0][0])

    for i in range(T):
        for j in range(V):
            up, down = x.double().clone(), x.double().clone()
            up[i, j] += h
            down[i, j] -= h
            want = (total(up) - total(down)) / (2 * h)
            # h^2 times the third derivative, 64 bits over 2 h, binary32 of the kernel
            assert abs(float(got[i, j]) - want) < 1e-7 + 2e-6 * (1 + abs(want))


def test_no_rows():
    """Nothing to do gives totals of 0 and gradients without rows."""
    head = arc.TokenLogProbs(V=10, rows=4, dtype="bf16")
    x = torch.zeros(0, 10, dtype=torch.bfloat16).cuda()
    y, v = torch.zeros(0, dtype=torch.int64).cuda(), torch.zeros(0).cuda()
    out = head.policy_loss(x, y, v, old_logp=v, ref_logp=v, kl_coef=0.1, entropy_coef=0.1)
    assert out.totals.tolist() == [0.0] * 5 and out.grad.shape == (0, 10)
    assert head.policy(v, y, v).totals.tolist() == [0.0] * 5
    for P in (0, 3):  # no pair, and pairs without tokens
        o = torch.zeros(2 * P + 1, dtype=torch.int64).cuda()
        out = head.preference_loss(x, y, o)
        want = [P * math.log(2.0), 0.0, 0.0]
        for got in (out, head.preference(v, y, o)):
            near("totals", got.totals, torch.tensor(want), 4 * EPS * P)
            assert got.rewards.tolist() == [0.0] * (2 * P)
        assert out.grad.shape == (0, 10)


# ---------------------------------------------------------------- large calls

@pytest.mark.parametrize("T,V,dtype", [(1_100_003, 9, "f32"), (45_000, 50_257, "bf16")])
def test_rows_and_offsets_of_large_calls(T, V, dtype):
    """More rows than one launch takes, and elements beyond 32 bits: each row's results
    are those of a smaller call (its kernel is the same one)."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    x = torch.randn(T, V, generator=gen, device="cuda", dtype=kind)
    y = torch.randint(-1, V, (T,), generator=gen, device="cuda")
    old, ref, A = (torch.randn(T, generator=gen, device="cuda") for _ in range(3))
    old, ref = old - math.log(V), ref - math.log(V)
    w = torch.rand(T, generator=gen, device="cuda")
    kw = dict(kl_coef=0.05, entropy_coef=0.01, dual=3.0)
    head = arc.TokenLogProbs(V=V, rows=T, dtype=dtype)
    got = head.policy_loss(x, y, A, old_logp=old, ref_logp=ref, weights=w, **kw)
    # a pair of two halves, and rows behind it
    o = torch.tensor([0, T // 2, T - 9]).cuda()
    pairs = head.preference_loss(x, y, o, ref_logp=ref, beta=1e-4)
    terms = head.preference(pairs.logp, y, o, ref_logp=ref, beta=1e-4)
    assert torch.equal(terms.totals, pairs.totals) and torch.equal(terms.loss, pairs.loss)
    for rows in (slice(0, 300), slice(1 << 20, (1 << 20) + 300), slice(T - 300, T)):
        if rows.start >= T:
            continue
        part = head.policy_loss(x[rows], y[rows], A[rows], old_logp=old[rows],
                                ref_logp=ref[rows], weights=w[rows], **kw)
        for name in ("logp", "entropy", "lse", "loss", "ratio", "kl", "grad"):
            assert torch.equal(getattr(got, name)[rows], getattr(part, name)), name
        want = formulas(x[rows], y[rows], 1.0, 0)
        near("logp", pairs.logp[rows], want["logp"],
             slack(x[rows], 1.0) + 4 * EPS * want["logp"].abs())
        d = terms.d_logp[rows]
        check_policy_grad(x[rows], y[rows].cpu(), 1.0, dtype, want, (d, torch.zeros(300).cuda()),
                          {"d_logp": (d, EPS * d.double().abs().cpu())}, pairs.grad[rows])


# ---------------------------------------------------------------- streams, graphs, refusals

@pytest.mark.parametrize("T,lengths", [(200, [60, 40, 55, 45]), (90, [27, 18, 25, 20])])
def test_on_another_stream_and_in_a_graph(T, lengths):
    """Captured calls repeat on new contents, with eager calls of the same context
    between the replays."""
    V = 5001
    stream = torch.cuda.Stream()
    gen = torch.Generator().manual_seed(1)
    x = place(torch.randn(T, V, generator=gen), "bf16")
    fresh = [torch.randn(T, V, generator=gen).bfloat16().cuda() for _ in range(3)]
    y = tokens(T, V - 10, 3)
    s = policy_inputs(T, 1)
    p = pair_inputs(lengths, 1)
    head = arc.TokenLogProbs(V=V, rows=T, dtype="bf16", stream=stream)
    torch.cuda.synchronize()

    def calls():
        a = head.policy_loss(x, y, s["A"], old_logp=s["old"], kl_coef=0.1, ref_logp=s["ref"],
                             entropy_coef=0.1)
        b = head.preference_loss(x, y, p["offsets"], beta=0.2)
        c = head.preference(a.logp, y, p["offsets"], beta=0.2)
        d = head.policy(b.logp, y, s["A"], old_logp=s["old"])
        return [*a, *b, *c, *(v for v in d if v is not None)]

    for _ in range(2):
        eager = calls()  # from the default stream: outputs are the stream's
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        captured = calls()
    for z in fresh:
        x.copy_(z)
        torch.cuda.synchronize()
        eager = calls()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
            graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, eager):
            assert torch.equal(a.nan_to_num(), b.nan_to_num())


def test_refusals():
    head = arc.TokenLogProbs(V=10, rows=8, dtype="f32")
    x = torch.zeros(8, 10).cuda()
    y = torch.zeros(8, dtype=torch.int64).cuda()
    v = torch.zeros(8).cuda()
    o = torch.tensor([0, 4, 8]).cuda()
    for kw in (dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_low=NAN), dict(clip_high=-0.1),
               dict(clip_high=NAN), dict(dual=0.5), dict(dual=INF), dict(dual=NAN),
               dict(kl_coef=-1.0, ref_logp=v), dict(kl_coef=0.1), dict(kl_coef=INF, ref_logp=v),
               dict(entropy_coef=NAN), dict(scale=INF)):
        with pytest.raises(arc.ArcError):
            head.policy_loss(x, y, v, **kw)
        with pytest.raises(arc.ArcError):
            head.policy(v, y, v, entropy=v, **kw)
    with pytest.raises(arc.ArcError):
        head.policy(v, y, v, entropy_coef=0.1)
    for kw in (dict(beta=0.0), dict(beta=-1.0), dict(beta=NAN), dict(beta=INF),
               dict(margin=INF), dict(smoothing=0.6), dict(smoothing=-0.1),
               dict(smoothing=0.1, kind="hinge"), dict(scale=NAN)):
        with pytest.raises(arc.ArcError):
            head.preference_loss(x, y, o, **kw)
        with pytest.raises(arc.ArcError):
            head.preference(v, y, o, **kw)
    for bad in (lambda: head.policy(v, y, v[:7]), lambda: head.policy(v.double(), y, v),
                lambda: head.policy(v, y, v, old_logp=v.cpu()),
                lambda: head.preference(v, y, o[:2]), lambda: head.preference(v, y, o.int()),
                lambda: head.preference(v, y, o, weights=v),
                lambda: head.policy_loss(x[:, :9], y, v),
                lambda: head.policy(v, torch.zeros(16, dtype=torch.int64).cuda()[::2], v)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(KeyError):
        head.preference(v, y, o, kind="none")
    with pytest.raises(arc.ArcError):  # more rows than the context has
        big = torch.zeros(9).cuda()
        head.policy(big, torch.zeros(9, dtype=torch.int64).cuda(), big)
    # outputs on inputs
    cfg = arc.arc_policy_config(0.2, 0.2, 0.0, 0.0, 0.0, 1.0)
    t = torch.zeros(5).cuda()
    L = _lib._lib

    def status(*a):
        return L.arc_tokens_policy_terms(head.ctx, ctypes.byref(cfg), 8,
                                         *(None if q is None else q.data_ptr() for q in a))

    w = torch.zeros(8).cuda()
    ok = (v, None, y, None, None, w, None)
    assert status(*ok, None, None, None, t, None, None) == arc.ARC_OK
    for outs in ((v, None, None, t, None, None), (None, None, None, t, w, None),
                 (None, None, None, v, None, None), (t, None, None, t, None, None)):
        assert status(*ok, *outs) == arc.ARC_ERR_INVALID
    assert status(*ok, None, None, None, None, None, None) == arc.ARC_ERR_INVALID  # totals
    assert status(None, *ok[1:], None, None, None, t, None, None) == arc.ARC_ERR_INVALID
    torch.cuda.synchronize()
