"""Matrices orthogonalised by Newton-Schulz products and the optimizer made of
them, against the same polynomials in 64 bits: sides from one up, odd ones, tall
and wide, every kernel variant, matrices of zeros, NaN and no elements."""
import ctypes
import math

import pytest
import torch

import paper_2510_26709_amd as arc
from paper_2510_26709_amd import _lib

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
QUINTIC = (3.4445, -4.7750, 2.0315)
NAN = math.nan


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def f32(v):
    return ctypes.c_float(v).value


def polynomials(u, steps=5, coefficients=QUINTIC, dtype=torch.float64):
    """The definition, in 64 bits or with every product in 32."""
    if not u.numel():
        return u.to(dtype)
    rows = [coefficients] * steps if not isinstance(coefficients[0], tuple) else coefficients
    tall = u.shape[0] > u.shape[1]
    x = (u.t() if tall else u).double()
    norm = x.norm()
    x = (x / norm if norm > 0 else x).to(dtype).contiguous()
    for a, b, c in rows:
        a, b, c = f32(a), f32(b), f32(c)
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return (x.t() if tall else x).contiguous()


def rounded(u, seed, steps=5, coefficients=QUINTIC):
    """The definition in 64 bits with the roundings of pairs put in at random: a pair
    is off by at most 2^-23 of its number (11 bits, then 11 of what is left), and a
    product of pairs lacks lo lo, at most 2^-24 of a term (2^-12 of each factor)."""
    rows = [coefficients] * steps if not isinstance(coefficients[0], tuple) else coefficients
    gen = torch.Generator(device=u.device).manual_seed(seed)

    def noise(x, size):
        r = torch.rand(x.shape, generator=gen, device=x.device, dtype=torch.float64) * 2 - 1
        return r * x.abs() * size

    def pairs(x):
        return x + noise(x, 2.0 ** -23)

    def product(x, y):  # the terms' errors add at random: the root of their squares' sum
        r = torch.randn(x.shape[0], y.shape[1], generator=gen, device=x.device,
                        dtype=torch.float64)
        return x @ y + r * ((x * x) @ (y * y)).sqrt() * 2.0 ** -24

    tall = u.shape[0] > u.shape[1]
    x = (u.t() if tall else u).double().contiguous()
    norm = x.norm()
    x = pairs(x / norm if norm > 0 else x)
    for k, (a, b, c) in enumerate(rows):
        a, b, c = f32(a), f32(b), f32(c)
        gram = pairs(product(x, x.t().contiguous()))
        poly = b * gram + c * product(gram, gram)
        poly.diagonal().add_(a)
        x = product(pairs(poly), x)
        x = pairs(x) if k + 1 < len(rows) else x
    return (x.t() if tall else x).contiguous()


def allowed_error(u, want, **kw):
    """Of all elements together: four times what the pairs' roundings do in three
    trials, and four times what the sums of binary32 products do, which has the
    kernel's number of additions.  (Both are random; their spread over matrices of
    few elements is what the factor is for.)"""
    plain = polynomials(u, dtype=torch.float32, **kw).double()
    model = max(float((rounded(u, seed, **kw) - want).norm()) for seed in range(3))
    return 4 * (model + float((plain - want).norm()))


def close_to(got, u, what, **kw):
    want = polynomials(u, **kw)
    g = got.double()
    step = 2.0 ** -8 if got.dtype == torch.bfloat16 else EPS
    size = float(want.norm())
    off = float((g - want).norm())
    allowed = allowed_error(u, want, **kw) + step * size
    assert off <= allowed, f"{what}: off by {off / size:.3e}, allowed {allowed / size:.3e}"
    # and every element, by the same measure: 12 times the root of the mean square
    most = float((g - want).abs().max())
    each = 12 * allowed / math.sqrt(u.numel()) + step * float(want.abs().max())
    assert most <= each, f"{what}: one off by {most:.3e}, allowed {each:.3e}"


def matrices(shapes, seed, dtype=torch.float32):
    """Strong directions above noise, each at a scale of its own."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for k, (r, c) in enumerate(shapes):
        q = max(1, min(4, r, c))
        u = torch.randn(r, c, device="cuda", generator=gen)
        if r and c:
            u += (torch.randn(r, q, device="cuda", generator=gen)
                  @ torch.randn(q, c, device="cuda", generator=gen)) * 2
        out.append((u * 10.0 ** (k % 7 - 4)).to(dtype))
    return out


SHAPES = [(1, 1), (1, 7), (7, 1), (2, 3), (5, 4), (16, 16), (31, 64), (63, 65), (64, 64),
          (65, 63), (65, 129), (128, 128), (129, 257), (257, 1001), (1000, 100), (31, 2048),
          (3000, 17), (640, 640), (5, 20_000), (1, 70_001), (511, 513)]
WORDS = {torch.float32: "f32", torch.bfloat16: "bf16"}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES)
def test_one_matrix(shape, dtype):
    u, = matrices([shape], sum(shape), dtype)
    opt = arc.Muon([shape], grad_dtype=WORDS[dtype])
    got, = opt.orthogonalize([u])
    again, = opt.orthogonalize([u])
    assert got.shape == shape and torch.equal(got, again), "a call repeats its bits"
    close_to(got, u, shape)
    opt = arc.Muon([shape], grad_dtype=WORDS[dtype], param_dtype="bf16")
    low, = opt.orthogonalize([u])
    close_to(low, u, ("bf16", shape))


MANY = [(512, 2048), (2048, 512), (300, 1100), (1024, 1024), (1, 5), (0, 9), (129, 2000),
        (1500, 700), (1000, 1000), (9, 0), (64, 4096), (33, 31), (768, 2304)]


@pytest.mark.parametrize("param", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", [MANY, SHAPES[:-1], [(33, 65)] * 170 + [(70, 20)],
                                    [(2048, 2048)], [(1100, 2500), (2500, 1100)],
                                    [(5, 3)] * 1000],
                         ids=["many", "all", "batches", "square", "wide", "tiny"])
def test_many_matrices(shapes, param):
    u = matrices(shapes, 5)
    opt = arc.Muon(shapes, param_dtype=param)
    got = opt.orthogonalize(u)
    for k, (shape, x) in enumerate(zip(shapes, u)):
        if x.numel() and (k < 20 or k > len(shapes) - 3):
            close_to(got[k], x, (k, shape))
    flat = opt.orthogonalize(torch.cat([x.reshape(-1) for x in u]))
    assert torch.equal(flat, torch.cat([x.reshape(-1) for x in got]))


@pytest.mark.parametrize("steps,coefficients", [
    (1, QUINTIC), (2, QUINTIC), (8, (1.5, -0.5, 0.0)), (6, (15 / 8, -10 / 8, 3 / 8)),
    (3, [(3.4445, -4.7750, 2.0315), (2.5, -3.0, 1.2), (1.875, -1.25, 0.375)])])
def test_other_polynomials(steps, coefficients):
    shapes = [(100, 300), (300, 100), (65, 65)]
    u = matrices(shapes, 3)
    got = arc.Muon(shapes, steps=steps, coefficients=coefficients).orthogonalize(u)
    for k in range(3):
        close_to(got[k], u[k], (steps, shapes[k]), steps=steps, coefficients=coefficients)


@pytest.mark.parametrize("rank", [1, 4, 64])
@pytest.mark.parametrize("shape,count", [((300, 1100), 1), ((1100, 300), 3), ((897, 3588), 12)])
def test_few_directions(shape, count, rank):
    """All other directions hold roundings alone, which grow 485 times in five steps: by
    as much as with binary32 products, step by step and in runs of steps."""
    gen = torch.Generator(device="cuda").manual_seed(rank)
    u = [torch.randn(shape[0], rank, device="cuda", generator=gen)
         @ torch.randn(rank, shape[1], device="cuda", generator=gen) for _ in range(count)]
    opt = arc.Muon([shape] * count, lr_scale=1.0)
    got = opt.orthogonalize(u)
    x = [torch.zeros_like(v) for v in u]
    opt.step(x, u, lr=1.0, momentum=0.0, nesterov=False)
    for k in {0, count - 1}:
        close_to(got[k], u[k], (k, "alone"))
        close_to(-x[k], u[k], (k, "a step"))


@pytest.mark.parametrize("tall", [False, True])
def test_offsets_beyond_32_bits(tall):
    """4096 x 2^20 with one number in each row (or column), at the far end: their singular
    values are those numbers over the norm, and every product is theirs alone."""
    m, n = 4096, 1 << 20
    u = torch.zeros((n, m) if tall else (m, n), dtype=torch.bfloat16, device="cuda")
    values = torch.linspace(0.5, 4.0, m, device="cuda").bfloat16()
    short = torch.arange(m, device="cuda")
    long = n - 1 - 3 * short.flip(0)
    at = (long, short) if tall else (short, long)
    u[at] = values
    opt = arc.Muon([tuple(u.shape)], param_dtype="bf16", grad_dtype="bf16")
    got, = opt.orthogonalize([u])
    x = values.double() / values.double().norm()
    for a, b, c in [QUINTIC] * 5:
        x = f32(a) * x + f32(b) * x ** 3 + f32(c) * x ** 5
    # pairs are off by 2^-23, a product's one term by 2^-24 and its sum by 2^-24; a singular
    # value's error grows 3.4445 times in a step, with three roundings of pairs and four of
    # products in each: less than 12 EPS, 5 times, and the result's half step
    grown = sum(3.4445 ** k for k in range(6)) * 12 * EPS
    off = (got[at].double() - x).abs()
    assert bool((off <= (grown + 2.0 ** -8) * x.abs() + grown * 1e-3).all())
    got[at] = 0
    assert not bool(got.any()), "zeros elsewhere"


def test_singular_values_come_together():
    gen = torch.Generator(device="cuda").manual_seed(1)
    u = torch.randn(200, 500, device="cuda", generator=gen)
    got, = arc.Muon([(200, 500)]).orthogonalize([u])
    s = torch.linalg.svdvals(got.double().cpu())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25
    got, = arc.Muon([(200, 500)], steps=16, coefficients=(1.5, -0.5, 0.0)).orthogonalize([u])
    s = torch.linalg.svdvals(got.double().cpu())
    assert float((s - 1).abs().max()) < 1e-3


def test_scale_does_not_count():
    """Powers of two leave every bit, to the ends of binary32's range."""
    u, = matrices([(70, 130)], 2)
    u = u / u.abs().max()
    opt = arc.Muon([(70, 130)])
    want, = opt.orthogonalize([u])
    for e in (-90, -40, 1, 60, 127):
        got, = opt.orthogonalize([u * 2.0 ** e])
        assert torch.equal(got, want), e
    tiny = u * 2.0 ** -140  # subnormal: as they are stored
    close_to(opt.orthogonalize([tiny])[0], tiny, "subnormal")


def test_zeros_nan_and_infinity_stay_in_their_matrix():
    shapes = [(70, 200), (64, 64), (200, 70), (33, 5), (130, 130)]
    u = matrices(shapes, 4)
    clean = arc.Muon(shapes).orthogonalize(u)
    u[0][:] = 0.0
    u[1][3, 60] = NAN
    u[3][32, 4] = math.inf
    got = arc.Muon(shapes).orthogonalize(u)
    assert bool((got[0] == 0).all())
    assert bool(torch.isnan(got[1]).all()) and bool(torch.isnan(got[3]).all())
    assert torch.equal(got[2], clean[2]) and torch.equal(got[4], clean[4])
    u[1][:] = 0.0
    u[1][5, 7] = -3.0  # of rank one: the outer product with sign
    got = arc.Muon(shapes).orthogonalize(u)
    want = polynomials(u[1])
    assert bool((got[1][want == 0] == 0).all())
    close_to(got[1], u[1], "one element")


def placed(x, dtype, shift):
    """x's values `shift` elements into memory that is NaN around them."""
    buf = torch.full((x.numel() + 2 * shift + 3,), NAN, dtype=dtype, device="cuda")
    view = buf[shift:shift + x.numel()].view(x.shape)
    view.copy_(x)
    return buf, view


def run_steps(shapes, param, grad, copy, nesterov, shift):
    num, lr, mu = len(shapes), 0.03, 0.9
    wd = [(0.1, 0.0, 0.2, 0.0, 0.1, 0.0)[k % 6] for k in range(num)]
    scales = [(1.0, 2.0, 0.5, 1.0, -1.0, 1.0)[k % 6] for k in range(num)]
    pd = torch.float32 if param == "f32" else torch.bfloat16
    gd = torch.float32 if grad == "f32" else torch.bfloat16
    opt = arc.Muon(shapes, param_dtype=param, grad_dtype=grad, weight_decay=wd, lr_scale=scales)
    x0 = [0.1 * m / m.abs().amax().clamp(min=1e-30) if m.numel() else m
          for m in matrices(shapes, 9)]
    kept = [placed(m, pd, shift) for m in x0]
    x = [v for _, v in kept]
    copies = [placed(m, torch.bfloat16, shift) for m in x0] if copy else None
    cs = [None if k == 2 else copies[k][1] for k in range(num)] if copy else None
    factor = torch.tensor([7.0, 0.25]).cuda()
    m = [torch.zeros(s, dtype=torch.float64, device="cuda") for s in shapes]
    for t in range(3):
        g = [placed(v, gd, shift)[1] for v in matrices(shapes, 20 + t)]
        before = [v.clone() for v in x]
        opt.step(x, g, lr=lr, momentum=mu, nesterov=nesterov, factor=factor, copies=cs)
        for k, shape in enumerate(shapes):
            if not x[k].numel():
                continue
            at = opt.offsets[k]
            held = opt.m[at:at + x[k].numel()].view(shape)
            gk = g[k].double() * 0.25
            want_m = f32(mu) * m[k] + gk
            assert bool(((held.double() - want_m).abs() <=
                         2 * EPS * (want_m.abs() + (f32(mu) * m[k]).abs())).all())
            m[k] = held.double()  # each step from what is held
            u = (gk + f32(mu) * m[k] if nesterov else m[k]).float()
            o = polynomials(u)
            step = f32(lr) * scales[k]
            want = before[k].double() * (1 - step * f32(wd[k])) - step * o
            # O as in close_to(), each element by 12 times the root of the mean square;
            # U rounded once; three roundings of x
            off_o = allowed_error(u, o) + EPS * float(o.norm())
            tol = abs(step) * (12 * off_o / math.sqrt(u.numel()) + EPS * 4) + \
                4 * EPS * (want.abs() + before[k].double().abs())
            tol = tol + (want.abs() + tol) * (2.0 ** -8 if param == "bf16" else 0)
            assert bool(((x[k].double() - want).abs() <= tol).all()), (t, shape)
            if cs and cs[k] is not None:
                assert torch.equal(cs[k], x[k].bfloat16())
    # what lies around them, and between the momenta, is as it was
    for buf, v in kept + (copies or []):
        n = v.numel()
        assert bool(torch.isnan(buf[:shift]).all()) and bool(torch.isnan(buf[shift + n:]).all())
    inside = torch.zeros(opt.m.numel(), dtype=torch.bool, device="cuda")
    for at, n in zip(opt.offsets, opt.sizes):
        inside[at:at + n] = True
    assert bool((opt.m[~inside] == 0).all())
    if copy:
        assert torch.equal(copies[2][1], x0[2].bfloat16())


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("param,grad,copy", [("f32", "f32", True), ("f32", "bf16", True),
                                             ("bf16", "bf16", False), ("bf16", "f32", False)])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_steps(param, grad, copy, nesterov, shift):
    run_steps([(100, 260), (260, 100), (7, 3), (0, 5), (129, 129), (1, 1)], param, grad, copy,
              nesterov, shift)


# Contexts of more work, whose products have larger tiles, step by step and in runs.
LARGER = [[(641, 643)] * 4 + [(643, 130)],
          [(1500, 2100), (2101, 1501), (7, 3), (129, 129)],
          [(1001, 1003)] * 4 + [(1003, 1001)] * 4 + [(9, 70)],
          [(897, 3588)] * 6 + [(3588, 897)] * 6 + [(65, 3)]]


@pytest.mark.parametrize("param,grad,copy,shift", [("f32", "f32", True, 1),
                                                   ("bf16", "bf16", False, 3)])
@pytest.mark.parametrize("shapes", LARGER, ids=["640", "1500", "1000", "four"])
def test_larger_contexts(shapes, param, grad, copy, shift):
    u = matrices(shapes, 13, torch.float32 if grad == "f32" else torch.bfloat16)
    opt = arc.Muon(shapes, param_dtype=param, grad_dtype=grad)
    got = opt.orthogonalize(u)
    again = opt.orthogonalize(u)
    for k, (shape, x) in enumerate(zip(shapes, u)):
        assert torch.equal(got[k], again[k]), "a call repeats its bits"
        if k < 2 or k > len(shapes) - 3:
            close_to(got[k], x, (k, shape))
    run_steps(shapes, param, grad, copy, True, shift)


def test_factors_that_are_not_finite_leave_everything():
    shapes = [(100, 300), (300, 100)]
    x, g = matrices(shapes, 1), matrices(shapes, 2)
    opt = arc.Muon(shapes)
    opt.step(x, g, lr=0.1)
    before = [v.clone() for v in x] + [opt.m.clone()]
    for bad in (NAN, math.inf, -math.inf):
        opt.step(x, g, lr=0.1, factor=torch.tensor([1.0, bad]).cuda())
    for a, b in zip([*x, opt.m], before):
        assert torch.equal(a, b)


def test_after_the_norms_of_adamw():
    """The two optimizers of one model, clipped together: a NaN gradient stops both."""
    shapes, vector = [(64, 96), (96, 64)], 64
    x, g = matrices(shapes, 1), matrices(shapes, 2)
    flat_x = torch.cat([v.reshape(-1) for v in x] + [torch.ones(vector).cuda()])
    flat_g = torch.cat([v.reshape(-1) for v in g] + [torch.ones(vector).cuda()])
    n = flat_x.numel() - vector
    norms = arc.AdamW([r * c for r, c in shapes] + [vector])
    rest, mats = arc.AdamW([vector]), arc.Muon(shapes)
    total = norms.norm(flat_g, max_norm=1.0, scale=0.5).total
    mats.step(flat_x[:n], flat_g[:n], lr=0.1, factor=total)
    rest.step(0, flat_x[n:], flat_g[n:], lr=0.1, factor=total)
    o = polynomials(g[0])  # the factor does not count, the momentum starts at zero
    want = x[0].double() - 0.1 * o
    assert float((flat_x[:n][:64 * 96].view(64, 96).double() - want).abs().max()) < 1e-4
    before = flat_x.clone()
    flat_g[5] = NAN
    total = norms.norm(flat_g, max_norm=1.0, scale=0.5).total
    mats.step(flat_x[:n], flat_g[:n], lr=0.1, factor=total)
    rest.step(1, flat_x[n:], flat_g[n:], lr=0.1, factor=total)
    assert torch.equal(flat_x, before)


def test_states_in_place_and_assigned():
    shapes = [(40, 50)]
    x, g = matrices(shapes, 1), matrices(shapes, 2)
    m = torch.zeros(2048, device="cuda")
    opt = arc.Muon(shapes, states={"m": m})
    assert opt.m is m and opt.offsets == [0]
    opt.step(x, g, lr=0.1)
    assert torch.equal(m[:2000].view(40, 50), g[0])
    other = torch.ones(2048, device="cuda")
    opt.m = other
    opt.step(x, g, lr=0.1, momentum=0.5)
    assert torch.equal(other[:2000].view(40, 50), g[0] + 0.5)
    with pytest.raises(ValueError):
        opt.m = torch.zeros(2047, device="cuda")
    with pytest.raises(ValueError):
        arc.Muon(shapes, states={"m": m.double()})


def test_on_another_stream_and_in_a_graph():
    shapes = [(130, 200), (200, 130), (64, 700)]
    stream = torch.cuda.Stream()
    sides = [r * c for r, c in shapes]
    opt = arc.Muon(shapes, stream=stream)
    ref = arc.Muon(shapes, stream=stream)
    x = torch.zeros(sum(sides), device="cuda")
    y = x.clone()
    g = torch.cat([v.reshape(-1) for v in matrices(shapes, 1)])
    torch.cuda.synchronize()
    out = opt.orthogonalize(g)
    opt.step(x, g, lr=0.1)
    ref.step(y, g, lr=0.1)
    torch.cuda.synchronize()
    assert torch.equal(x, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = opt.orthogonalize(g)
        opt.step(x, g, lr=0.1)
    for t in range(3):
        g.copy_(torch.cat([v.reshape(-1) for v in matrices(shapes, 30 + t)]))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        want = ref.orthogonalize(g)
        ref.step(y, g, lr=0.1)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(x, y) and torch.equal(opt.m, ref.m)


def test_refusals():
    shapes = [(4, 6), (6, 4)]
    opt = arc.Muon(shapes)
    x, g = matrices(shapes, 1), matrices(shapes, 2)
    for kw in (dict(lr=NAN), dict(lr=math.inf), dict(lr=0.1, momentum=1.0),
               dict(lr=0.1, momentum=-0.1), dict(lr=0.1, momentum=NAN)):
        with pytest.raises(arc.ArcError):
            opt.step(x, g, **kw)
    for bad in (lambda: opt.step(x[:1], g, lr=0.1), lambda: opt.step(x, [g[0], g[0][:, :5]], lr=0.1),
                lambda: opt.step(x, [g[0], None], lr=0.1),
                lambda: opt.step(x, [g[0], g[1].cpu()], lr=0.1),
                lambda: opt.step(x, [g[0].t(), g[1]], lr=0.1),
                lambda: opt.step(x, [g[1], g[0]], lr=0.1),
                lambda: opt.step(x, [g[0].double(), g[1]], lr=0.1),
                lambda: opt.step(x, g, lr=0.1, factor=torch.ones(1).cuda()),
                lambda: opt.orthogonalize(g, out=g[:1]),
                lambda: opt.orthogonalize(torch.zeros(47).cuda())):
        with pytest.raises(ValueError):
            bad()
    mixed = arc.Muon(shapes, param_dtype=["f32", "bf16"])
    with pytest.raises(ValueError):
        mixed.orthogonalize(torch.zeros(48).cuda())
    assert [v.dtype for v in mixed.orthogonalize(g)] == [torch.float32, torch.bfloat16]
    L = _lib._lib
    table = (ctypes.c_void_p * 2)(x[0].data_ptr(), x[1].data_ptr())
    for sc in (arc.arc_muon_step_config(0.1, 0.9, 2, 0), arc.arc_muon_step_config(0.1, 0.9, 0, 1)):
        assert L.arc_muon_step(opt.ctx, ctypes.byref(sc), table, table, None, None,
                               opt.m.data_ptr()) == arc.ARC_ERR_INVALID
    sc = arc.arc_muon_step_config(0.1, 0.9, 1, 0)
    for m, factor in ((None, None), (opt.m.data_ptr() + 4, None),
                      (opt.m.data_ptr(), opt.m.data_ptr() + 8)):
        assert L.arc_muon_step(opt.ctx, ctypes.byref(sc), table, table, None, factor,
                               m) == arc.ARC_ERR_INVALID
    torch.cuda.synchronize()
