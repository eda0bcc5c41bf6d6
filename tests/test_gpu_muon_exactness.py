"""How exact optimizer steps are, whose products of several steps' polynomials are taken
first: for matrices of few strong directions, whose others an error of X X' hits most."""
import math

import pytest
import torch

import paper_2510_26709_amd as arc
from test_gpu_muon import QUINTIC, allowed_error, matrices, polynomials

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def spread(m, n, s, seed):
    """A matrix of the singular values s."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q, _ = torch.linalg.qr(torch.randn(m, m, generator=gen, device="cuda", dtype=torch.float64))
    r, _ = torch.linalg.qr(torch.randn(n, m, generator=gen, device="cuda", dtype=torch.float64))
    return ((q * s) @ r.t()).float()


def spectra(m):
    one = torch.ones(m, device="cuda", dtype=torch.float64)
    for small in (0.3, 0.1, 0.06, 0.03, 0.01, 0.003):
        for big in sorted({1, 2, max(1, m // 4), m // 2}):
            if big < m:
                yield torch.where(torch.arange(m, device="cuda") < big, 1.0, small * one)
    yield torch.arange(1, m + 1, device="cuda", dtype=torch.float64) ** -1.5


# An error d of X X', up to 1.2 * 2^-24 of elements up to 1 (a pair's rounding and a sum's of
# blocks), grows 3.4445^2 = 12 times in a run of two, and goes into a direction of O by
# 4.775 / 3.4445 of that.
RUN_LOSES = 12 * 1.2 * 2.0 ** -24 * 4.775 / 3.4445


def check(u, **kw):
    """Steps from zero with lr 1 are -O.  Beside large matrices, with which steps are taken
    in runs (O alone, step by step, has other bits)."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    large = [torch.randn(1001, 1003, generator=gen, device="cuda") for _ in range(4)]
    opt = arc.Muon([tuple(x.shape) for x in u + large], lr_scale=1.0, **kw)
    x = [torch.zeros_like(v) for v in u + large]
    opt.step(x, u + large, lr=1.0, momentum=0.0, nesterov=False)
    alone = opt.orthogonalize(u + large)
    opt.close()
    for k, (v, got) in enumerate(zip(u, x)):
        want = polynomials(v, **kw)
        size = float(want.norm())
        off = float((-got.double() - want).norm())
        allowed = RUN_LOSES * size + allowed_error(v, want, **kw)
        assert off <= allowed, f"{k}: off by {off / size:.2e}, allowed {allowed / size:.2e}"
    return not torch.equal(alone[-1], -x[-1])


@pytest.mark.parametrize("m,n", [(2, 16_384), (4, 16_384), (4, 65_536), (16, 500), (16, 16_384),
                                 (16, 65_536), (64, 4096), (64, 16_384), (128, 4096),
                                 (300, 4000)])
def test_few_strong_directions(m, n):
    u = [spread(m, n, s, k) for k, s in enumerate(spectra(m))]
    in_runs = check(u + [v for k in range(2) for v in matrices([(m, n)], k)])
    assert in_runs or n < 1000


@pytest.mark.parametrize("steps,coefficients", [
    (3, QUINTIC), (4, QUINTIC), (6, QUINTIC), (8, (1.5, -0.5, 0.0)),
    (3, [(7.443, -29.711, 23.721), (6.68, -11.923, 4.256), (0.9, -0.15, 0.011)]),
    (3, [(7.5, -20.0, 13.4), (4.0, -2.8, 0.5), (1.2, -0.4, 0.05)])])
def test_other_runs(steps, coefficients):
    u = [spread(16, 8192, s, k) for k, s in enumerate(spectra(16)) if k % 3 == 0]
    check(u, steps=steps, coefficients=coefficients)


@pytest.mark.parametrize("m,n", [(4, 16_384), (64, 4096), (128, 4096), (300, 4000)])
def test_bfloat16_results(m, n):
    """In runs of three, whose error is within 1e-4 of the norm: beside what the rounding
    to bfloat16 is off by, some 1.7e-3, less than 1% more."""
    u = [spread(m, n, s, k) for k, s in enumerate(spectra(m))]
    gen = torch.Generator(device="cuda").manual_seed(1)
    large = [torch.randn(1001, 1003, generator=gen, device="cuda") for _ in range(4)]
    opt = arc.Muon([tuple(x.shape) for x in u + large], param_dtype="bf16")
    got = opt.orthogonalize(u + large)
    for v, x in zip(u, got):
        want = polynomials(v)
        rounding = float((want.bfloat16().double() - want).norm())
        off = float((x.double() - want).norm())
        assert off <= math.hypot(rounding, 1e-4 * float(want.norm())) + \
            allowed_error(v, want), (off, rounding)
        # and no element further than its rounding and 12 times the root of the mean square
        each = (x.double() - want).abs() - want.abs() * 2.0 ** -8
        assert float(each.max()) <= 12 * (1e-4 * float(want.norm()) + allowed_error(v, want)) \
            / math.sqrt(v.numel())


@pytest.mark.parametrize("m,n", [(1, 2_097_152), (16, 2_097_152), (64, 524_288), (130, 262_144)])
def test_long_sums(m, n):
    """In blocks, whose number is about that of a block's lines: 2^-24 times the root of the
    768 additions of a block and of 256 blocks, 2e-6, and as much for the pairs (sums of
    2^21 numbers one after the other are off by 1e-5 and more)."""
    for seed in range(2):
        u, = matrices([(m, n)], seed)
        opt = arc.Muon([(m, n)], lr_scale=1.0)
        x = torch.zeros_like(u)
        opt.step([x], [u], lr=1.0, momentum=0.0, nesterov=False)
        want = polynomials(u)
        for got in (opt.orthogonalize([u])[0], -x):
            off, size = float((got.double() - want).norm()), float(want.norm())
            assert off <= 4e-6 * size, f"off by {off / size:.2e}"
        opt.close()
