"""AdamW where v is near an end of binary32's range, and with any eps that is
accepted: the update's formula in 64 bits, of m and v in binary32 as they are
defined; 8-bit states there, bit by bit."""
import math

import numpy as np
import pytest
import torch

import paper_2510_26709_amd as arc
from test_gpu_optim import BLOCK, EPS, eight_bit_step, f32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def moments(m, v, g, factor, beta1, beta2):
    """m and v after a step, every product and sum rounded to binary32 by itself."""
    b1, b2 = np.float32(beta1), np.float32(beta2)
    with np.errstate(over="ignore", under="ignore"):
        g = g * np.float32(factor)
        return (b1 * m + (np.float32(1) - b1) * g,
                b2 * v + (np.float32(1) - b2) * (g * g))


def updated(x, m, v, t, lr, beta1, beta2, eps, decay):
    """x after the step and the size of its update, in 64 bits."""
    c1, c2 = 1 - f32(beta1) ** (t + 1), 1 - f32(beta2) ** (t + 1)
    with np.errstate(divide="ignore"):
        move = f32(lr) / c1 * m.astype(np.float64) / (
            np.sqrt(v.astype(np.float64)) / math.sqrt(c2) + f32(eps))
    return x.astype(np.float64) * (1 - f32(lr) * f32(decay)) - move, np.abs(move)


def gradients(n, lo, hi, seed):
    """Magnitudes spread evenly over their logarithm, of both signs."""
    rng = np.random.default_rng(seed)
    size = np.exp(rng.uniform(math.log(lo), math.log(hi), n))
    return (size * rng.choice([-1.0, 1.0], n)).astype(np.float32)


RANGES = [(1e-24, 1e-18), (1e-19, 1e-12), (1e16, 1.7e19), (1e19, 1e22), (1e21, 3e38)]


@pytest.mark.parametrize("state", ["f32", "f8"])
@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-30, 1e-20, 1e-8])
@pytest.mark.parametrize("lo,hi", RANGES)
@pytest.mark.parametrize("beta1,beta2", [(0.9, 0.95), (0.0, 0.0)])
def test_updates_at_both_ends_of_the_range(beta1, beta2, lo, hi, eps, state):
    n, lr, decay = 70_003, 1e-3, 0.1
    g = gradients(n, lo, hi, 3)
    x0 = np.random.default_rng(4).normal(size=n).astype(np.float32)
    zero = np.zeros(n, np.float32)
    m, v = moments(zero, zero, g, 0.5, beta1, beta2)
    want, move = updated(x0, m, v, 0, lr, beta1, beta2, eps, decay)
    opt = arc.AdamW([n], state=state, weight_decay=decay)
    x = torch.from_numpy(x0).cuda()
    opt.step(0, x, torch.from_numpy(g).cuda(), lr=lr, beta1=beta1, beta2=beta2, eps=eps,
             factor=torch.tensor([0.0, 0.5], device="cuda"))
    got = x.cpu().numpy().astype(np.float64)
    if state == "f32":
        assert np.array_equal(opt.m.cpu().numpy()[:n], m)
        assert np.array_equal(opt.v.cpu().numpy()[:n], v)
    # five roundings of about |x| and fewer than a dozen of the update
    off = np.abs(got - want) - EPS * (6 * np.abs(x0) + 24 * move)
    worst = int(np.argmax(off.astype(np.float64)))
    assert bool((off <= 0).all()), (worst, g[worst], got[worst], want[worst])


@pytest.mark.parametrize("lo,hi", [(1e-23, 1e-18), (1e-20, 1e-19), (1e-3, 1e3), (1e15, 1e18)])
def test_8_bit_states_at_both_ends_are_their_definition(lo, hi):
    n = 40 * BLOCK
    opt = arc.AdamW([n], state="f8", seed=5, weight_decay=0.0)
    x = torch.zeros(n, device="cuda")
    for t in range(3):
        g = gradients(n, lo, hi, 10 + t)
        m = (opt.m.float() * opt.m_scale.repeat_interleave(BLOCK)).cpu().numpy()
        u = (opt.v.float() * opt.v_scale.repeat_interleave(BLOCK)).cpu().numpy()
        with np.errstate(under="ignore"):
            qm, ms, qv, vs, root = eight_bit_step(m, u * u, g, n, 5, t, 0)
        opt.step(t, x, torch.from_numpy(g).cuda(), lr=1e-3, beta2=0.95)
        assert np.array_equal(opt.m_scale.cpu().numpy(), ms), t
        assert np.array_equal(opt.v_scale.cpu().numpy(), vs), t
        assert np.array_equal(opt.m.view(torch.uint8).cpu().numpy(), qm), t
        assert np.array_equal(opt.v.view(torch.uint8).cpu().numpy(), qv), t
        assert bool(((qv & 0x7F) > 0)[root > 0].all()), "a v above 0 stays above 0"


def test_an_infinite_v_of_32_bits_stays_and_its_parameter_only_decays():
    x = torch.full((300,), 2.0, device="cuda")
    g = torch.ones(300, device="cuda")
    g[7] = -1e25
    opt = arc.AdamW([300], weight_decay=0.5)
    for t in range(3):
        opt.step(t, x, g, lr=0.25)
    assert opt.v[7].item() == math.inf and math.isfinite(opt.m[7].item())
    want = 2.0
    for t in range(3):
        want *= 1 - 0.25 * 0.5
    assert x[7].item() == want
    assert bool(torch.isfinite(x).all()) and bool((x[8:] < want).all())


@pytest.mark.parametrize("value", [1e25, math.inf, -math.inf, math.nan])
def test_values_that_8_bits_do_not_hold_are_nan(value):
    """An infinite v, and what a gradient that is not finite makes of m and v."""
    x = torch.full((300,), 2.0, device="cuda")
    g = torch.ones(300, device="cuda")
    g[7] = value
    opt = arc.AdamW([300], state="f8", weight_decay=0.0)
    opt.step(0, x, g, lr=0.25)
    finite = math.isfinite(value)
    assert math.isnan(opt.v[7].float().item())
    assert math.isnan(opt.m[7].float().item()) != finite
    assert x[7].item() == 2.0 if finite else math.isnan(x[7].item())
    assert bool(torch.isfinite(x[8:]).all())
    assert bool(torch.isfinite(opt.v[BLOCK:].float()).all()), "other blocks"


@pytest.mark.parametrize("grads", ["f32", "bf16"])
def test_norms_of_more_tensors_than_one_launch_takes(grads):
    gen = torch.Generator().manual_seed(8)
    sizes = [int(k) for k in torch.randint(0, 3000, (1301,), generator=gen)]
    sizes[479] = sizes[480] = sizes[960] = 0
    sizes[1300] = 100_003
    opt = arc.AdamW(sizes, grad_dtype=grads)
    flat = torch.randn(sum(sizes), generator=gen)
    flat = flat.bfloat16() if grads == "bf16" else flat
    each = torch.stack([t.double().norm() for t in torch.split(flat, sizes)])
    total, norms = opt.norm(flat.cuda(), max_norm=1.0, scale=0.5)
    # a binary64 sum of exact squares, rounded once
    assert bool(((norms.cpu().double() - 0.5 * each).abs() <= 2 * EPS * each).all())
    norm = 0.5 * float(each.norm())
    assert abs(total[0].item() - norm) <= 2 * EPS * norm
    assert abs(total[1].item() - 0.5 / norm) <= 4 * EPS / norm
