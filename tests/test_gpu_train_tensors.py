"""Which memory the training operators' classes use: states that are assigned,
tensors whose storage was replaced."""
import pytest
import torch

import paper_2510_26709_amd as arc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def names(state):
    return ("m", "v") if state == "f32" else ("m", "v", "m_scale", "v_scale")


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("state", ["f32", "f8"])
@pytest.mark.parametrize("how", ["assigned", "data"])
def test_states_that_are_replaced_are_the_ones_that_steps_use(how, state):
    """A run that is continued from a checkpoint by assigning its states."""
    sizes = [300, 5000]
    g = torch.randn(5300, generator=torch.Generator().manual_seed(1)).cuda()
    x = torch.zeros(5300, device="cuda")
    a = arc.AdamW(sizes, state=state, seed=4)
    a.step(0, x, g, lr=1e-2)
    checkpoint = {k: getattr(a, k).clone() for k in names(state)}
    at = x.clone()
    a.step(1, x, g, lr=1e-2)

    b = arc.AdamW(sizes, state=state, seed=4)
    before = {k: getattr(b, k).view(torch.uint8).detach() for k in names(state)}  # kept alive
    for k, v in checkpoint.items():
        if how == "assigned":
            setattr(b, k, v)
            assert getattr(b, k) is v
        else:
            getattr(b, k).data = v
    b.step(1, at, g, lr=1e-2)
    assert torch.equal(at, x)
    assert all(same(getattr(a, k), getattr(b, k)) for k in names(state))
    assert all(same(getattr(b, k), checkpoint[k]) for k in names(state))
    assert not any(bool(v.any()) for v in before.values())


@pytest.mark.parametrize("state", ["f32", "f8"])
def test_states_of_another_kind_are_refused(state):
    opt = arc.AdamW([300, 5000], state=state)
    n = opt.m.numel()
    kept = opt.m
    for bad in (torch.zeros(n, device="cuda", dtype=torch.float16),
                opt.m[:-128], torch.zeros(n).to(opt.m.dtype),
                torch.zeros(2 * n, device="cuda").to(opt.m.dtype)[::2]):
        with pytest.raises(ValueError):
            opt.m = bad
    if state == "f32":
        with pytest.raises(ValueError):
            opt.m_scale = torch.zeros(n // 128, device="cuda")
        assert opt.m_scale is None
    assert opt.m is kept
    x, g = torch.zeros(5300, device="cuda"), torch.zeros(5300, device="cuda")
    opt.step(0, x, g, lr=1e-2)
    opt.v.data = opt.v[:-128]   # the same address
    with pytest.raises(ValueError):
        opt.step(1, x, torch.ones_like(x), lr=1e-2)
    assert not bool(x.any())
