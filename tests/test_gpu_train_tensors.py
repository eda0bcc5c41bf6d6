"""Which memory the training operators' classes use, and for how long: states that
are assigned, tensors whose storage was replaced, tensors dropped while another
stream's call still uses them."""
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


def busy(stream):
    """About a second of work that touches no memory."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(1 << 31)


def token_calls(h, x, y, up):
    s = h.score(x, y)
    yield lambda a, b, c: h.score(a, b)
    yield lambda a, b, c: h.grad(a, b, s.lse, None, c)
    yield lambda a, b, c: h.loss(a, b, c)
    yield lambda a, b, c: h.loss(a, b, c, out=a)


@pytest.mark.parametrize("call", range(4))
def test_inputs_dropped_after_a_call_are_not_handed_out_while_it_runs(call):
    T, V = 64, 32768
    stream = torch.cuda.Stream()
    h = arc.TokenLogProbs(V=V, rows=T, dtype="f32", stream=stream)
    x, y = torch.zeros(T, V, device="cuda"), torch.zeros(T, dtype=torch.int64, device="cuda")
    up = torch.ones(T, device="cuda")
    torch.cuda.synchronize()
    make = list(token_calls(h, x, y, up))[call]
    torch.cuda.synchronize()
    busy(stream)
    out = make(x, y, up)
    assert not stream.query(), "the stream is still at work"
    used = [x, y, up] if call else [x, y]  # scores have no upstream gradient
    before = {t.data_ptr() for t in used}
    sizes = [(t.shape, t.dtype) for t in used]
    del x, y, used, out
    if call:
        del up
    after = [torch.empty(s, dtype=d, device="cuda") for s, d in sizes]
    assert not stream.query(), "the stream is still at work"
    assert not before & {t.data_ptr() for t in after}
    stream.synchronize()


@pytest.mark.parametrize("flat", [True, False])
@pytest.mark.parametrize("state", ["f32", "f8"])
def test_tensors_of_a_step_dropped_after_it_are_not_handed_out_while_it_runs(state, flat):
    sizes = [300_000, 700_000, 5_000_000]
    stream = torch.cuda.Stream()
    opt = arc.AdamW(sizes, state=state, stream=stream)

    def made(dtype=torch.float32):
        if flat:
            return torch.zeros(sum(sizes), dtype=dtype, device="cuda")
        return [torch.zeros(n, dtype=dtype, device="cuda") for n in sizes]

    x, g, c = made(), made(), made(torch.bfloat16)
    n = opt.m.numel()
    opt.m = torch.zeros(n, device="cuda").to(opt.m.dtype)  # the current stream's memory
    torch.cuda.synchronize()
    busy(stream)
    norms = opt.norm(g, max_norm=1.0)
    opt.step(0, x, g, lr=1e-2, factor=norms.total, copies=c)
    used = [t for v in (x, g, c) for t in ([v] if flat else v)] + [opt.m]
    before = {t.data_ptr() for t in used}
    shapes = [(t.shape, t.dtype) for t in used]
    opt.m = torch.zeros(n, device="cuda").to(opt.m.dtype)
    del x, g, c, used, norms
    after = [torch.empty(s, dtype=d, device="cuda") for s, d in shapes]
    assert not stream.query(), "the stream is still at work"
    assert not before & {t.data_ptr() for t in after}
    stream.synchronize()


def test_outputs_dropped_are_not_written_again_while_the_callers_stream_reads_them():
    T, V = 64, 1000
    stream = torch.cuda.Stream()
    h = arc.TokenLogProbs(V=V, rows=T, dtype="f32", top=5, stream=stream)
    x, y = torch.randn(T, V, device="cuda"), torch.zeros(T, dtype=torch.int64, device="cuda")
    other = torch.zeros_like(x)
    torch.cuda.synchronize()
    out = h.score(x, y)
    stream.synchronize()
    want = out.lse.clone()
    torch.cuda.synchronize()
    busy(torch.cuda.current_stream())
    got = out.lse.clone()
    at = out.logp.data_ptr()
    del out
    again = h.score(other, y)
    assert not torch.cuda.current_stream().query(), "the current stream is still at work"
    assert again.logp.data_ptr() != at
    torch.cuda.synchronize()
    assert torch.equal(got, want)
