"""The objectives and optimizers together, as examples/align_lm.py runs them: it runs,
its model's gradients are those of the formulas, and a step moves the parameters by
them."""
import importlib.util
import math
import os

import pytest
import torch

import paper_2510_26709_amd as arc

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("align_lm",
                                                  os.path.join(ROOT, "examples", "align_lm.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("objective", ["policy", "preference"])
def test_it_runs(example, objective):
    first, last, totals = example.train(objective=objective, steps=6, rows=16, length=5)
    assert 0 <= first <= 1 and 0 <= last <= 1
    assert totals.numel() == (5 if objective == "policy" else 3)
    assert bool(torch.isfinite(totals).all())


def loss_in_64_bits(objective, parameters, x, given, extra):
    E, W, b, U = parameters
    h = torch.tanh(E[x] @ W + b)
    q = torch.log_softmax(h @ U.t(), 1)
    live = given >= 0
    logp = torch.where(live, q.gather(1, given.clamp(min=0)[:, None])[:, 0], 0.0)
    if objective == "preference":
        d = torch.where(live, logp - extra["ref"], 0.0).view(extra["rows"], -1).sum(1)
        P = extra["rows"] // 2
        return -torch.nn.functional.logsigmoid(0.3 * (d[:P] - d[P:])).mean()
    w = live.double() / live.sum()
    r = torch.exp(logp - extra["old"])
    gain = torch.minimum(r * extra["A"], r.clamp(0.8, 1.2) * extra["A"])
    away = extra["ref"] - logp
    H = -(q.exp() * q).sum(1)
    return (w * (-gain + 0.02 * (away.exp() - away - 1) - 1e-3 * H)).sum()


@pytest.mark.parametrize("objective", ["policy", "preference"])
def test_gradients_of_the_model(example, objective):
    """From logits through the library and the model's own products, against automatic
    differentiation of the same loss in 64 bits."""
    vocab, hidden, rows, prompt, length = 40, 16, 8, 2, 6
    device = torch.device("cuda:0")
    model = example.Model(vocab, hidden, device, seed=1)
    gen = torch.Generator(device=device).manual_seed(2)
    tokens = torch.randint(0, vocab, (rows, prompt + length), device=device, generator=gen)
    x, given = example.rows_of(tokens, prompt)
    T = x.numel()
    head = arc.TokenLogProbs(V=vocab, rows=T, dtype="f32", device=device)
    e, h = model.forward(x)
    logits = model.logits(h)
    scored = head.score(logits, given).logp
    noise = torch.randn(T, device=device, generator=gen)
    extra = {"ref": scored + 0.3 * noise, "rows": rows,
             "old": scored - 0.1 * noise.flip(0).clamp(-1.7, 1.7),
             "A": torch.randn(T, device=device, generator=gen)}
    if objective == "preference":
        offsets = torch.arange(rows + 1, device=device) * (prompt + length - 1)
        out = head.preference_loss(logits, given, offsets, ref_logp=extra["ref"], beta=0.3,
                                   scale=2.0 / rows)
    else:
        out = head.policy_loss(logits, given, extra["A"], old_logp=extra["old"],
                               ref_logp=extra["ref"], kl_coef=0.02, entropy_coef=1e-3,
                               scale=1.0 / int((given >= 0).sum()))
    grad = torch.empty_like(model.x)
    model.backward(x, e, h, out.grad, grad)
    want = [v.double().cpu().requires_grad_() for v in model.views(model.x)]
    loss = loss_in_64_bits(objective, want, x.cpu(), given.cpu(), {
        k: v.double().cpu() if isinstance(v, torch.Tensor) else v for k, v in extra.items()})
    loss.backward()
    # binary32 logits of magnitude 3 or so from sums of 16 terms, log probabilities
    # from them, sums of 56 rows: some 100 roundings of the largest element
    loss = float(loss.detach())
    assert abs(float(out.totals[0]) - loss) < 100 * 2.0 ** -24 * (1 + abs(loss))
    for got, w in zip(model.views(grad), want):
        tol = 100 * 2.0 ** -24 * float(w.grad.abs().max())
        assert float((got.double().cpu() - w.grad).abs().max()) < tol


def test_a_step_of_both_optimizers(example):
    """Clipped together, each tensor goes its optimizer's way."""
    device = torch.device("cuda:0")
    model = example.Model(50, 24, device, seed=1)
    opt = example.Optimizer(model, device)
    assert opt.matrices == [1] and opt.rest == [0, 2, 3]
    gen = torch.Generator(device=device).manual_seed(3)
    grad = torch.randn(model.x.shape, device=device, generator=gen)
    before = [v.clone() for v in model.views(model.x)]
    total = opt.step(0, grad, 0.01, 2)
    assert abs(float(total[0]) - 0.5 * float(grad.double().norm())) < 1e-4 * float(total[0])
    after, g = model.views(model.x), model.views(grad)
    for i in opt.rest:  # the first step of AdamW goes by the gradient's signs
        step = (before[i] - after[i]).double()
        assert float((step - 0.01 * torch.sign(g[i])).abs().max()) < 1e-4
    u = g[1].double()
    u = u / u.norm()
    for _ in range(5):
        a = u @ u.t()
        u = 3.4445 * u + (-4.7750 * a + 2.0315 * a @ a) @ u
    # coefficients in binary32, products as exact, x rounded
    assert float(((before[1] - after[1]).double() - 0.01 * u).abs().max()) < 1e-6
    assert math.isfinite(float(model.x.sum()))
