"""The token kernels' variants, each by a row length and a number of rows that
choose it: more than 512 rows are not split, and their length decides the
workgroup's threads.  A few rows of different kinds are repeated: the first of
each is held to the formulas in 64 bits, the others to the first one's bits."""
import math

import pytest
import torch

import paper_2510_26709_amd as arc
from test_gpu_tokens import EPS, dtype_of, formulas, kind, near, tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def repeated(x, y, times, dtype, pad=0, shift=0):
    """Logits and targets `times` after one another, on the GPU.  (V + pad even:
    a row's sums have the same order wherever it begins at a whole word.)"""
    K, V = x.shape
    T = K * times
    buf = torch.full((shift + T * (V + pad),), math.nan, dtype=dtype_of(dtype), device="cuda")
    view = buf[shift:].view(T, V + pad)[:, :V]
    stored = x.to(dtype_of(dtype)).cuda()
    for lo in range(0, T, K):
        view[lo:lo + K] = stored
    return view, y.cuda().repeat(times)


def slack(x, scale):
    """Absolute error [T] of logp: relative errors of each exponent's argument (a
    difference and a product, at most 110 in magnitude where the exponential is
    not 0; one product more for a scale that is not 1), and of a sum whose
    longest chain is a lane's share of the row in a workgroup of 64, and joins."""
    z = x.double().cpu() * scale
    z = torch.where(torch.isfinite(z), z, -math.inf)
    most = z.amax(1, keepdim=True)
    live = torch.where(z >= most - 110, z, most)
    most = torch.where(most == -math.inf, 0.0, most)
    live = torch.where(live == -math.inf, 0.0, live)
    product = live.abs().amax(1) if scale != 1.0 else 0.0
    return EPS * (8 * (most - live).amax(1) + 4 * product + min(x.shape[1], 65_536) / 64 + 64)


def same_bits(name, got, K):
    for lo in range(K, got.shape[0], K):
        assert torch.equal(got[lo:lo + K].view(torch.int32), got[:K].view(torch.int32)), (
            f"{name}: rows {lo}.. differ from the same rows before")


def check_scores(x, y, K, scale, top, dtype):
    """Scores of rows of which the first K come again and again."""
    V = x.shape[1]
    h = arc.TokenLogProbs(V=V, rows=x.shape[0], dtype=dtype, top=top, scale=scale)
    got = h.score(x, y)
    torch.cuda.synchronize()
    for name, v in got._asdict().items():
        same_bits(name, v, K)
    head = [v[:K] for v in got]
    want = formulas(x[:K], y[:K], scale, top)
    tol = slack(x[:K], scale)
    large = lambda v: 4 * EPS * v.abs().nan_to_num(posinf=0.0)  # noqa: E731
    near("logp", head[0], want["logp"], tol + large(want["logp"]))
    near("entropy", head[1], want["entropy"], tol * (2 + 2 * math.log(V + 1)))
    near("lse", head[2], want["lse"], tol + large(want["lse"]))
    assert torch.equal(head[3].cpu().long(), want["top_ids"]), "alternatives"
    near("top_logp", head[4], want["top_logp"], tol[:, None] + large(want["top_logp"]))
    h.close()


# 16-byte chunks of a row, for workgroups of 64, 256, 256, 512 and 1024 threads.
CHUNKS = [100, 1500, 2900, 5000, 20_000]


def length(chunks, dtype):
    return chunks * (8 if dtype == "bf16" else 4) + 5


def floods(V, gen):
    """Rows with more logits at the bound of the alternatives than lists take, or
    with fewer live tokens than alternatives."""
    words = ["equal", "ties", "zeros of both signs", "ascending", "descending", "run of 100",
             "run of 300" if V < 3000 else "run of 3000"]
    rows = [kind(w, 1, V, gen)[0] for w in words]
    lowest = torch.finfo(torch.bfloat16).min
    for mask in (-math.inf, lowest, 0.0):
        for live in ([], [V - 1], [0, 1, 2, V // 2, V - 2], list(range(V // 7, V, V // 20))):
            row = torch.full((V,), mask)
            row[live] = torch.rand(len(live), generator=gen) + 1
            rows.append(row)
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("chunks", CHUNKS)
@pytest.mark.parametrize("top", [32, 1])
def test_rows_that_flood_the_lists_unsplit(top, chunks, dtype):
    V = length(chunks, dtype)
    x = floods(V, torch.Generator().manual_seed(chunks))
    K = x.shape[0]
    y = tokens(K, V, chunks)
    x, y = repeated(x, y, -(-513 // K), dtype, pad=3, shift=1)
    check_scores(x, y, K, 1.0, top, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("chunks", [2100, 6000, 40_000])
@pytest.mark.parametrize("times", [1, 13])
def test_rows_that_flood_the_lists_split(times, chunks, dtype):
    V = length(chunks, dtype)
    x = floods(V, torch.Generator().manual_seed(chunks))
    K = x.shape[0]
    x, y = repeated(x, tokens(K, V, chunks), times, dtype, pad=3)
    check_scores(x, y, K, 1.0, 32, dtype)


def mixed(V, gen):
    """Rows of every sort: noise, masked, non-finite, far from zero; their targets."""
    inf, nan = math.inf, math.nan
    x = torch.randn(14, V, generator=gen) * 3
    x[1, V // 2:] = -inf             # half masked
    x[2] = -inf                      # nothing left
    x[3, 1:] = -inf                  # one token left
    x[4, V - 1] = nan
    x[5, V // 3] = inf
    x[6, ::2] = -inf
    x[7, V // 3:] = torch.finfo(torch.bfloat16).min
    x[8] -= 1e4
    x[9, V // 2] += 200.0
    x[10] = 3e9 * x[10].sign()       # far from zero: the largest alone count
    x[11] = -1.0
    y = torch.tensor([V - 1, 0, 0, 0, 1, 7, 1, V // 3 - 1, V // 2, V // 2, 5, 2, -1, V + 3])
    return x, y


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("chunks", CHUNKS + [13_000, 40_000])
@pytest.mark.parametrize("top,scale", [(20, 1.0), (0, 0.7)])
def test_scores_of_rows_unsplit(top, scale, chunks, dtype):
    V = length(chunks, dtype)
    x, y = mixed(V, torch.Generator().manual_seed(chunks))
    K = x.shape[0]
    x, y = repeated(x, y, -(-513 // K), dtype, pad=3, shift=1)
    check_scores(x, y, K, scale, top, dtype)


def gradient(x, y, scale, want, ups, dtype):
    """The gradient of rows in 64 bits, and a bound of its error: p relative to the
    row's largest logit (its error is logp's), the entropy's, and the last
    roundings."""
    T, V = x.shape
    dl, dh, dz = (torch.zeros(T, dtype=torch.float64) if u is None else u.double().cpu()
                  for u in ups)
    y = y.cpu()
    dl = torch.where(y < 0, 0.0, dl)
    q, H = want["q"], want["entropy"]
    logq = torch.where(q > 0, want["logq"], 0.0)
    g = q * (dz - dl)[:, None] - dh[:, None] * q * (logq + H[:, None])
    at = (y >= 0) & (y < V)
    g[torch.arange(T)[at], y[at]] += dl[at]
    g *= scale
    g[((dl == 0) & (dh == 0) & (dz == 0)) | want["empty"]] = 0.0
    tol = slack(x, scale)[:, None]
    size = (dl.abs() + dz.abs() + dh.abs() * (H.abs().nan_to_num() + 2))[:, None] + \
        dh.abs()[:, None] * logq.abs().nan_to_num()
    p = q.nan_to_num()
    bound = scale * p * size * (4 * tol + 8 * EPS + 8 * EPS * logq.abs().nan_to_num())
    bound = bound + scale * dl.abs()[:, None] * 4 * EPS
    bound = bound + scale * dh.abs()[:, None] * p * tol * (4 + 2 * math.log(V + 1))
    if dtype == "bf16":
        bound = bound + (g.abs().nan_to_num() + bound) * 2.0 ** -8
    return g, bound + 1e-37


# Chunks up to which a workgroup's registers hold a row, each variant's first and
# last, and beyond them all (two launches).
LOSS_CHUNKS = [1, 512, 513, 1280, 1281, 4096, 4097, 8192, 8193, 12_288, 12_289, 24_576, 24_577]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("chunks", LOSS_CHUNKS)
@pytest.mark.parametrize("times", [1, 10])   # 14 rows (long ones: two launches), 140
def test_losses(times, chunks, dtype):
    V = chunks * (8 if dtype == "bf16" else 4) + 3
    gen = torch.Generator().manual_seed(chunks)
    x, y = mixed(V, gen)
    K, scale = x.shape[0], 1.25
    ups = torch.randn(3, K, generator=gen)
    ups[:, 11] = 0.0
    logits, targets = x, y
    x, y = repeated(logits, targets, times, dtype, pad=1)
    h = arc.TokenLogProbs(V=V, rows=x.shape[0], dtype=dtype, scale=scale)
    want = formulas(x[:K], y[:K], scale, 0)
    tol = slack(x[:K], scale)
    for which in ((0,), (0, 1, 2), (1,), (0, 2)):
        up = [ups[k].cuda().repeat(times) if k in which else None for k in range(3)]
        loss = h.loss(x, y, *up)
        z = repeated(logits, targets, times, dtype, pad=1)[0]
        inside = h.loss(z, y, *up, out=z)
        torch.cuda.synchronize()
        assert inside.grad.data_ptr() == z.data_ptr()
        for name in ("logp", "entropy", "lse"):
            a, b = getattr(loss, name), getattr(inside, name)
            assert torch.equal(a.view(torch.int32), b.view(torch.int32)), name
            same_bits(name, a, K)
        assert torch.equal(loss.grad.nan_to_num(nan=7.0), z.nan_to_num(nan=7.0)), "in place"
        for lo in range(K, x.shape[0], K):
            assert torch.equal(loss.grad[lo:lo + K].nan_to_num(nan=7.0),
                               loss.grad[:K].nan_to_num(nan=7.0)), lo
        large = lambda v: 4 * EPS * v.abs().nan_to_num(posinf=0.0)  # noqa: E731
        near("logp", loss.logp[:K], want["logp"], tol + large(want["logp"]))
        near("entropy", loss.entropy[:K], want["entropy"], tol * (2 + 2 * math.log(V + 1)))
        near("lse", loss.lse[:K], want["lse"], tol + large(want["lse"]))
        g, bound = gradient(x[:K], y[:K], scale, want, [None if u is None else u[:K] for u in up],
                            dtype)
        near("grad", loss.grad[:K], g, bound)
    h.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [(1 << 20) + 1000, (1 << 23) + 1000])
def test_more_rows_than_one_launch_takes(rows, dtype):
    V, scale = 9, 1.0
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(997, V, generator=gen) * 3
    y = torch.randint(-1, V, (997,), generator=gen)
    K, times = 997, -(-rows // 997)
    ups = torch.randn(3, K, generator=gen)
    x, y = repeated(x, y, times, dtype, pad=1)
    if rows < 1 << 21:
        check_scores(x, y, K, scale, 5, dtype)
    h = arc.TokenLogProbs(V=V, rows=x.shape[0], dtype=dtype, scale=scale)
    up = [u.cuda().repeat(times) for u in ups]
    s = h.score(x, y)
    want = formulas(x[:K], y[:K], scale, 0)
    g, bound = gradient(x[:K], y[:K], scale, want, [u[:K] for u in up], dtype)
    # (lse rounded to binary32: its own error in the exponent, of at most 16)
    bound = bound * 2 + 16 * 8 * EPS * g.abs()
    for grad in (h.grad(x, y, s.lse, s.entropy, *up), h.loss(x, y, *up).grad):
        near("grad", grad[:K], g, bound)
        assert torch.equal(grad.view(times, K, V), grad[:K].expand(times, K, V))
    for v in (s.logp, s.entropy, s.lse):
        assert torch.equal(v.view(times, K), v[:K].expand(times, K))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_longest_row(dtype):
    """2^31 - 1 logits, all equal but for three: the lists flood in every piece,
    the last of which ends where token numbers do."""
    V = (1 << 31) - 1
    x = torch.full((1, V), 0.25, dtype=dtype_of(dtype), device="cuda")
    y = torch.tensor([V - 2], device="cuda")
    for j, v in ((V - 1, 3.0), (V - 2, 2.0), (5, 1.0)):
        x[0, j] = v
    h = arc.TokenLogProbs(V=V, rows=1, dtype=dtype, top=8)
    got = h.score(x, y)
    assert got.top_ids.tolist() == [[V - 1, V - 2, 5, 0, 1, 2, 3, 4]]
    total = (V - 3) * math.exp(0.25) + math.exp(3) + math.exp(2) + math.exp(1)
    lse = math.log(total)
    # a lane's chain of at most V / 8192 terms, and joins
    tol = EPS * (V / 8192 + 64)
    near("lse", got.lse, torch.tensor([lse], dtype=torch.float64), tol)
    near("logp", got.logp, torch.tensor([2 - lse]), tol + 64 * EPS)
    near("top_logp", got.top_logp, torch.tensor([[3.0, 2, 1] + [0.25] * 5]) - lse, tol + 64 * EPS)
    grad = h.loss(x, y, torch.ones(1, device="cuda"), out=x).grad
    p = [math.exp(v - lse) for v in (0.25, 1.0, 2.0, 3.0)]
    want = torch.tensor([[-p[0], -p[1], 1 - p[2], -p[3], -p[0]]], dtype=torch.float64)
    at = [0, 5, V - 2, V - 1, V - 3]
    near("grad", grad[:, at], want, want.abs() * (tol + 64 * EPS + (dtype == "bf16") * 2.0 ** -8))
    assert int((grad == grad[0, 0]).sum()) == V - 3
