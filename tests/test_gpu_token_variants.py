"""The token kernels' variants, each by a row length and a number of rows that
choose it: more than 512 rows are not split, and their length decides the
workgroup's threads.  A few rows of different kinds are repeated: the first of
each is held to the formulas in 64 bits, the others to the first one's bits."""
import math

import pytest
import torch

import paper_2510_26709_amd as arc
from test_gpu_tokens import EPS, dtype_of, formulas, kind, near, place, tokens

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
CHUNKS = [100, 1500, 2900, 5000, 13_000]


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
