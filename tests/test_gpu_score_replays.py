"""Scores of few long rows, whose pieces are joined by the last workgroup to arrive, after
replays of graphs of one context that overlapped in time (which they must not): whatever
those gave, no later call finds a count that was left behind."""
import pytest
import torch

import paper_2510_26709_amd as arc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("first,second", [(2, 2), (2, 100), (1, 200), (100, 500)])
def test_scores_after_replays_that_overlapped(first, second):
    """Rows of 131,077: up to 100 of them in eight pieces, 200 in five and 500 in two."""
    V, most = 131_077, 500
    stream = torch.cuda.Stream()
    head = arc.TokenLogProbs(V=V, rows=most, dtype="bf16", top=3, stream=stream)
    gen = torch.Generator(device="cuda").manual_seed(first)
    x = torch.randn(most, V, generator=gen, device="cuda").bfloat16()
    y = torch.randint(0, V, (most,), generator=gen, device="cuda")
    torch.cuda.synchronize()
    sizes = (first, second, 1, 2, 100, 200, 500)
    with torch.cuda.stream(stream):
        want = {n: head.score(x[:n], y[:n]) for n in sizes}
        stream.synchronize()
        graphs = []
        for n in (first, second):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                out = head.score(x[:n], y[:n])
            graphs.append((g, out, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for g, _, on in graphs:
            with torch.cuda.stream(on):
                g.replay()
    torch.cuda.synchronize()
    for n, (g, out, on) in zip((first, second), graphs):
        with torch.cuda.stream(on):
            g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want[n]):
            assert torch.equal(a, b), n
    for n in sizes:
        with torch.cuda.stream(stream):
            got = head.score(x[:n], y[:n])
        torch.cuda.synchronize()
        for a, b in zip(got, want[n]):
            assert torch.equal(a, b), n
