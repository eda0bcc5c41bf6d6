"""Norms after replays of graphs of one context that overlapped in time (which they must
not): whatever those gave, no later call finds a count that was left behind."""
import pytest
import torch

import paper_2510_26709_amd as arc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("sizes", [[1000], [7, 100_000, 0, 3, 5_000_000], [129] * 700])
def test_norms_after_replays_that_overlapped(sizes):
    stream = torch.cuda.Stream()
    opt = arc.AdamW(sizes, stream=stream)
    g = torch.randn(sum(sizes), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        want = opt.norm(g, max_norm=0.5)
        stream.synchronize()
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                out = opt.norm(g, max_norm=0.5)
            graphs.append((graph, out, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, _, on in graphs:
            with torch.cuda.stream(on):
                graph.replay()
    torch.cuda.synchronize()
    for graph, out, on in graphs:
        with torch.cuda.stream(on):
            out.total.fill_(7.0)
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.total, want.total) and torch.equal(out.norms, want.norms)
    for _ in range(2):
        with torch.cuda.stream(stream):
            got = opt.norm(g, max_norm=0.5)
        torch.cuda.synchronize()
        assert torch.equal(got.total, want.total) and torch.equal(got.norms, want.norms)
