"""Orthogonalised matrices after replays of graphs of one context that overlapped in time
(which they must not): whatever those gave, no later call finds a count of parts that was
left behind."""
import pytest
import torch

import paper_2510_26709_amd as arc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# sums in parts in every one of them
@pytest.mark.parametrize("shapes", [[(257, 1001)], [(512, 4608)] * 3 + [(4608, 512), (64, 576)],
                                    [(33, 4000)] * 170])
def test_matrices_after_replays_that_overlapped(shapes):
    stream = torch.cuda.Stream()
    opt = arc.Muon(shapes, stream=stream)
    n = sum(r * c for r, c in shapes)
    u = torch.randn(n, device="cuda")
    x = torch.zeros(n, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        want = opt.orthogonalize(u)
        opt.step(x, u, lr=1.0, momentum=0.0, nesterov=False)
        stream.synchronize()
        stepped = x.clone()
        graphs = []
        for k in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                out = opt.orthogonalize(u)
                if k:
                    opt.step(x, u, lr=1.0, momentum=0.0, nesterov=False)
            graphs.append((graph, out, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for graph, _, on in graphs:
            with torch.cuda.stream(on):
                graph.replay()
    torch.cuda.synchronize()
    for _ in range(2):
        for graph, out, on in graphs:
            with torch.cuda.stream(on):
                x.zero_()
                out.fill_(7.0)
                graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
        assert torch.equal(x, stepped)
        with torch.cuda.stream(stream):
            got = opt.orthogonalize(u)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
