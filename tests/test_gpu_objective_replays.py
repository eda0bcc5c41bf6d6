"""Graphs captured from one token context share its workspace, and their replays must
not overlap in time.  Where they did, their own totals are what they are, but no call
after them finds a count that was left behind."""
import pytest
import torch

import paper_2510_26709_amd as arc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def calls(head, seed=2):
    """Calls of some numbers of workgroups: [(name, call)]; each returns its tuple."""
    gen = torch.Generator().manual_seed(seed)
    n = 100_003
    l = -torch.rand(n, generator=gen).cuda()
    A = torch.randn(n, generator=gen).cuda()
    y = torch.zeros(n, dtype=torch.int64).cuda()
    x = torch.randn(98, 501, generator=gen).cuda()
    pairs = (torch.arange(197) * 500).cuda()  # 98 pairs
    few = (torch.arange(9) * 12_000).cuda()   # 4 pairs, in parts
    more = (torch.arange(11) * 10_000).cuda()  # 5
    m = 40_000
    return [("98 workgroups", lambda: head.policy(l, y, A)),
            ("40 workgroups", lambda: head.policy(l[:m], y[:m], A[:m])),
            ("98 rows of logits", lambda: head.policy_loss(x, y[:98], A[:98])),
            ("97 rows of logits", lambda: head.policy_loss(x[:97], y[:97], A[:97])),
            ("98 pairs", lambda: head.preference(l, y, pairs)),
            ("4 pairs in parts", lambda: head.preference(l, y, few)),
            ("5 pairs in parts", lambda: head.preference(l, y, more))]


@pytest.mark.parametrize("first,second", [(0, 0), (0, 1), (0, 2), (2, 3), (1, 4), (2, 4), (5, 6)])
def test_calls_after_replays_that_overlapped(first, second):
    stream = torch.cuda.Stream()
    head = arc.TokenLogProbs(V=501, rows=100_003, dtype="f32", stream=stream)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        each = calls(head)
        stream.synchronize()
        want = [[None if t is None else t.clone() for t in call()] for _, call in each]
        stream.synchronize()
        graphs = []
        for k in (first, second):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                out = each[k][1]()
            graphs.append((g, out, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for g, _, on in graphs:
            with torch.cuda.stream(on):
                g.replay()
    torch.cuda.synchronize()
    for _ in range(2):
        for k, (g, out, on) in zip((first, second), graphs):  # one after the other again
            for t in out:
                if t is not None:
                    t.fill_(7.0)
            torch.cuda.synchronize()
            with torch.cuda.stream(on):
                g.replay()
            torch.cuda.synchronize()
            for a, b in zip(out, want[k]):
                assert b is None or torch.equal(a, b), each[k][0]
        with torch.cuda.stream(stream):
            for (name, call), expected in zip(each, want):
                got = call()
                stream.synchronize()
                for a, b in zip(got, expected):
                    assert b is None or torch.equal(a, b), name
