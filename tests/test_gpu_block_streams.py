"""The decoder block's classes on several streams and in several captured graphs.

Nothing that would race is launched: what two calls that may run side by side are given to
work in is compared first."""
import pytest
import torch

from test_gpu_block import BF16, P, batch, gen

pytestmark = pytest.mark.gpu


def capture(step):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    return graph, out


def test_captured_graphs_of_one_cache_have_their_own_workspace(monkeypatch):
    """Two graphs and the eager calls of one cache never work in the same bytes, so the graphs
    may be replayed side by side."""
    from paper_2503_21135_amd import api
    cache, off = batch([4000], [1], 64, 2, 128, BF16, 95)
    qs = [torch.randn(1, 8, 128, device="cuda", generator=gen(i)).to(BF16) for i in range(3)]
    want = [cache.attend(q, off, 1, 4001) for q in qs]
    torch.cuda.synchronize()
    seen = []
    call = api.moe_tree_attention

    def noted(*args):
        ws = next(t for t in args if torch.is_tensor(t) and t.dtype is torch.uint8)
        seen.append((ws.data_ptr(), ws.data_ptr() + ws.numel()))
        return call(*args)
    monkeypatch.setattr(api, "moe_tree_attention", noted)
    side = torch.cuda.Stream()
    graphs = [capture(lambda q=q: cache.attend(q, off, 1, 4001)) for q in qs[:1]]
    graphs.append(capture(lambda: cache.attend(qs[1], off, 1, 4001, stream=torch.cuda.current_stream())))
    eager = [cache.attend(qs[2], off, 1, 4001)]
    with torch.cuda.stream(side):
        eager.append(cache.attend(qs[2], off, 1, 4001))
    torch.cuda.synchronize()
    assert len(seen) == 4
    for i, (a, b) in enumerate(seen):
        for c, d in seen[:i]:
            assert b <= c or d <= a, "two calls that may run side by side share their workspace"
    assert all(torch.equal(o, want[2]) for o in eager)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(20):
        for (graph, out), s in zip(graphs, streams):
            out.zero_()
        torch.cuda.synchronize()
        for (graph, out), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                for _ in range(4):
                    graph.replay()
        more = cache.attend(qs[2], off, 1, 4001)
        torch.cuda.synchronize()
        assert torch.equal(more, want[2])
        for (graph, out), w in zip(graphs, want):
            assert torch.equal(out, w)
