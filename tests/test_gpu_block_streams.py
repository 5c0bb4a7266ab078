"""The decoder block's classes on several streams, in several captured graphs and over many
batch sizes.

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


def small_block(seed=77):
    import moe_inputs as mi
    pkg = P()
    wk = mi.WORKLOADS["tiny"]
    d, Hq, Hkv, D = wk.layer.d_model, 4, 2, 64
    g = gen(seed)

    def w(*shape):
        return 0.05 * torch.randn(*shape, device="cuda", generator=g)
    return pkg.DecoderBlock(pkg.MoELayer(mi.LayerInputs(wk.layer), device="cuda:0"), w((Hq + 2 * Hkv) * D, d), w(d, Hq * D),
                            Hq, Hkv, D, dict(attn=1 + w(d), ffn=1 + w(d)), group=64), d


class Request:
    """One batch of tokens with a cache of its own through a block."""

    def __init__(self, block, d, T, seed, ctx=30):
        self.block, self.T = block, T
        self.cache = P().PagedCache.create(1, ctx + T, block.Hkv, block.D, page_size=32)
        self.cache.k.copy_(torch.randn(self.cache.k.shape, device="cuda", generator=gen(seed)))
        self.cache.v.copy_(torch.randn(self.cache.v.shape, device="cuda", generator=gen(seed + 1)))
        self.cache.lens.fill_(ctx)
        self.ctx = ctx
        self.off = torch.tensor([0, T], dtype=torch.int32, device="cuda")
        self.r0 = torch.randn(T, d, device="cuda", generator=gen(seed + 2))
        self.r, self.h = self.r0.clone(), torch.empty(T, d, dtype=BF16, device="cuda")
        self.reset()

    def reset(self):
        self.r.copy_(self.r0)
        P().moe_block_norm(self.r, self.h, w_pre=self.block.norms["attn"])

    def step(self, stream=None):
        self.block.forward(self.r, self.h, self.cache, self.off, self.T, self.ctx + self.T, stream=stream)

    def result(self):
        return self.r.clone(), self.h.clone()


def note_ffn_memory(monkeypatch):
    """Byte ranges that each call of the expert FFN writes."""
    from paper_2503_21135_amd import api
    seen = []
    call = api.moe_expert_ffn_mixed

    def noted(desc, x, k, offsets, perm, o, ws, **kw):
        seen.append([(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in (offsets, perm, o, ws)])
        return call(desc, x, k, offsets, perm, o, ws, **kw)
    monkeypatch.setattr(api, "moe_expert_ffn_mixed", noted)
    return seen


def disjoint(calls):
    ranges = [r for c in calls for r in c]
    return all(b <= c or d <= a for i, (a, b) in enumerate(ranges) for c, d in ranges[:i])


def test_block_on_two_streams(monkeypatch):
    """Two batches of equal size through one block on two streams give what they give alone."""
    block, d = small_block()
    reqs = [Request(block, d, 24, 100 + 10 * i) for i in range(2)]
    want = []
    for q in reqs:
        q.step()
        want.append(q.result())
        q.reset()
    torch.cuda.synchronize()
    seen = note_ffn_memory(monkeypatch)
    streams = [torch.cuda.Stream() for _ in reqs]
    for q, s in zip(reqs, streams):      # one after the other
        q.step(s)
        torch.cuda.synchronize()
    assert len(seen) == 2 and disjoint(seen), "calls on two streams share the expert layer's buffers"
    for _ in range(20):
        for q in reqs:
            q.reset()
        torch.cuda.synchronize()
        for q, s in zip(reqs, streams):
            q.step(s)
        torch.cuda.synchronize()
        for q, w in zip(reqs, want):
            assert all(torch.equal(a, b) for a, b in zip(q.result(), w))
    # and with each stream made the current one
    for q, s in zip(reqs, streams):
        q.reset()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            q.step()
        torch.cuda.synchronize()
    assert seen[-2:] == seen[:2]
    assert all(torch.equal(a, b) for q, w in zip(reqs, want) for a, b in zip(q.result(), w))


def test_block_in_two_captured_graphs(monkeypatch):
    """The same as two graphs that are replayed side by side, with eager calls next to them."""
    block, d = small_block(78)
    reqs = [Request(block, d, 24, 200 + 10 * i) for i in range(3)]
    want = []
    for q in reqs:
        q.step()
        want.append(q.result())
        q.reset()
    torch.cuda.synchronize()
    seen = note_ffn_memory(monkeypatch)
    graphs = [capture(q.step)[0] for q in reqs[:2]]
    reqs[2].step()
    torch.cuda.synchronize()
    assert len(seen) == 3 and disjoint(seen), "calls that may run side by side share the expert layer's buffers"
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(10):
        for q in reqs:
            q.reset()
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        reqs[2].step()
        torch.cuda.synchronize()
        for q, w in zip(reqs, want):
            assert all(torch.equal(a, b) for a, b in zip(q.result(), w))


def test_block_memory_stays_bounded_over_many_sizes():
    """Batches of ever other sizes through a block hold memory for the largest few times over,
    not for each size, and give what they give with buffers of their own."""
    block, d = small_block(79)
    torch.cuda.synchronize()
    sizes = list(range(1, 160))
    req = Request(block, d, 160, 300)

    def one(T):
        q = Request.__new__(Request)
        q.block, q.T, q.cache, q.ctx = block, T, req.cache, req.ctx
        q.off = torch.tensor([0, T], dtype=torch.int32, device="cuda")
        q.r, q.h = req.r0[:T].clone(), torch.empty(T, d, dtype=BF16, device="cuda")
        P().moe_block_norm(q.r, q.h, w_pre=block.norms["attn"])
        q.step()
        return q.r, q.h
    one(1)
    own = block.moe.new_buffers(160)
    largest = sum(t.numel() * t.element_size() for t in vars(own).values() if torch.is_tensor(t))
    del own
    before = torch.cuda.memory_allocated()
    first = {T: one(T) for T in (3, 40, 41)}
    for T in sizes + sizes[::-1]:
        one(T)
    again = {T: one(T) for T in first}
    assert all(torch.equal(a, b) for T in first for a, b in zip(first[T], again[T]))
    del first, again
    held = torch.cuda.memory_allocated() - before
    assert held <= 4 * largest, "%d bytes held, a batch of the largest size needs %d" % (held, largest)


@pytest.mark.parametrize("T,size,code", [(24, 1e6, 0), (700, 1.0, 0), (700, 1e6, -6)])
def test_block_tells_of_values_past_the_expert_layers_range(T, size, code):
    """Few tokens take any bf16 activation; many, whose operands are fp16, say so when one is
    beyond 65504 (a norm weight of 10^6 makes some)."""
    block, d = small_block(80)
    block.norms = dict(block.norms, ffn=torch.full((d,), size, device="cuda"))
    Request(block, d, T, 400).step()
    assert block.status_value() == code
    block.moe.clear_ffn_status()
    assert block.status_value() == 0
