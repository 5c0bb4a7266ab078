"""Verification of drafts against the walk taken one draft at a time in 64 bits."""
import math
import random

import pytest
import torch

from test_gpu_block import BF16, FP16, FP32, P, gen

pytestmark = pytest.mark.gpu


def want_of(logits, tokens, off, parents, draft, u, u_next, heat, max_new):
    """(keep, n_keep, next) by the definition, sequence by sequence."""
    V, keep, count, last = logits.shape[1], [], [], []
    for b in range(len(off) - 1):
        first, n = off[b], off[b + 1] - off[b]
        t = 1.0 if heat is None else float(heat[b])
        greedy = u is None or t == 0
        path, cur = [0] if n else [], 0

        def p_of(i):
            x = logits[first + i].double()
            if not t >= 0 or math.isinf(t) or x.isnan().any() or (x == math.inf).any() or (x == -math.inf).all():
                return None
            if greedy:
                r = torch.zeros(V, dtype=torch.float64)
                r[int((x == x.max()).nonzero()[0])] = 1
                return r
            e = ((x - x.max()) / t).exp()
            return e / e.sum()
        r = p_of(0) if n else None
        for i in range(1, n):
            par = i - 1 if parents is None else parents[first + i]
            x = int(tokens[first + i])
            if r is None or par != cur or not 0 <= x < V:
                continue
            d = torch.zeros(V, dtype=torch.float64)
            if draft is None or greedy:
                d[x] = 1
            else:
                d = draft[first + cur].double()
            ui = 0.5 if greedy else min(max(float(u[first + i]), 0.0), 1 - 2.0 ** -24)
            if ui * d[x] < r[x]:
                cur = i
                path.append(i)
                r = p_of(i)
            else:
                left = (r - d).clamp(min=0)
                if left.sum() > 0:
                    r = left / left.sum()
        if r is None:
            last.append(-1)
        elif greedy:
            last.append(int(r.argmax()))
        else:
            up = r.cumsum(0)
            aim = min(max(float(u_next[b]), 0.0), 1 - 2.0 ** -24) * up[-1]
            last.append(int((up <= aim).sum()))
        keep.append(path + [-1] * (max_new - len(path)))
        count.append(len(path))
    return keep, count, last


def drafts(new, V, kind, seed, dt=FP32, draft_dt=None, spread=2.0, noise=0.7, fan=3):
    """A batch of trees (kind: chain, tree, or wide with many drafts below a token)."""
    r, g = random.Random(seed), gen(seed)
    off = [sum(new[:b]) for b in range(len(new) + 1)]
    N = off[-1]
    guess = spread * torch.randn(N, V, device="cuda", generator=g)
    logits = (guess + noise * torch.randn(N, V, device="cuda", generator=g)).to(dt)
    parents = []
    for n in new:
        for i in range(n):
            parents.append(-1 if i == 0 else i - 1 if kind == "chain" else r.randint(max(0, i - fan), i - 1) if kind == "tree" else (i - 1) // fan)
    q = torch.softmax(guess, 1)
    above = torch.tensor([off[b] + max(0, parents[off[b] + i]) for b, n in enumerate(new) for i in range(n)], device="cuda")
    if draft_dt is not None:
        q = q.to(draft_dt)
    pick = torch.multinomial(q[above].float(), 1, generator=g)[:, 0] if N else torch.zeros(0, device="cuda")
    if draft_dt is None and N:   # picked: the likeliest, with repeats among siblings
        pick = torch.where(torch.rand(N, device="cuda", generator=g) < 0.7, q[above].argmax(1), pick)
    u, last = torch.rand(N, device="cuda", generator=g), torch.rand(len(new), device="cuda", generator=g)
    return dict(logits=logits, tokens=pick.int(), off=off, parents=None if kind == "chain" else parents,
                draft=q if draft_dt is not None else None, u=u, last=last)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def check(s, max_new, heat=None, greedy=False, **kw):
    v = P().DraftVerifier()
    u, last = (None, None) if greedy else (s["u"], s["last"])
    par = None if s["parents"] is None else i32(s["parents"])
    args = dict(parents=par, draft_probs=s["draft"], u=u, u_next=last, temperature=heat, **kw)
    keep, n, nxt = v(s["logits"], s["tokens"], i32(s["off"]), max_new, **args)
    want = want_of(s["logits"].cpu(), s["tokens"].cpu(), s["off"], s["parents"], None if s["draft"] is None else s["draft"].cpu(),
                   None if u is None else u.cpu(), None if last is None else last.cpu(), heat, max_new)
    got = keep.tolist(), n.tolist(), nxt.tolist()
    for a, b, what in zip(got, want, ("keep", "n_keep", "next")):
        assert a == b, (what, [(i, x, y) for i, (x, y) in enumerate(zip(a, b)) if x != y][:4])
    again = v(s["logits"], s["tokens"], i32(s["off"]), max_new, **args)
    assert all(torch.equal(a, b) for a, b in zip(again, (keep, n, nxt)))
    return v, got


CASES = [
    # new, vocabulary, kind, type, draft type
    ([1], 1, "chain", FP32, None), ([1], 5, "chain", BF16, None), ([2, 1, 0, 5], 300, "chain", FP16, FP32),
    ([8] * 20, 1000, "chain", BF16, BF16), ([5], 32000, "chain", FP32, None), ([9, 3], 4096, "chain", FP32, FP16),
    ([16] * 12, 501, "tree", FP32, FP32), ([16] * 12, 4097, "wide", BF16, FP32), ([31, 2, 0, 17], 8193, "tree", FP16, None),
    ([40, 40], 33, "wide", FP32, None), ([100], 777, "tree", FP32, BF16), ([6] * 3, 131073, "wide", BF16, BF16),
    ([1024], 64, "tree", FP32, FP32), ([3] * 300, 257, "wide", FP32, FP32)]


@pytest.mark.parametrize("new,V,kind,dt,draft_dt", CASES)
def test_verify(new, V, kind, dt, draft_dt):
    s = drafts(new, V, kind, 3 + V, dt, draft_dt)
    v, (keep, n, nxt) = check(s, max(new))
    assert v.status_value() == 0
    check(s, max(new) + 2 if max(new) < 1023 else 1024, greedy=True)
    heat = (0.3 + 1.5 * torch.rand(len(new), device="cuda", generator=gen(1)))
    heat[::4] = 0
    check(s, max(new), heat=heat)


def test_some_are_accepted_and_some_are_not():
    """The batches above cover both, at every depth and place among siblings."""
    got, refused_then_accepted = [], 0
    for kind, draft_dt in (("chain", FP32), ("wide", FP32), ("wide", None)):
        s = drafts([16] * 64, 200, kind, 11, FP32, draft_dt, noise=0.4)
        _, (keep, n, _) = check(s, 16)
        got += n
        if kind == "wide":
            for k in keep:
                refused_then_accepted += any(k[i] > 0 and (k[i] - 1) % 3 > 0 for i in range(1, 16))
    assert min(got) == 1 and max(got) >= 5 and refused_then_accepted > 20


@pytest.mark.parametrize("kind,draft_dt", [("chain", FP32), ("chain", None), ("tree", FP32), ("tree", None)])
def test_walks_longer_than_a_wave(kind, draft_dt):
    new = [300, 1, 64, 65, 130]
    s = drafts(new, 40, kind, 23, FP32, draft_dt, spread=4.0, noise=0.002, fan=70)
    _, (_, n, _) = check(s, 300)
    assert kind == "tree" or draft_dt is None or n[0] > 64
    # every draft the likeliest below its parent: a chain is kept whole, of a tree the eldest
    up = [s["off"][b] + (i - 1 if s["parents"] is None else s["parents"][s["off"][b] + i]) for b, m in enumerate(new) for i in range(m)]
    s["tokens"] = s["logits"][torch.tensor(up, device="cuda").clamp(min=0)].argmax(1).int()
    _, (_, n, _) = check(s, 300, greedy=True)
    assert kind == "tree" or n == new
    check(s, 300)     # picked ones are the same among siblings


@pytest.mark.parametrize("kind,draft_dt", [("chain", FP32), ("wide", BF16), ("wide", None)])
def test_ruled_out_tokens(kind, draft_dt):
    """-infinity, in all but a few places; and rows with an offset that suits no exponential."""
    s = drafts([9] * 30, 3000, kind, 5, FP32, draft_dt)
    s["logits"].masked_fill_(torch.rand(s["logits"].shape, device="cuda", generator=gen(2)) < 0.99, -math.inf)
    s["logits"][:, 7] = 0.0
    s["logits"] += torch.linspace(-1e4, 1e4, s["logits"].shape[0], device="cuda")[:, None]
    v, (_, _, nxt) = check(s, 9)
    assert v.status_value() == 0
    last = [s["off"][b] + max(k) for b, k in enumerate(check(s, 9)[1][0])]
    assert all(s["logits"][i, t].item() > -math.inf for i, t in zip(last, nxt))
    # a single token left
    s["logits"].fill_(-math.inf)
    s["logits"][:, 1234] = -3e38
    check(s, 9)


def test_rows_without_a_distribution():
    s = drafts([4] * 8, 5000, "chain", 6, FP32, FP32, noise=0.0)
    s["u"].zero_()        # everything possible is accepted
    for row, val in ((0, math.nan), (5, math.inf), (10, math.nan), (15, math.inf)):
        s["logits"][row, 4999] = val
    s["logits"][18] = -math.inf
    heat = torch.ones(8, device="cuda")
    heat[5], heat[6], heat[7] = -1.0, math.nan, math.inf
    v, (keep, n, nxt) = check(s, 4, heat=heat)
    assert v.status_value() == -6
    assert n == [1, 2, 3, 4, 3, 1, 1, 1] and nxt == [-1] * 8
    v, (keep, n, nxt) = check(s, 4, greedy=True)
    assert v.status_value() == -6 and nxt[0] == -1


def test_tokens_parents_and_rows_out_of_range():
    s = drafts([6] * 4, 100, "wide", 8, FP32, FP32, noise=0.0)
    s["u"].zero_()
    s["tokens"][[1, 2]] = i32([-1, 100])
    s["tokens"][[0, 6, 12]] = i32([-9, 10 ** 9, 100])     # the first rows' tokens are not read
    s["parents"][7] = 3                                  # not below its own index
    s["parents"][13] = -1
    v, _ = check(s, 6)
    assert v.status_value() == -5
    s["parents"][7], s["parents"][8] = 1, -7
    v, _ = check(s, 6)
    assert v.status_value() == -5
    # a sequence whose rows are not there, and one with more than max_new
    good = drafts([3, 3, 3], 100, "chain", 9, FP32, FP32)
    _, (keep, n, nxt) = check(good, 3)
    for off in ([0, 3, 10, 9], [0, 3, 2, 9], [-1, 3, 6, 9]):
        v = P().DraftVerifier()
        k2, n2, x2 = v(good["logits"], good["tokens"], i32(off), 3, draft_probs=good["draft"], u=good["u"], u_next=good["last"])
        assert v.status_value() == -5
        for b in range(3):
            if off[b:b + 2] == good["off"][b:b + 2]:
                assert k2[b].tolist() == keep[b] and int(x2[b]) == nxt[b]
            elif not 0 <= off[b + 1] - off[b] <= 3 or off[b] < 0 or off[b + 1] > 9:
                assert int(n2[b]) == 0 and int(x2[b]) == -1 and (k2[b] == -1).all()


def test_no_rows_and_no_sequences():
    v = P().DraftVerifier()
    f = torch.zeros
    keep, n, nxt = v(f(0, 50, device="cuda"), i32([]), i32([0]), 3)
    assert keep.shape == (0, 3) and n.numel() == nxt.numel() == 0
    for u in (None, f(0, device="cuda")):
        keep, n, nxt = v(f(0, 50, device="cuda"), i32([]), i32([0, 0, 0]), 3, u=u, u_next=None if u is None else f(2, device="cuda"))
        assert keep.tolist() == [[-1] * 3] * 2 and n.tolist() == [0, 0] and nxt.tolist() == [-1, -1]
    keep, n, nxt = v(f(2, 50, device="cuda"), i32([1, 1]), i32([0, 1, 2]), 0)     # rows that max_new leaves out
    assert keep.shape == (2, 0) and n.tolist() == [0, 0] and nxt.tolist() == [-1, -1]
    assert v.status_value() == -5     # MOE_ERR_SLOT


def test_edges_of_the_random_numbers():
    """0, the largest below 1, and numbers outside, which count as the nearest inside."""
    s = drafts([4] * 6, 50, "chain", 12, FP32, FP32)
    s["logits"][:, :3] = -math.inf
    s["logits"][:, -4:] = -math.inf
    top = 1 - 2.0 ** -24
    s["last"] = torch.tensor([0.0, top, 1.0, -3.0, math.inf, 0.5], device="cuda")
    s["u"][:12:2], s["u"][1:12:2] = 0.0, top
    s["u"][12:16], s["u"][16:20] = 7.0, -1.0
    _, (_, _, nxt) = check(s, 4)
    assert all(3 <= x < 46 for x in nxt)
    # NaN counts as 0
    s["u"][:] = math.nan
    a = P().DraftVerifier()(s["logits"], s["tokens"], i32(s["off"]), 4, draft_probs=s["draft"], u=s["u"], u_next=s["last"])
    s["u"][:] = 0.0
    b = P().DraftVerifier()(s["logits"], s["tokens"], i32(s["off"]), 4, draft_probs=s["draft"], u=s["u"], u_next=s["last"])
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_draft_and_model_agree():
    """The same distribution on both sides: everything is accepted, and where all of it has been
    refused by a draft of another one, what was there before is drawn from."""
    s = drafts([5] * 40, 600, "chain", 13, FP32, FP32, noise=0.0)
    s["u"].clamp_(max=0.999)
    _, (_, n, _) = check(s, 5)
    assert n == [5] * 40
    s["draft"].fill_(1.0)          # covers every probability, so nothing remains when it refuses
    s["u"].fill_(top := 1 - 2.0 ** -24)
    assert top < 1
    _, (_, n, _) = check(s, 5)
    assert min(n) == 1
    wide = drafts([7] * 10, 600, "wide", 14, FP32, FP32)
    wide["draft"].fill_(1.0)
    wide["u"].fill_(top)
    check(wide, 7)


@pytest.mark.parametrize("heat", [1e-45, 1e-38, 1e-20, 1e-3, 1e3, 3e38])
def test_temperatures_of_any_size(heat):
    s = drafts([5] * 10, 3000, "wide", 19, FP32, FP32)
    s["logits"][3] *= 1e30
    check(s, 5, heat=torch.full((10,), heat, device="cuda"))


def test_graphs_and_eager_calls_work_in_memory_of_their_own(monkeypatch):
    from paper_2503_21135_amd import api
    s = drafts([8] * 6, 5000, "wide", 16, FP32, FP32)
    v, off, par, seen = P().DraftVerifier(), i32(s["off"]), i32(s["parents"]), []
    call = api.moe_draft_verify

    def noted(*args):
        ws = next(t for t in args if torch.is_tensor(t) and t.dtype is torch.uint8)
        seen.append((ws.data_ptr(), ws.data_ptr() + ws.numel()))
        return call(*args)
    monkeypatch.setattr(api, "moe_draft_verify", noted)

    def step():
        return v(s["logits"], s["tokens"], off, 8, parents=par, draft_probs=s["draft"], u=s["u"], u_next=s["last"])
    want, graphs = step(), []
    torch.cuda.synchronize()
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = step()
    assert len(seen) == 4 and all(b <= c or d <= a for i, (a, b) in enumerate(seen) for c, d in seen[:i])
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(10):
        for (g, _), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        more = step()
        torch.cuda.synchronize()
        for out in [more, other] + [o for _, o in graphs]:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_greedy_ties_go_to_the_first():
    logits = torch.zeros(6, 9000, device="cuda")
    logits[:, [8999, 5000, 4096, 17]] = 4.0
    logits[1, 17] = 0.0
    s = dict(logits=logits, tokens=i32([0, 17, 4096, 17, 17, 5000]), off=[0, 6], parents=None, draft=None)
    _, (keep, n, nxt) = check(s, 6, greedy=True)
    assert keep == [[0, 1, 2, 3, 4, -1]] and nxt == [17]


@pytest.mark.parametrize("draft_dt", [None, FP32])
def test_what_comes_out_is_distributed_as_the_model_says(draft_dt):
    """40000 sequences of one text with independent random numbers: the first token that comes
    out has the model's distribution (each count within five of its standard deviations)."""
    V, B, n = 12, 40000, 4      # three drafts below the known token
    g = gen(21)
    logits = torch.randn(1, V, device="cuda", generator=g).mul(1.5).expand(B * n, V).contiguous()
    guess = torch.randn(1, V, device="cuda", generator=g).mul(1.5).softmax(1)
    tokens = torch.multinomial(guess.expand(B * n, V), 1, generator=g)[:, 0].int() if draft_dt is not None else \
        guess.topk(n - 1).indices.repeat(B, 1).int()
    if draft_dt is None:
        tokens = torch.cat((torch.zeros(B, 1, dtype=torch.int32, device="cuda"), tokens.view(B, n - 1)), 1).flatten()
    off = torch.arange(0, B * n + 1, n, device="cuda").int()
    keep, count, nxt = P().DraftVerifier()(
        logits, tokens, off, n, parents=i32([-1, 0, 0, 0]).repeat(B), u=torch.rand(B * n, device="cuda", generator=g),
        u_next=torch.rand(B, device="cuda", generator=g), draft_probs=None if draft_dt is None else guess.expand(B * n, V).contiguous())
    one = tokens.view(B, n).gather(1, keep[:, 1:2].clamp(min=0).long())[:, 0]
    out = torch.where(count > 1, one, nxt)
    p = logits[0].double().softmax(0)
    hist = torch.bincount(out.long(), minlength=V).double()
    assert ((hist - B * p).abs() <= 5 * (B * p * (1 - p)).sqrt() + 1).all()
    assert 0.2 * B < (count > 1).sum() < 0.99 * B


def test_rows_past_32_bits_and_strides():
    V, ld = 1000, (1 << 30) + 8
    far = torch.empty(3 * ld + V, device="cuda").as_strided((4, V), (ld, 1))
    s = drafts([4], V, "chain", 15, FP32, FP32)
    _, want = check(s, 4)
    far.copy_(s["logits"])
    check(dict(s, logits=far), 4)
    del far
    wide = torch.full((4, V + 3), math.nan, device="cuda").to(BF16)
    wide[:, 1:-2] = s["logits"].to(BF16)
    room = torch.full((4, V + 9), math.nan, device="cuda")
    room[:, 4:-5] = s["draft"]
    check(dict(s, logits=wide[:, 1:-2], draft=room[:, 4:-5]), 4)


def test_streams_and_a_captured_graph():
    s = drafts([8] * 6, 5000, "wide", 16, FP32, FP32)
    v, off, par = P().DraftVerifier(), i32(s["off"]), i32(s["parents"])

    def step(stream=None):
        return v(s["logits"], s["tokens"], off, 8, parents=par, draft_probs=s["draft"], u=s["u"], u_next=s["last"], stream=stream)
    want = step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [step(streams[i % 2]) for i in range(10)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs for a, b in zip(o, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    big = drafts([8] * 12, 9000, "chain", 17)
    v(big["logits"], big["tokens"], i32(big["off"]), 8, u=big["u"], u_next=big["last"])    # a larger workspace
    for i in range(4):
        s["u"].copy_(torch.rand(48, device="cuda", generator=gen(30 + i)))
        s["logits"].copy_(torch.randn(48, 5000, device="cuda", generator=gen(40 + i)))
        want = [t.clone() for t in step()]
        for t in got:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert v.status_value() == 0


def test_kept_drafts_go_to_the_cache():
    """The verifier's lists are what the caches' keep takes."""
    s = drafts([6, 5, 6], 300, "wide", 18, FP32, FP32, noise=0.2)
    keep, n, _ = P().DraftVerifier()(s["logits"], s["tokens"], i32(s["off"]), 6, parents=i32(s["parents"]), draft_probs=s["draft"],
                                     u=s["u"], u_next=s["last"])
    cache = P().QuantPagedCache.create(3, 64, 2, 64)
    x = torch.randn(17, 2, 64, device="cuda", generator=gen(1)).to(BF16)
    cache.append(None, x, x, i32(s["off"]), 6)
    all_k, _ = cache.read(cache.lens, i32(s["off"]), 6, rows=17)
    lens = cache.keep(i32(s["off"]), keep, n)
    assert torch.equal(lens, n) and cache.status_value() == 0
    ends = i32([0] + n.cumsum(0).tolist())
    got, _ = cache.read(cache.lens, ends, 6, rows=int(ends[-1]))
    rows = [s["off"][b] + k for b, ks in enumerate(keep.tolist()) for k in ks if k >= 0]
    assert torch.equal(got, all_k[rows])


def test_tensors_that_do_not_fit_are_refused():
    pkg = P()
    s = drafts([3, 4], 50, "tree", 3, FP32, FP32)
    ok = dict(logits=s["logits"], tokens=s["tokens"], new_off=i32(s["off"]), max_new=4, parents=i32(s["parents"]),
              draft_probs=s["draft"], u=s["u"], u_next=s["last"], temperature=torch.ones(2, device="cuda"))
    v = pkg.DraftVerifier()
    v(**ok)
    for bad in (dict(logits=s["logits"].double()), dict(logits=s["logits"].t().contiguous().t()), dict(tokens=s["tokens"].long()),
                dict(tokens=s["tokens"][:5]), dict(new_off=ok["new_off"].long()), dict(parents=ok["parents"][:3]),
                dict(draft_probs=s["draft"][:, :40]), dict(draft_probs=s["draft"].double()), dict(u=None), dict(u_next=None),
                dict(u=s["u"].half()), dict(u_next=s["last"][:1]), dict(temperature=torch.ones(3, device="cuda")),
                dict(tokens=s["tokens"].cpu()), dict(draft_probs=s["draft"].cpu()), dict(max_new=2000)):
        with pytest.raises(pkg.MoEError):
            v(**dict(ok, **bad))
    assert v.status_value() == 0
