"""Operators that decoding with drafts needs next to the paged cache and its attention, at the sizes a decoding
program calls them.

Four kinds of call ("op"):
  append  normalise each head's query and key, rotate them, and write keys and values into a paged cache: as they are
          (store 16), or as 8-bit codes with one scale per token and head, read back afterwards (store 8)
  attend  attention of a tree of drafted tokens over a cache in 8 bits
  keep    move the accepted drafts together in a cache in 8 bits, and read them back
  verify  accept drafted tokens against the model's logits from given random numbers, and draw the token after them

Head counts, pages and lengths follow perf/operators.py (heads of 64 and 128, contexts up to 32768); vocabularies are
generic.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-6
LEAST, MOST = 2.0 ** -64, 2.0 ** 64  # a row's scale is held between these


def listed():
    def cache(name, op, B, new, ctx, Hq, Hkv, D, page, t, **kw):
        return dict(name=name, op=op, B=B, new=new, ctx=ctx, Hq=Hq, Hkv=Hkv, D=D, page=page, type=t, **kw)

    def verify(name, B, new, V, fan, t, draft, greedy=False, cut=False):
        return dict(name=name, op="verify", B=B, new=new, V=V, fan=fan, type=t, draft=draft, greedy=greedy, cut=cut)
    return [
        # one token of a small model stored with normed heads: latency only
        cache("append 1 token normed", "append", 1, 1, 100, 4, 2, 64, 64, "bf16", store=16, norm=True, interleaved=False),
        # a prompt stored with normed heads
        cache("append prompt normed", "append", 1, 8192, 0, 32, 8, 128, 64, "bf16", store=16, norm=True, interleaved=False),
        # a batch of draft trees stored in 8 bits after ragged contexts
        cache("append 32 trees 8-bit", "append", 32, 32, 4096, 32, 8, 128, 64, "bf16", store=8, norm=True, interleaved=False),
        # a prompt stored in 8 bits, of a model without norms on its heads
        cache("append prompt 8-bit", "append", 1, 8192, 0, 32, 8, 128, 64, "fp16", store=8, norm=False, interleaved=True),
        # one sequence, one token, a short context: latency only
        cache("attend 1 token over 100", "attend", 1, 1, 100, 4, 2, 64, 64, "bf16"),
        # batched generation over ragged contexts of thousands of tokens
        cache("attend 64x1 over 4096", "attend", 64, 1, 4096, 32, 8, 128, 64, "bf16"),
        # large draft trees over long contexts
        cache("attend 4x64 over 32768", "attend", 4, 64, 32768, 32, 8, 128, 128, "fp16"),
        # one sequence's accepted drafts
        cache("keep 1 tree", "keep", 1, 16, 1000, 4, 2, 64, 64, "fp16", kept=4),
        # a large batch's accepted drafts
        cache("keep 256 trees", "keep", 256, 32, 500, 32, 8, 128, 64, "bf16", kept=12),
        # one sequence, four drafts of a cheap guesser that gives no probabilities: latency
        verify("verify 1 chain of 4", 1, 5, 32000, 1, "fp32", "none"),
        # a serving batch's chains, drawn by a draft model
        verify("verify 64 chains of 7", 64, 8, 32000, 1, "bf16", "bf16"),
        # trees with several drafts below a token, over a large vocabulary
        verify("verify 16 trees of 31", 16, 32, 131072, 4, "fp32", "fp32"),
    ]


def draw(rng):
    def log(lo, hi):
        return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
    op = rng.choices(("append", "attend", "keep", "verify"), (4, 4, 1, 4))[0]
    t = rng.choice(("bf16", "fp16"))
    if op == "verify":
        B = log(1, 64)
        new = rng.randint(1, max(1, min(32, 512 // B)))
        draft = rng.choice(("none", "bf16", "fp32"))
        return dict(op=op, B=B, new=new, V=log(300, min(131072, 67108864 // (B * new))), fan=rng.choice((1, 1, 2, 4)),
                    type=rng.choice((t, "fp32")), draft=draft, greedy=draft == "none" and rng.random() < 0.4,
                    cut=rng.random() < 0.4)
    Hkv = rng.choice((1, 2, 4, 8))
    case = dict(op=op, Hkv=Hkv, Hq=Hkv * rng.choice((1, 2, 3, 4, 8)), D=rng.choice((64, 64, 128, 128, 256)),
                page=rng.choice((64, 128, 256)), type=t)
    if case["Hkv"] * case["D"] > 1024:
        case["D"] = 128
    if op == "append":
        B, store = log(1, 64), rng.choice((16, 8, 8))
        return dict(case, B=B, new=log(1, 8192 // B), ctx=log(1, 4096), store=store, norm=store == 16 or rng.random() < 0.7,
                    interleaved=rng.random() < 0.3)
    if op == "attend":
        B = log(1, 64)
        new = min(log(1, 64), max(1, 8192 // (B * case["Hq"])))
        return dict(case, B=B, new=new, ctx=log(1, 4 * 32768 // max(4, B)))
    return dict(case, B=log(1, 256), new=rng.randint(8, 64), ctx=log(1, 1000), kept=rng.randint(2, 8))


# ------------------------------------------------------------------ shapes of a ragged batch
def layout(c):
    """Per sequence: committed length, new tokens, and each new token's parent among them (-1: the committed text).
    A single sequence has the case's sizes, the others of a batch are shorter by up to half."""
    r = random.Random("%(op)s %(B)d %(new)d" % c)
    lens = [c["ctx"] - (r.randint(0, c["ctx"] // 2) if b else 0) for b in range(c["B"])] if "ctx" in c else None
    new = [c["new"] - (r.randint(0, c["new"] // 2) if b else 0) for b in range(c["B"])]
    parents = []
    for n in new:
        if c["op"] == "verify":  # below the first row, the last token that is known
            parents.append([-1] + [i - 1 if c["fan"] == 1 else (i - 1) // c["fan"] if r.random() < 0.5 else r.randint(max(0, i - 4), i - 1)
                                   for i in range(1, n)])
            continue
        par = []
        for i in range(n):
            par.append(r.randint(max(-1, i - 12), i - 1))
        parents.append(par)
    return lens, new, parents


def paths(c):
    """Per sequence: the accepted drafts, ascending."""
    r = random.Random("keep %(B)d %(new)d %(kept)d" % c)
    _, new, _ = layout(c)
    return [sorted(r.sample(range(n), r.randint(1 if b else min(n, c["kept"]), min(n, c["kept"])))) for b, n in enumerate(new)]


def mask_words(parents, width):
    """Bit m of row i: draft m is i or an ancestor of i."""
    rows = []
    for par in parents:
        seen = []
        for i, p in enumerate(par):
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        rows += seen
    return [[(s >> 64 * w) & (1 << 64) - 1 for w in range(width)] for s in rows]


def offsets(counts):
    return torch.tensor([sum(counts[:b]) for b in range(len(counts) + 1)], dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return globals()["prepare_verify" if case["op"] == "verify" else "prepare_cache"](case, g)


def prepare_cache(c, g):
    dev, t, Hq, Hkv, D, page, B = "cuda", DT[c["type"]], c["Hq"], c["Hkv"], c["D"], c["page"], c["B"]

    def rand(*shape):
        return torch.randn(*shape, device=dev, generator=g)
    lens, new, parents = layout(c)
    need = [-(-(a + n) // page) for a, n in zip(lens, new)]
    ids = torch.randperm(sum(need), device=dev, generator=g).int()
    table = torch.zeros(B, max(need), dtype=torch.int32, device=dev)
    owner = torch.arange(max(need), device=dev) < torch.tensor(need, device=dev)[:, None]
    table[owner] = ids
    N = sum(new)
    s = dict(c=c, table=table, lens=torch.tensor(lens, dtype=torch.int32, device=dev), off=offsets(new),
             seq=torch.repeat_interleave(torch.arange(B, device=dev), torch.tensor(new, device=dev)))
    channel = 1 + 3 * (torch.rand(Hkv, 1, D, device=dev, generator=g) > 0.95)  # channels of keys that stand out
    k = rand(sum(need), Hkv, page, D) * channel
    v = rand(sum(need), Hkv, page, D) * (0.5 * rand(sum(need), Hkv, page, 1)).exp()
    if c.get("store", 8) == 16:
        s["k"], s["v"] = k.to(t), v.to(t).transpose(2, 3).contiguous()
    else:
        s["k"], s["ks"] = quantised(k.to(t).float())
        v, s["vs"] = quantised(v.to(t).float())
        s["v"] = v.transpose(2, 3).contiguous()
    del k, v
    if c["op"] == "keep":
        kept = paths(c)
        wide = max(map(len, kept))
        s["idx"] = torch.tensor([p + [0] * (wide - len(p)) for p in kept], dtype=torch.int32, device=dev)
        s["n"] = torch.tensor([len(p) for p in kept], dtype=torch.int32, device=dev)
        s["len_out"] = torch.empty(B, dtype=torch.int32, device=dev)
        counts = [len(p) for p in kept]
        s["back"], s["most"] = offsets(counts), wide
        s["bseq"] = torch.repeat_interleave(torch.arange(B, device=dev), s["n"].long())
        s["k_out"], s["v_out"] = (torch.empty(sum(counts), Hkv, D, dtype=t, device=dev) for _ in "kv")
    if c["op"] == "attend":
        s["q"] = rand(N, Hq, D).to(t)
        s["out"] = torch.empty_like(s["q"])
        width = -(-max(new) // 64)
        words = [[x - (1 << 64) if x >> 63 else x for x in row] for row in mask_words(parents, width)]
        s["mask"] = torch.tensor(words, dtype=torch.int64, device=dev)
    if c["op"] == "append":
        qkv = rand(N, Hq + 2 * Hkv, D)
        qkv[:, Hq:Hq + Hkv] *= channel[:, 0]
        qkv = qkv.to(t)  # one projection's output, split by heads
        s["q"], s["knew"], s["vnew"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["q_out"] = torch.empty(N, Hq, D, dtype=t, device=dev)
        s["w_q"], s["w_k"] = (1 + 0.1 * rand(D), 1 + 0.1 * rand(D)) if c["norm"] else (None, None)
        at = torch.arange(N, device=dev) - s["off"][s["seq"]]
        s["pos"] = (s["lens"][s["seq"]] + at).int()
        angle = torch.arange(max(a + n for a, n in zip(lens, new)), device=dev)[:, None] * 10000.0 ** (
            -torch.arange(D // 2, device=dev) / (D // 2))
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        if c["store"] == 8:
            s["k_out"], s["v_out"] = (torch.empty(N, Hkv, D, dtype=t, device=dev) for _ in "kv")
    return s


def prepare_verify(c, g):
    dev, B, V = "cuda", c["B"], c["V"]
    _, new, parents = layout(c)
    N, n = sum(new), max(new)
    off = offsets(new)
    guess = 2.5 * torch.randn(N, V, device=dev, generator=g)  # the draft model's logits
    logits = guess + 0.7 * torch.randn(N, V, device=dev, generator=g)
    if c["cut"]:  # a program keeps the largest few and rules the others out
        logits.masked_fill_(logits < logits.topk(min(V, 100), 1).values[:, -1:], -math.inf)
    q = torch.softmax(guess, 1)
    del guess
    parent = torch.tensor([p for par in parents for p in par], dtype=torch.int32, device=dev)
    first = off[:-1].repeat_interleave(torch.tensor(new, device=dev))
    above = (first + parent.clamp(min=0)).long()
    if c["draft"] == "none":  # the guesser's likeliest tokens, the next one for each further draft of a token
        place = torch.tensor([sum(par[j] == p for j in range(i)) for par in parents for i, p in enumerate(par)], device=dev)
        tokens = q.topk(min(V, int(place.max()) + 1), 1).indices[above, place.clamp(max=V - 1)]
    else:  # drawn from the draft model's probabilities, as they are stored
        q = q.to(DT[c["draft"]])
        up = torch.cumsum(q[above].double(), 1)
        pick = torch.rand(N, 1, device=dev, generator=g, dtype=torch.float64) * up[:, -1:]
        tokens = torch.searchsorted(up, pick)[:, 0].clamp(max=V - 1)
        del up
    return dict(c=c, logits=logits.to(DT[c["type"]]), draft=None if c["draft"] == "none" else q, tokens=tokens.int(), off=off,
                new=torch.tensor(new, device=dev), most=n, parent=None if c["fan"] == 1 else parent, chain=parent,
                u=None if c["greedy"] else torch.rand(N, device=dev, generator=g),
                last=None if c["greedy"] else torch.rand(B, device=dev, generator=g),
                heat=None if c["greedy"] else 0.6 + 0.8 * torch.rand(B, device=dev, generator=g))


def quantised(x):
    """8-bit codes of rows and their scales: the largest magnitude becomes 127."""
    s = (x.abs().amax(-1) / 127).clamp(LEAST, MOST)
    return (x / s[..., None]).round().clamp(-127, 127).to(torch.int8), s


# ------------------------------------------------------------------ one pass
def run(s):
    return globals()[("own_" if own else "plain_") + s["c"]["op"]](s)


def places(s, first, seq, off):
    """Page and place in it of rows that stand, sequence by sequence, behind `first`."""
    at = first[seq] + torch.arange(len(seq), device="cuda") - off[seq]
    return s["table"][seq, at // s["c"]["page"]].long(), at % s["c"]["page"]


def back(s, pg, o):
    """What the 8-bit rows at these places stand for."""
    t = DT[s["c"]["type"]]
    return [(s["k"][pg, :, o].float() * s["ks"][pg, :, o][..., None]).to(t), (s["v"][pg, :, :, o].float() * s["vs"][pg, :, o][..., None]).to(t)]


def turned(x, cos, sin, interleaved):
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else x.chunk(2, -1)
    u, v = a * cos - b * sin, a * sin + b * cos
    return torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)


def plain_append(s):
    c, t = s["c"], DT[s["c"]["type"]]
    cos, sin = (x[s["pos"].long()][:, None] for x in (s["cos"], s["sin"]))

    def normed(x, w):
        x = x.float()
        return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    q = turned(normed(s["q"], s["w_q"]), cos, sin, c["interleaved"]).to(t)
    k = turned(normed(s["knew"], s["w_k"]), cos, sin, c["interleaved"])
    pg, o = places(s, s["lens"], s["seq"], s["off"])
    if c["store"] == 16:
        s["k"][pg, :, o] = k.to(t)
        s["v"][pg, :, :, o] = s["vnew"]
        return [q, s["k"], s["v"]]
    s["k"][pg, :, o], s["ks"][pg, :, o] = quantised(k)
    s["v"][pg, :, :, o], s["vs"][pg, :, o] = quantised(s["vnew"].float())
    return [q] + back(s, pg, o)


def plain_attend(s):
    c = s["c"]
    B, Hq, Hkv, D, n = c["B"], c["Hq"], c["Hkv"], c["D"], c["new"]
    tot = s["table"].shape[1] * c["page"]
    pages = s["table"].long()
    k = (s["k"][pages].float() * s["ks"][pages][..., None]).transpose(1, 2).reshape(B, Hkv, tot, D)  # [B][pages][Hkv][page][D]
    v = (s["v"][pages].float() * s["vs"][pages][..., None, :]).permute(0, 2, 1, 4, 3).reshape(B, Hkv, tot, D)
    i = torch.arange(len(s["seq"]), device="cuda") - s["off"][s["seq"]]
    q = torch.zeros(B, n, Hq, D, device="cuda")
    q[s["seq"], i] = s["q"].float()
    q = q.view(B, n, Hkv, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D)
    bits = torch.zeros(B, n, 64 * s["mask"].shape[1], dtype=torch.bool, device="cuda")
    bits[s["seq"], i] = (s["mask"][..., None] >> torch.arange(64, device="cuda") & 1).bool().flatten(1)
    j = torch.arange(tot, device="cuda") - s["lens"][:, None]  # [B][tot]: place among the new tokens
    sees = (j < 0)[:, None] | (bits.gather(2, j.clamp(0, bits.shape[2] - 1)[:, None].expand(-1, n, -1)) & ((j >= 0) & (j < n))[:, None])
    sees = sees[:, None, :, None].expand(-1, -1, -1, Hq // Hkv, -1).reshape(B, 1, -1, tot)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) * D ** -0.5
    score = score.masked_fill(~sees, -math.inf)
    p = (score - score.amax(3, keepdim=True).clamp(min=-3e38)).exp()
    o = torch.matmul(p, v) / p.sum(3, keepdim=True).clamp(min=1e-30)
    o = o.view(B, Hkv, n, Hq // Hkv, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    return o[s["seq"], i].to(s["q"].dtype)


def plain_keep(s):
    page, wide = s["c"]["page"], s["idx"].shape[1]
    j = torch.arange(wide, device="cuda").expand_as(s["idx"])
    b, j = (j < s["n"][:, None]).nonzero(as_tuple=True)
    src, dst = s["lens"][b] + s["idx"][b, j], s["lens"][b] + j
    sp, dp = s["table"][b, src // page].long(), s["table"][b, dst // page].long()
    k, ks, v, vs = s["k"][sp, :, src % page], s["ks"][sp, :, src % page], s["v"][sp, :, :, src % page], s["vs"][sp, :, src % page]
    s["k"][dp, :, dst % page] = k
    s["ks"][dp, :, dst % page] = ks
    s["v"][dp, :, :, dst % page] = v
    s["vs"][dp, :, dst % page] = vs
    return [s["lens"] + s["n"]] + back(s, *places(s, s["lens"], s["bseq"], s["back"]))


def plain_verify(s):
    """In 64 bits, where the border between two tokens lies.  r: what is left of the distribution at `cur`."""
    c, first, B, n = s["c"], s["off"][:-1].long(), s["c"]["B"], s["most"]
    heat = 1.0 if s["heat"] is None else s["heat"].double()[:, None]
    seqs = torch.arange(B, device="cuda")

    def at(row):
        x = s["logits"][row].double()
        return torch.nn.functional.one_hot(x.argmax(1), c["V"]).double() if c["greedy"] else torch.softmax(x / heat, 1)
    cur, r = torch.zeros_like(first), at(first)
    keep = torch.full((B, n), -1, dtype=torch.int32, device="cuda")
    keep[:, 0] = 0
    count = torch.ones_like(first)
    for i in range(1, n):  # parents stand before their drafts
        row = first + torch.where(i < s["new"], i, 0)
        here = (i < s["new"]) & (s["chain"][row] == cur)
        x = s["tokens"][row].long()
        q = torch.nn.functional.one_hot(x, c["V"]).double() if s["draft"] is None else s["draft"][first + cur].double()
        u = 0.5 if c["greedy"] else s["u"][row].double()
        yes = here & (u * q[seqs, x] < r[seqs, x])
        left = (r - q).clamp(min=0)
        total = left.sum(1, keepdim=True)
        r = torch.where((here & ~yes)[:, None] & (total > 0), left / total.clamp(min=1e-300), r)
        r = torch.where(yes[:, None], at(row), r)
        cur = torch.where(yes, i, cur)
        keep[seqs, count.clamp(max=n - 1)] = torch.where(yes, i, keep[seqs, count.clamp(max=n - 1)]).int()
        count = count + yes
    if c["greedy"]:
        return [keep, count.int(), s["logits"][first + cur].double().argmax(1).int()]
    up = r.cumsum(1)
    return [keep, count.int(), (up <= s["last"].double()[:, None] * up[:, -1:]).sum(1).clamp(max=c["V"] - 1).int()]


def kept(s, make):
    """The object that a decoding program keeps, with its workspace."""
    if "mine" not in s:
        s["mine"] = make()
    return s["mine"]


def cache_of(s):
    from paper_2503_21135_amd import PagedCache, QuantPagedCache
    if s["c"].get("store", 8) == 16:
        return PagedCache(s["k"], s["v"], s["table"], s["lens"])
    return QuantPagedCache(s["k"], s["v"], s["ks"], s["vs"], s["table"], s["lens"], dtype=DT[s["c"]["type"]])


def own_append(s):
    c, cache = s["c"], kept(s, lambda: cache_of(s))
    cache.append(s["q"], s["knew"], s["vnew"], s["off"], c["new"], positions=s["pos"], cos=s["cos"], sin=s["sin"],
                 interleaved=c["interleaved"], q_out=s["q_out"], w_q=s["w_q"], w_k=s["w_k"], eps=EPS)
    if c["store"] == 16:
        return [s["q_out"], s["k"], s["v"]]
    cache.read(s["lens"], s["off"], c["new"], k_out=s["k_out"], v_out=s["v_out"])
    return [s["q_out"], s["k_out"], s["v_out"]]


def own_attend(s):
    c = s["c"]
    return kept(s, lambda: cache_of(s)).attend(s["q"], s["off"], c["new"], c["ctx"] + c["new"], mask=s["mask"],
                                               scale=c["D"] ** -0.5, out=s["out"])


def own_keep(s):
    cache = kept(s, lambda: cache_of(s))
    cache.keep(s["off"], s["idx"], s["n"], len_out=s["len_out"])
    cache.read(s["lens"], s["back"], s["most"], k_out=s["k_out"], v_out=s["v_out"])
    return [s["len_out"], s["k_out"], s["v_out"]]


def own_verify(s):
    from paper_2503_21135_amd import DraftVerifier
    return list(kept(s, DraftVerifier)(s["logits"], s["tokens"], s["off"], s["most"], parents=s["parent"],
                                       draft_probs=s["draft"], u=s["u"], u_next=s["last"], temperature=s["heat"]))


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    if case["op"] == "verify":
        return None  # whole numbers alone
    return globals()["exact_" + case["op"]](prepare(case, seed), case)


def steps(x):
    """The 8-bit rows' values: multiples of a 127th of the row's largest magnitude (the scale is held in 32 bits)."""
    s = (x.abs().amax(-1, keepdim=True) / 127).clamp(LEAST, MOST)
    return torch.round(x / s) * s


def exact_append(s, c):
    lens, new, _ = layout(c)
    half, page = c["D"] // 2, c["page"]
    angle = torch.complex(s["cos"].double(), s["sin"].double())[s["pos"].long()][:, None]

    def turn(x, w):
        x = x.double()
        if w is not None:
            x = x / ((x ** 2).sum(-1, keepdim=True) / c["D"] + EPS).sqrt() * w.double()
        if c["interleaved"]:
            return torch.view_as_real(torch.view_as_complex(x.reshape(*x.shape[:-1], half, 2)) * angle).flatten(-2)
        y = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * angle
        return torch.cat((y.real, y.imag), -1)
    q, kt, vt = turn(s["q"], s["w_q"]), turn(s["knew"], s["w_k"]), s["vnew"].double()
    if c["store"] == 8:
        return [q, steps(kt), steps(vt)]
    k, v, n, pages = s["k"].double(), s["v"].double(), 0, s["table"].tolist()
    for b in range(c["B"]):
        i = 0
        while i < new[b]:  # one run of slots inside a page at a time
            at = lens[b] + i
            m = min(new[b] - i, page - at % page)
            pg, o = pages[b][at // page], at % page
            k[pg, :, o:o + m] = kt[n + i:n + i + m].transpose(0, 1)
            v[pg, :, :, o:o + m] = vt[n + i:n + i + m].permute(1, 2, 0)
            i += m
        n += new[b]
    return [q, k, v]


def exact_attend(s, c):
    lens, new, parents = layout(c)
    G, n, outs = c["Hq"] // c["Hkv"], 0, []
    for b in range(c["B"]):
        m, tot = new[b], lens[b] + new[b]
        pages = s["table"][b, :-(-tot // c["page"])].long()
        sees = torch.zeros(m, tot, dtype=torch.bool)
        sees[:, :lens[b]] = True
        for i in range(m):
            a = i
            while a >= 0:
                sees[i, lens[b] + a] = True
                a = parents[b][a]
        hide = torch.where(sees, 0.0, -math.inf).double().cuda()
        heads = []
        for h in range(c["Hkv"]):
            kk = (s["k"][pages, h].double().reshape(-1, c["D"]) * s["ks"][pages, h].double().reshape(-1, 1))[:tot]
            vv = (s["v"][pages, h].double().transpose(1, 2).reshape(-1, c["D"]) * s["vs"][pages, h].double().reshape(-1, 1))[:tot]
            q = s["q"][n:n + m, h * G:(h + 1) * G].double().transpose(0, 1)
            w = torch.softmax((q.reshape(-1, c["D"]) @ kk.t()).view(G, m, tot) / math.sqrt(c["D"]) + hide, 2)
            heads.append((w.view(G * m, tot) @ vv).view(G, m, c["D"]).transpose(0, 1))
        outs.append(torch.cat(heads, 1))
        n += m
    return torch.cat(outs)


def exact_keep(s, c):
    lens, pages, p = layout(c)[0], s["table"].tolist(), c["page"]
    ks, vs = [], []
    for b, path in enumerate(paths(c)):
        for i in path:  # the row that the accepted draft was written to
            a = lens[b] + i
            pg, o = pages[b][a // p], a % p
            ks.append(s["k"][pg, :, o].double() * s["ks"][pg, :, o, None].double())
            vs.append(s["v"][pg, :, :, o].double() * s["vs"][pg, :, o, None].double())
    return [None, torch.stack(ks), torch.stack(vs)]


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    lens, new, parents = layout(c)
    N = sum(new)
    if c["op"] == "verify":
        # every row's logits, and where drafts came with probabilities the last row's
        return {"bytes": N * c["V"] * BYTES[c["type"]] + (0 if c["draft"] == "none" else c["B"] * c["V"] * BYTES[c["draft"]]) + 16 * N,
                "flops": 4 * N * c["V"]}
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    if c["op"] == "append":
        angles = 4 * D * (max(a + n for a, n in zip(lens, new)) if c["B"] == 1 else N)
        q, new_rows = 2 * 2 * N * Hq * D, 2 * 2 * N * Hkv * D
        stored = new_rows if c["store"] == 16 else 2 * N * Hkv * (D + 4) + new_rows  # and back in 16 bits
        return {"bytes": q + new_rows + stored + min(angles, 4 * D * N) + (8 * D if c["norm"] else 0), "flops": 8 * N * (Hq + 2 * Hkv) * D}
    if c["op"] == "attend":
        keys = sum(a + n for a, n in zip(lens, new))
        return {"bytes": 2 * keys * Hkv * (D + 4) + 2 * 2 * N * Hq * D,
                "flops": sum(4 * n * (a + n) for a, n in zip(lens, new)) * Hq * D}
    rows = sum(map(len, paths(c)))
    moved = sum(i != j for path in paths(c) for j, i in enumerate(path))
    return {"bytes": 2 * Hkv * (2 * moved * (D + 4) + rows * (D + 4) + 2 * rows * D), "flops": 2 * rows * Hkv * D}
