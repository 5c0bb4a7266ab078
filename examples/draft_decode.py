"""Decoding with trees of drafts through DecoderBlocks, as a serving program would.

A small model (random weights): embedding, two DecoderBlocks (4-bit projections, paged
cache, tree attention, mixed-precision MoE layer) and a 4-bit vocabulary projection.
Each step drafts a tree of tokens, runs the whole tree through the model at once, follows
the greedy choices down the tree, keeps the accepted path in every layer's cache and
drafts again from there.

    python examples/draft_decode.py
"""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import moe_inputs as mi  # noqa: E402
import paper_2503_21135_amd as P  # noqa: E402


class Model:
    def __init__(self, n_blocks=2, vocab=500, heads=(4, 2, 64), max_len=512, seed=0):
        dev = "cuda:0"
        g = torch.Generator(device=dev).manual_seed(seed)
        layer = mi.WORKLOADS["tiny"].layer
        d, (Hq, Hkv, D) = layer.d_model, heads

        def w(*shape, scale=0.06):
            return scale * torch.randn(*shape, device=dev, generator=g)
        angle = torch.arange(max_len, device=dev)[:, None] * 10000.0 ** (-torch.arange(D // 2, device=dev) / (D // 2))
        self.blocks = [P.DecoderBlock(P.MoELayer(mi.LayerInputs(layer), device=dev), w((Hq + 2 * Hkv) * D, d), w(d, Hq * D),
                                      Hq, Hkv, D, dict(attn=1 + w(d), ffn=1 + w(d), attn_post=1 + w(d), ffn_post=1 + w(d)),
                                      angle.cos(), angle.sin(), group=64) for _ in range(n_blocks)]
        self.embed, self.last_norm = w(vocab, d, scale=1.0), 1 + w(d)
        self.head = P.QuantLinear(w(vocab, d), group=64)
        self.caches = [P.PagedCache.create(1, max_len, Hkv, D, page_size=32, device=dev) for _ in range(n_blocks)]
        self.len = 0      # the caches' length, which the program knows without asking the device

    def logits(self, tokens, positions=None, mask=None):
        """Logits [tokens][vocab] of new tokens; their keys and values are appended, not kept."""
        n = len(tokens)
        off = torch.tensor([0, n], dtype=torch.int32, device="cuda:0")
        r = self.embed[tokens].clone()
        h = torch.empty(r.shape, dtype=torch.bfloat16, device=r.device)
        P.moe_block_norm(r, h, w_pre=self.blocks[0].norms["attn"])
        for i, b in enumerate(self.blocks):
            after = self.blocks[i + 1].norms["attn"] if i + 1 < len(self.blocks) else self.last_norm
            b.forward(r, h, self.caches[i], off, n, self.len + n, positions, mask, after)
        return self.head(h, torch.empty(n, self.head.R, device=r.device)), off

    def keep(self, off, path):
        """Keep the new tokens of `path` (indices, ascending) in every layer's cache."""
        keep = torch.tensor([path], dtype=torch.int32, device="cuda:0")
        n = torch.tensor([len(path)], dtype=torch.int32, device="cuda:0")
        for c in self.caches:
            c.lens.copy_(c.keep(off, keep, n))
        self.len += len(path)

    def draft(self, token, depth=3, fan=2):
        """A tree below `token` by a far cheaper model: the projection of the bare embedding.
        Returns (tokens, parents), the token itself first."""
        tokens, parents, level = [token], [-1], [0]
        for _ in range(depth):
            h = torch.empty(len(level), self.embed.shape[1], dtype=torch.bfloat16, device="cuda:0")
            P.moe_block_norm(self.embed[[tokens[i] for i in level]], h, w_pre=self.last_norm)
            best = self.head(h).topk(fan, dim=1).indices.tolist()
            below = []
            for i, choice in zip(level, best):
                for c in choice:
                    below.append(len(tokens))
                    tokens.append(c)
                    parents.append(i)
            level = below
        return tokens, parents


def decode(model, prompt, n_new):
    """n_new greedy tokens; (tokens, steps of the model it took)."""
    logits, off = model.logits(torch.tensor(prompt, device="cuda:0"))
    model.keep(off, list(range(len(prompt))))
    out, steps = [int(logits[-1].argmax())], 1
    while len(out) < n_new:
        tokens, parents = model.draft(out[-1])
        depth = []
        for p in parents:
            depth.append(0 if p < 0 else depth[p] + 1)
        positions = torch.tensor([model.len + x for x in depth], dtype=torch.int32, device="cuda:0")
        logits, off = model.logits(torch.tensor(tokens, device="cuda:0"), positions, P.tree_mask([parents]))
        choice, path = logits.argmax(1).tolist(), [0]
        while True:      # down the tree as long as a draft is what the model chose
            out.append(choice[path[-1]])
            child = [i for i, p in enumerate(parents) if p == path[-1] and tokens[i] == out[-1]]
            if not child:
                break
            path.append(child[0])
        model.keep(off, path)
        steps += 1
    return out[:n_new], steps


def decode_plain(model, prompt, n_new):
    """The same, one token at a time."""
    logits, off = model.logits(torch.tensor(prompt, device="cuda:0"))
    model.keep(off, list(range(len(prompt))))
    out = [int(logits[-1].argmax())]
    while len(out) < n_new:
        logits, off = model.logits(torch.tensor(out[-1:], device="cuda:0"))
        model.keep(off, [0])
        out.append(int(logits[0].argmax()))
    return out


def main():
    prompt = [(7 * i) % 500 for i in range(40)]
    model, plain = Model(), Model()
    out, steps = decode(model, prompt, 60)
    want = decode_plain(plain, prompt, 60)
    same = sum(a == b for a, b in zip(out, want))
    assert all(x.status_value() == 0 for m in (model, plain) for x in m.caches + m.blocks)
    print("%d tokens in %d steps of the model; %d of them as one token at a time gives" % (len(out), steps, same))
    return out, want, steps


if __name__ == "__main__":
    main()
