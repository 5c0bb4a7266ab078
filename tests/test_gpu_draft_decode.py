"""Decoding with drafts that the model accepts: what is kept of each tree continues as if it
had been decoded one token at a time."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "draft_decode.py")
    spec = importlib.util.spec_from_file_location("draft_decode", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_accepted_paths_continue_as_single_tokens_do():
    """Trees whose right path is known: the tokens that single steps choose, hidden among
    others.  Every kept path is longer than its root, and the logits along it are those of the
    same tokens one at a time."""
    mod = example()
    prompt, n_new = [(7 * i) % 500 for i in range(40)], 60
    plain = mod.Model()
    logits, off = plain.logits(torch.tensor(prompt, device="cuda:0"))
    plain.keep(off, list(range(len(prompt))))
    tokens, single = [int(logits[-1].argmax())], [logits[-1].clone()]
    while len(tokens) < n_new + 8:
        logits, off = plain.logits(torch.tensor(tokens[-1:], device="cuda:0"))
        plain.keep(off, [0])
        single.append(logits[0].clone())
        tokens.append(int(logits[0].argmax()))

    model, kept, seen = mod.Model(), [], []
    at, call_logits, call_keep = [0], model.logits, model.keep

    def draft(token):
        """The next four tokens as a path among a tree's 12 others, in places that vary."""
        i = at[0]
        assert token == tokens[i]
        tree, parents, right = [token], [-1], 0
        for d in range(1, 5):
            below = [(tokens[i + d] + 1 + j) % 500 for j in range(3)]
            below.insert((i + d) % 4, tokens[i + d])
            first = len(tree)
            tree += below
            parents += [right] * 4
            right = first + (i + d) % 4
        return tree, parents

    def logits_of(tok, positions=None, mask=None):
        out = call_logits(tok, positions, mask)
        seen.append(out[0].clone())
        return out

    def keep(off, path):
        if seen[-1].shape[0] != len(prompt):
            for j, p in enumerate(path):
                want = single[at[0] + 1 + j]
                err = float((seen[-1][p] - want).norm() / want.norm())
                # bf16 activations of two layers: their roundings differ where sums run in another order
                assert err < 2e-2, (at[0], j, err)
            kept.append(len(path))
            at[0] += len(path)
        call_keep(off, path)
    model.draft, model.logits, model.keep = draft, logits_of, keep
    out, steps = mod.decode(model, prompt, n_new)
    assert out == tokens[:n_new]
    assert min(kept) > 1 and sum(kept) / len(kept) > 4 and steps < n_new / 3
    assert all(x.status_value() == 0 for m in (model, plain) for x in m.caches + m.blocks)
