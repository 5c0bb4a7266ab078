"""Decoding with drafts over caches in 8 bits, with normed heads and random numbers: the operators
together, as a serving program runs them."""
import pytest
import torch

from test_gpu_draft_decode import example

pytestmark = pytest.mark.gpu
PROMPT = [(7 * i) % 500 for i in range(40)]


def small(mod, **kw):
    import paper_2503_21135_amd as P
    return mod.Model(cache=P.QuantPagedCache, page=64, norms=True, **kw)


def test_draws_over_a_cache_in_8_bits():
    mod = example()
    model = small(mod)
    out, steps = mod.decode(model, PROMPT, 50, temperature=0.9, seed=3)
    assert len(out) == 50 and 2 <= steps <= 50 and all(0 <= t < 500 for t in out)
    assert all(x.status_value() == 0 for x in model.caches + model.blocks)
    # what the caches hold is as long as the text that has been kept, and the same from the same numbers
    assert [int(c.lens) for c in model.caches] == [model.len] * 2 and model.len >= len(PROMPT) + 49
    assert mod.decode(small(mod), PROMPT, 50, temperature=0.9, seed=3)[0] == out
    assert mod.decode(small(mod), PROMPT, 50, temperature=0.9, seed=4)[0] != out


def test_greedy_over_a_cache_in_8_bits_agrees_with_single_tokens():
    """Every kept path's logits are those of the same tokens one at a time."""
    mod = example()
    plain, model, kept, seen = small(mod), small(mod), [], []
    tokens, single = [], []
    logits, off = plain.logits(torch.tensor(PROMPT, device="cuda:0"))
    plain.keep(off, list(range(len(PROMPT))))
    tokens.append(int(logits[-1].argmax()))
    while len(tokens) < 40:
        logits, off = plain.logits(torch.tensor(tokens[-1:], device="cuda:0"))
        plain.keep(off, [0])
        single.append(logits[0].clone())
        tokens.append(int(logits[0].argmax()))
    call_logits, call_keep, at = model.logits, model.keep, [0]

    def draft(token):      # the right path among others
        i = at[0]
        tree, parents, right = [token], [-1], 0
        for d in range(1, 4):
            below = [(tokens[i + d] + 1) % 500, tokens[i + d], (tokens[i + d] + 2) % 500]
            first = len(tree)
            tree += below
            parents += [right] * 3
            right = first + 1
        return tree, parents

    def logits_of(tok, positions=None, mask=None):
        out = call_logits(tok, positions, mask)
        seen.append(out[0].clone())
        return out

    def keep(off, path):
        if len(path) < len(PROMPT):
            for j, p in enumerate(path):
                want = single[at[0] + j]
                # bf16 activations of two layers, and codes that fall the other way with them
                assert float((seen[-1][p] - want).norm() / want.norm()) < 3e-2, (at[0], j)
            kept.append(len(path))
            at[0] += len(path)
        call_keep(off, path)
    model.draft, model.logits, model.keep = draft, logits_of, keep
    out, steps = mod.decode(model, PROMPT, 30)
    assert out == tokens[:30] and min(kept) > 1 and steps < 15
