"""The decoding example end to end: append, attention over trees, sparse FFN,
commit in every layer.  Greedy decoding with guesses must give the text of
decoding token by token, in fewer steps, and the committed cache must be the
one that a single prompt pass over the text leaves."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (4, 4)])
def test_trees_give_the_text_of_single_tokens(pp, heads, kv_heads):
    import torch
    import tree_decode as td
    prompt = [(7 * i) % 23 for i in range(40)]
    plain, steps = td.generate(td.TreeDecoder(heads=heads, kv_heads=kv_heads), prompt, 60)
    assert steps == 60
    model = td.TreeDecoder(heads=heads, kv_heads=kv_heads)
    guessed, fewer = td.generate(model, prompt, 60, width=4)
    assert guessed == plain
    assert fewer < 60
    # the cache after the last step against one pass over the same tokens
    n = int(model.length.item())
    text = (prompt + guessed)[:n]
    assert n >= len(prompt) and len(text) == min(n, len(prompt) + 60)
    once = td.TreeDecoder(heads=heads, kv_heads=kv_heads)
    for i in range(0, len(text), 64):
        part = text[i:i + 64]
        once.forward(part)
        once.commit(list(range(len(part))))
    once.check()
    j = torch.arange(len(text), device="cuda")
    page, at = model.table[0].long()[j // td.PAGE], j % td.PAGE
    for a, b in ((model.k, once.k), (model.v, once.v)):
        x, y = a[:, page, at], b[:, page, at]
        # fp32 sums in another order through two layers
        assert torch.allclose(x, y, rtol=1e-4, atol=1e-4)


def test_example_runs_in_bf16(pp):
    import tree_decode as td
    tokens, steps = td.generate(td.TreeDecoder(dtype="bf16"), list(range(20)), 24, width=3)
    assert len(tokens) == 24 and steps <= 24
