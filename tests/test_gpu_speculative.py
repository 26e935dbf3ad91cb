"""The speculative decoding example: the operators together, as a server calls them."""
import os
import sys

import pytest

from gpu_util import torch_cuda

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    torch_cuda()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import speculative_decode
    finally:
        sys.path.pop(0)
    return speculative_decode


def test_tree_mask(example):
    assert example.tree_mask([-1, 0, 0, 1]) == [0b1, 0b11, 0b101, 0b1011]
    assert [example.DEPTH[p] + 1 for p in example.PARENT[1:]] == example.DEPTH[1:]


def test_speculative_decoding_says_what_one_by_one_says(example):
    """Greedy decoding is deterministic but for near-ties between tokens, which the two block sizes may round apart:
    the first tokens agree, and more than one is accepted a pass on average."""
    fast, slow, passes = example.main(B=2, T=150, steps=8, seed=3)
    for f, s in zip(fast, slow):
        assert len(f) > passes and f[:6] == s[:6]
    assert sum(len(f) - 1 for f in fast) > 2 * passes


def test_committed_rows_are_the_accepted_tokens_rows(example):
    """After the run the cache holds the prompt and the accepted tokens, each at its own position."""
    import torch
    B, T, steps = 2, 60, 6
    g = torch.Generator(device="cuda").manual_seed(9)
    prompt = torch.randint(0, 512, (B, T), generator=g, device="cuda")
    model = example.Model(B, T + 4 * steps + 8, seed=5)
    said = example.speculative(model, prompt, steps)
    held = model.cache.t["T_len"].tolist()
    for b in range(B):
        assert held[b] == T + len(said[b]) - 1            # the last token said is not in the cache yet
        tokens = torch.cat([prompt[b], torch.tensor(said[b][:-1], device="cuda")])[None]
        rows = model._inputs(tokens, torch.arange(held[b], device="cuda")[None])[2]
        got = model.cache.t["rows"][b, :held[b]].float()
        assert (got - rows[0].float()).abs().max() <= 2.0 ** -8 * rows.float().abs().max()
