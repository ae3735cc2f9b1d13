"""The generating example with drafted tokens: rotation, cache, attention over the shared prefix and verification together."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("cache", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("m", [1, 5])
def test_drafts_see_what_single_steps_see(cuda_device, cache, m):
    # the logits of several tokens at once against those of a token after the other over the same cache
    import generate as g

    w = g.merged_parameters()
    one, many = g.Decoder(w, 3, 48, cache, page_size=7), g.Decoder(w, 3, 48, cache, page_size=7)
    tokens = torch.randint(0, g.VOCAB, (3, 30), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    want = torch.stack([one.step(tokens[:, i], torch.full((3,), i, device="cuda")) for i in range(30)], 1)
    got = torch.cat([many.step_drafts(tokens[:, i:i + m], torch.full((3,), i, device="cuda")) for i in range(0, 30, m)], 1)
    one.check(), many.check()
    # Both round activations to bfloat16 (half a step, 2^-8) at eleven places a layer and three more, and values that differ by a rounding may be cached in
    # neighbouring steps (e4m3 2^-3, int8 2^-7 of a vector's largest); roundings do not all add up, so the sum of all is a generous bound.
    bound = (11 * g.LAYERS + 3) * 2.0 ** -8 + g.LAYERS * {"bf16": 2.0 ** -8, "e4m3": 2 * 2.0 ** -3, "int8": 2 * 2.0 ** -7}[cache]
    off = (got - want).norm(dim=-1) / want.norm(dim=-1)
    assert float(off.max()) < bound, float(off.max())


def test_greedy_drafts_are_the_largest_logits(cuda_device):
    import generate as g

    w = g.merged_parameters()
    decoder = g.Decoder(w, 4, 55, "bf16", page_size=16)
    first = torch.tensor([5, 77, 901, 5], device="cuda")  # (the table has room for the drafts of a sequence that has ended)
    tokens, rounds = g.generate_with_drafts(decoder, first, 50, 4)
    decoder.check()
    assert tokens.shape == (4, 51) and bool((tokens >= 0).all()) and torch.equal(tokens[0], tokens[3]) and rounds <= 50
    # each token against the logits that single steps give for its place: the largest, within what the two ways differ by
    other = g.Decoder(w, 4, 60, "bf16", page_size=16)
    for i in range(50):
        logits = other.step(tokens[:, i], torch.full((4,), i, device="cuda"))
        chosen = logits.gather(1, tokens[:, i + 1:i + 2])[:, 0]
        assert bool((chosen >= logits.amax(-1) - 0.25 * logits.norm(dim=-1) / logits.shape[-1] ** 0.5).all())


def test_drawn_tokens_and_lookups(cuda_device):
    import generate as g

    decoder = g.Decoder(g.merged_parameters(), 3, 60, "e4m3")
    first = torch.tensor([5, 77, 901], device="cuda")
    t = torch.tensor([0.0, 0.7, 1.0], device="cuda")
    tokens, rounds = g.generate_with_drafts(decoder, first, 40, 3, temperature=t, seed=1)
    again, _ = g.generate_with_drafts(g.Decoder(g.merged_parameters(), 3, 60, "e4m3"), first, 40, 3, temperature=t, seed=1)
    assert torch.equal(tokens, again) and tokens.shape == (3, 41) and bool((tokens >= 0).all()) and bool((tokens < g.VOCAB).all())
    history = torch.tensor([[1, 2, 3, 1, 2, 9, 1, -2, -2], [4, 5, 6, 7, -2, -2, -2, -2, -2]], device="cuda")
    drafts = g.look_up(history, torch.tensor([7, 4], device="cuda"), 4)
    assert drafts.tolist() == [[2, 9, 1, -1], [-1] * 4]
