"""What the generating example does with drafted tokens, call by call.

Attention: every row of every layer's bcp_kv_attend_shared against all tokens of its sequence up to its own, read from the same cache in 64 bits, within the bound that
the roundings of one call give (the whole pages before a draft and the tokens behind them are cut apart by the example; one that is lost or counted twice exceeds it).
Verification: drafts that are right are accepted."""
import os
import sys

import pytest
import torch

import paper_2407_20143_b200 as bcp
from test_gpu_shared import assert_attended

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("cache_type", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("m,page_size", [(1, 7), (5, 7), (5, 16), (3, 1)])
def test_every_row_sees_its_sequence_up_to_itself(cuda_device, monkeypatch, cache_type, m, page_size):
    import generate as g

    decoder = g.Decoder(g.merged_parameters(), 3, 48, cache_type, page_size=page_size)
    real, state, calls = bcp.bcp_kv_attend_shared, {}, []

    def checked(cache, q, *args, **more):
        out, lse = real(cache, q, *args, **more)
        rows = decoder.block_table.repeat_interleave(m, 0)
        lengths = [int(c) + i + 1 for c in state["cached"] for i in range(m)]
        seen = (out, lse, cache, q, rows[:0], [], [])
        assert_attended(*seen, rows, lengths)
        calls.append(max(lengths))
        if max(lengths) > 20:  # the bound is tight enough: the newest token left out, a token too many, a page of the prefix left out
            holed = rows.clone()
            holed[:, 0] = -1
            for t, n in ((rows, [x - 1 for x in lengths]), (rows, [x + 1 for x in lengths]), (holed, lengths)):
                with pytest.raises(AssertionError):
                    assert_attended(*seen, t, n)
        return out, lse

    monkeypatch.setattr(bcp, "bcp_kv_attend_shared", checked)
    tokens = torch.randint(0, g.VOCAB, (3, 30), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    at = torch.tensor([0, 1, 2], device="cuda")  # sequences of different lengths
    for c in decoder.caches:  # (what stands behind the newest token is not zero)
        n = c.n_pages * c.page_size
        x = torch.randn((n, c.n_heads, c.head_dim), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
        bcp.bcp_kv_write(c, x, x, torch.arange(n, device="cuda"))
    for i in range(0, 30 - m + 1, m):
        state["cached"] = (at + i).tolist()
        decoder.step_drafts(tokens[:, i:i + m], at + i)
    decoder.check()
    assert len(calls) == len(range(0, 30 - m + 1, m)) * g.LAYERS and max(calls) > 20


def test_right_drafts_are_accepted_and_wrong_ones_are_not(cuda_device, monkeypatch):
    import generate as g

    w, first, steps, n = g.merged_parameters(), torch.tensor([5, 77, 901, 300], device="cuda"), 50, 4
    tokens, _ = g.generate_with_drafts(g.Decoder(w, 4, 56, "bf16"), first, steps, n)
    real, seen = bcp.bcp_verify_drafts, []

    def checked(target, drafts, uniform, **more):
        out, accepted = real(target, drafts, uniform, **more)
        best = torch.where(target == target.amax(-1, keepdim=True), torch.arange(target.shape[-1], device="cuda"), target.shape[-1]).amin(-1)
        right = ((best[:, :n] == drafts) & (drafts >= 0)).long().cumprod(1).sum(1)
        assert torch.equal(accepted.long(), right)
        assert torch.equal(out.gather(1, right[:, None]), best.gather(1, right[:, None]))
        seen.append(int(right.sum()))
        return out, accepted

    monkeypatch.setattr(bcp, "bcp_verify_drafts", checked)
    for shift in (0, 1):  # what the first run gave, or the token next to it
        def known(history, lengths, k):
            take = lengths[:, None] + torch.arange(k, device="cuda")
            return torch.where(take <= steps, (tokens.gather(1, take.clamp_max(steps)) + shift) % g.VOCAB, -1)

        monkeypatch.setattr(g, "look_up", known)
        seen.clear()
        _, rounds = g.generate_with_drafts(g.Decoder(w, 4, 56, "bf16"), first, steps, n)
        assert len(seen) == rounds
        if shift:
            assert sum(seen) <= 4 and rounds >= 46
        else:  # ten rounds of five tokens; a tie that falls the other way ends what is known of its sequence
            assert sum(seen) >= 2 * 40 and rounds < steps
