"""Verification where rows hold no numbers: a NaN or an infinity in the row that the next token comes from, in a draft's row, at the draft itself, elsewhere."""
import math

import pytest
import torch

import paper_2407_20143_b200 as bcp

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def _weights(v, dtype, seed=1):
    """[1, 2, v] weights of the target, [1, 1, v] of the draft: the draft's token 5 has none in the target, so it is rejected."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    p = torch.rand((1, 2, v), generator=g, device="cuda") + 0.1
    q = torch.rand((1, 1, v), generator=g, device="cuda") + 0.1
    p[0, 0, 5] = 0.0
    return (p / p.sum(-1, keepdim=True)).to(dtype), (q / q.sum(-1, keepdim=True)).to(dtype)


def _verify(p, q, u=(0.5, 0.4), draft=5, **more):
    tokens, accepted = bcp.bcp_verify_drafts(p, torch.tensor([[draft]], device="cuda"), torch.tensor([u], device="cuda"), draft=q, **more)
    return tokens[0].tolist(), int(accepted)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("v", [30, 1000, 40001])
def test_weights_that_are_no_numbers(cuda_device, dtype, v):
    p, q = _weights(v, dtype)
    for draft in (q, None):
        (token, behind), accepted = _verify(p, draft, probabilities=True)
        assert accepted == 0 and 0 <= token < v and behind == -1
    for at in (0, 5, 17, v - 1):
        for bad in (math.nan, math.inf):
            broken = p.clone()
            broken[0, 0, at] = bad
            for draft in (q, None):
                # (an infinite weight at the draft is more than any other: the draft is accepted, and the row behind it has numbers)
                if at == 5 and bad == math.inf:
                    (token, behind), accepted = _verify(broken, draft, probabilities=True)
                    assert accepted == 1 and token == 5 and 0 <= behind < v
                else:
                    assert _verify(broken, draft, probabilities=True) == ([-1, -1], 0)
        # in the draft's row: it says nothing, the target's row itself is drawn from
        broken = q.clone()
        broken[0, 0, at] = math.nan
        plain = bcp.bcp_verify_drafts(p[:, :1], torch.zeros((1, 0), dtype=torch.int64, device="cuda"), torch.tensor([[0.4]], device="cuda"), probabilities=True)
        assert _verify(p, broken, probabilities=True) == ([int(plain[0]), -1], 0)
    # behind an accepted draft
    broken = p.clone()
    broken[0, 1, 11] = math.nan
    for draft in (q, None):
        assert _verify(broken, draft, u=(0.0, 0.4), draft=6, probabilities=True) == ([6, -1], 1)
