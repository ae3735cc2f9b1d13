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


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("v", [9, 1000, 40001, 128256])
def test_greedy_rows_that_hold_no_numbers(cuda_device, dtype, v):
    # a NaN: no logit is the largest, so no draft is it either; +infinity is the largest logit
    b, greedy = 6, torch.zeros(6, device="cuda")
    z = torch.randn((b, 2, v), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(dtype)
    best, behind = (torch.where(z == z.amax(-1, keepdim=True), torch.arange(v, device="cuda"), v).amin(-1)).unbind(1)
    for at in (0, 3, v // 2, v - 1):
        broken, drafts = z.clone(), best[:, None].clone()
        broken[0, 0, at] = math.nan
        broken[1, 0, at] = -math.nan
        broken[2, 0, at] = math.inf
        broken[3, 0, at], drafts[3] = math.inf, at
        broken[4, 1, at] = math.nan                        # behind the accepted draft
        broken[5, 0, :] = -math.inf
        broken[5, 0, at], drafts[5] = math.nan, at         # nothing but a NaN
        for draft in (None, z[:, :1]):
            tokens, accepted = bcp.bcp_verify_drafts(broken, drafts, torch.full((b, 2), 0.5, device="cuda"), draft=draft, temperature=greedy)
            second = at if int(best[2]) != at else int(behind[2])
            hit = int(best[2]) == at
            assert accepted.tolist() == [0, 0, int(hit), 1, 1, 0]
            assert tokens.tolist() == [[-1, -1], [-1, -1], [at, second] if hit else [at, -1], [at, int(behind[3])], [int(best[4]), -1], [-1, -1]]
    # warm rows of the same batch: a NaN or +infinity anywhere
    warm, _ = bcp.bcp_verify_drafts(broken, drafts, torch.full((b, 2), 0.5, device="cuda"))
    assert warm[[0, 1, 2, 5], 0].tolist() == [-1] * 4


def _sampled(weights, u):
    """The token that each random number draws from one row of weights (float32 [v], probabilities=True)."""
    n = len(u)
    tokens, _ = bcp.bcp_verify_drafts(weights.cuda().expand(n, 1, -1), torch.zeros((n, 0), dtype=torch.int64, device="cuda"),
                                      torch.tensor(u, dtype=F32, device="cuda")[:, None], probabilities=True)
    return tokens[:, 0].tolist()


def _want(weights, u):
    """The same in 64 bits.  Sums of whole numbers below 2^53, and their products with numbers of 24 bits below 2^29, are exact in any order."""
    line = weights.double().cumsum(0)
    return torch.searchsorted(line, torch.tensor(u, dtype=F32).double() * line[-1], right=True).tolist()


@pytest.mark.parametrize("v,big,border", [(512, 2 ** 24, 256), (600, 2 ** 24, 512), (5000, 2 ** 25, 1024), (40001, 2 ** 24, 20224)])
def test_sums_of_weights_are_held_in_64_bits(cuda_device, v, big, border):
    # ones beside weights of 2^24 and more, which sums of 32 bits round away; places one apart around the end of a stretch of 256 tokens
    weights = torch.ones(v)
    weights[border - 256] = weights[border] = big
    line = weights.double().cumsum(0)
    at = torch.tensor([float(line[border - 1]) + d for d in range(-300, 40, 3)], dtype=torch.float64) / float(line[-1])
    u = at.float().clamp(0, 1 - 2.0 ** -24).tolist()
    want = _want(weights, u)
    assert sum(border - 256 < w < border for w in want) > 20 and border in want  # (on both sides)
    assert _sampled(weights, u) == want


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [8, 300, 40001])
def test_large_weights(cuda_device, dtype, v):
    # any two add up to more than binary32 holds
    u = [0.0, 0.2503, 0.7501, 1 - 2.0 ** -24]
    n = len(u)
    weights = torch.full((1, 1, v), torch.finfo(dtype).max, dtype=dtype, device="cuda").expand(n, 1, v)
    tokens, _ = bcp.bcp_verify_drafts(weights, torch.zeros((n, 0), dtype=torch.int64, device="cuda"), torch.tensor(u, device="cuda")[:, None], probabilities=True)
    assert tokens[:, 0].tolist() == [int(torch.tensor(x, dtype=F32).double() * v) for x in u]
