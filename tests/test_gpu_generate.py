"""The example that merges a tensor-parallel checkpoint and generates from it, against a plain 32-bit forward pass over the
same merged parameters that recomputes every position."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def plain_logits(w, tokens, g):
    """Logits of the last position of one sequence of tokens, in 32 bits."""
    d, n = g.HEAD_DIM, len(tokens)
    f = torch.tensor([500000.0 ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64, device="cuda")
    angle = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * f
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turn(x):
        a, b = x[..., : d // 2], x[..., d // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    x = w["embed_tokens.weight"].float()[tokens]
    mask = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    for i in range(g.LAYERS):
        p = f"layers.{i}."
        qkv = (g.norm(x, w[p + "input_norm.weight"]) @ w[p + "attn.qkv.weight"].float().T).view(n, -1, d)
        q, k, v = qkv.split([g.Q_HEADS, g.KV_HEADS, g.KV_HEADS], 1)
        q, k = turn(q), turn(k).repeat_interleave(g.Q_HEADS // g.KV_HEADS, 1)
        v = v.repeat_interleave(g.Q_HEADS // g.KV_HEADS, 1)
        score = torch.einsum("qhd,khd->hqk", q, k) * d ** -0.5
        p_ = score.masked_fill(~mask, float("-inf")).softmax(-1)
        x = x + torch.einsum("hqk,khd->qhd", p_, v).reshape(n, -1) @ w[p + "attn.o.weight"].float().T
        gate, up = (g.norm(x, w[p + "post_norm.weight"]) @ w[p + "mlp.gate_up.weight"].float().T).split(g.FFN, -1)
        x = x + (torch.nn.functional.silu(gate) * up) @ w[p + "mlp.down.weight"].float().T
    return (g.norm(x, w["final_norm.weight"]) @ w["lm_head.weight"].float().T)[-1]


@pytest.mark.parametrize("cache", ["bf16", "e4m3", "int8"])
def test_merge_and_generate(cuda_device, cache):
    import generate as g

    w = g.merged_parameters()
    decoder = g.Decoder(w, 3, 40, cache, page_size=7)
    trace = g.generate(decoder, torch.tensor([5, 77, 901], device="cuda"), 40, stagger=4)
    decoder.check()
    # A layer rounds its activations to bfloat16 (2^-8) at eleven places, the ends at three more; cached values are
    # rounded by at most 2^-4 (e4m3) or half of 1/127 of a vector's largest (int8, 2^-8) on top, in each layer.  The
    # sum of all these, relative to the logits' norm, is a generous bound: roundings do not all add up.
    bound = (11 * g.LAYERS + 3) * 2.0 ** -8 + g.LAYERS * {"bf16": 2.0 ** -8, "e4m3": 2 * 2.0 ** -4, "int8": 2 * 2.0 ** -8}[cache]
    for b in range(3):
        went_in = [int(t[b]) for t, p, _ in trace if int(p[b]) >= 0]
        assert len(went_in) == 40 - 4 * b
        for n in (1, 7, 8, 25, len(went_in)):
            got = [lg[b] for _, p, lg in trace if int(p[b]) == n - 1][0]
            want = plain_logits(w, torch.tensor(went_in[:n], device="cuda"), g)
            assert float((got - want).norm() / want.norm()) < bound
