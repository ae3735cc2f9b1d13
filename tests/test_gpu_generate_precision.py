"""How precise the generating example is, and that the comparison would notice what it is there for.  Scores are spread over several
units (query and key rows of the merged parameters are made four times as large), so that positions and weights count.

The yardstick is computed: a plain forward pass that rounds where the example rounds (activations to bfloat16, keys and values to the
cache's format) is off from the one in 64 bits by some distance, and the example may be off by twice that.  The passes that
leave something out (rotation, weights, a position) have to be off by more.
"""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

TOKENS = 40
QMAX = {"e4m3": 448.0, "int8": 127.0}


def sharpened(w, g):
    w = dict(w)
    for i in range(g.LAYERS):
        name = f"layers.{i}.attn.qkv.weight"
        w[name] = w[name].clone()
        w[name][: (g.Q_HEADS + g.KV_HEADS) * g.HEAD_DIM] *= 4
    return w


def kept(x, cache):
    """Rows of x as the cache gives them back."""
    if cache not in QMAX:
        return x.bfloat16().double()
    scale = x.abs().amax(-1, keepdim=True) / QMAX[cache]
    y = x / scale
    return (y.round() if cache == "int8" else y.float().to(torch.float8_e4m3fn).double()) * scale


def logits(w, tokens, g, cache=None, change=None):
    """Logits of every position of one sequence, in 64 bits; with `cache`, rounded where the example rounds.  `change` leaves
    something out."""
    r = (lambda x: x.bfloat16().double()) if cache else (lambda x: x)
    d, n = g.HEAD_DIM, len(tokens)
    W = lambda name: w[name].double()  # noqa: E731
    f = torch.tensor([500000.0 ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64, device=tokens.device)

    def turn(x, shift=0):
        angle = (torch.arange(n, dtype=torch.float64, device=tokens.device) + shift)[:, None] * f
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        a, b = x[..., : d // 2], x[..., d // 2:]
        return x if change == "no rotation" else torch.cat([a * c - b * s, b * c + a * s], -1)

    def norm(x, weight):
        return r(x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5) * (1.0 + weight))

    x = W("embed_tokens.weight")[tokens]
    mask = torch.ones(n, n, dtype=torch.bool, device=tokens.device).tril(-1 if change == "the newest token is missed" else 0)
    mask[0, 0] = True
    for i in range(g.LAYERS):
        p = f"layers.{i}."
        qkv = r(norm(x, W(p + "input_norm.weight")) @ W(p + "attn.qkv.weight").T).view(n, -1, d)
        q, k, v = qkv.split([g.Q_HEADS, g.KV_HEADS, g.KV_HEADS], 1)
        q, k = r(turn(q, 1 if change == "queries a position off" else 0)), turn(k)
        if cache:
            k, v = kept(k, cache), kept(v, cache)
        if change == "heads exchanged":
            k = k.flip(1)
        k, v = (t.repeat_interleave(g.Q_HEADS // g.KV_HEADS, 1) for t in (k, v))
        score = torch.einsum("qhd,khd->hqk", q, k) * d ** -0.5 * (0.0 if change == "uniform weights" else 1.0)
        a = torch.softmax(score.masked_fill(~mask, float("-inf")), -1)
        x = r(x + r(r(torch.einsum("hqk,khd->qhd", a, v)).reshape(n, -1) @ W(p + "attn.o.weight").T))
        gate, up = r(norm(x, W(p + "post_norm.weight")) @ W(p + "mlp.gate_up.weight").T).split(g.FFN, -1)
        x = r(x + r(r(r(torch.nn.functional.silu(gate)) * up) @ W(p + "mlp.down.weight").T))
    return r(norm(x, W("final_norm.weight")) @ W("lm_head.weight").T)


def distance(a, b):
    """Relative distances of the logits, position by position, in the mean over the later ones."""
    return float(((a - b).norm(dim=-1) / b.norm(dim=-1))[TOKENS // 4:].mean())


@pytest.mark.parametrize("cache", ["bf16", "e4m3", "int8"])
def test_as_precise_as_its_roundings(cuda_device, cache):
    import generate as g

    w = sharpened(g.merged_parameters(), g)
    tokens = torch.randint(0, g.VOCAB, (3, TOKENS), generator=torch.Generator().manual_seed(2)).cuda()
    decoder = g.Decoder(w, 3, TOKENS, cache, page_size=7)
    got = torch.stack([decoder.step(tokens[:, s], torch.full((3,), s, device="cuda")) for s in range(TOKENS)], 1).double()
    decoder.check()
    for b in range(3):
        want = logits(w, tokens[b], g)
        bound = 2 * distance(logits(w, tokens[b], g, cache), want)
        assert distance(got[b], want) <= bound
        for change in ("no rotation", "uniform weights", "queries a position off", "the newest token is missed", "heads exchanged"):
            assert distance(logits(w, tokens[b], g, change=change), want) > bound, change
