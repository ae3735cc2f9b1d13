"""From a checkpoint saved under tensor parallelism to generated tokens, on one GPU.

The parameters of a small Llama-shaped model (synthetic, random) lie in two blobs, as two tensor-parallel
ranks saved them.  They are resharded for a single rank (bcp_plan, bcp_reshard), and the merged parameters
generate tokens: keys are rotated and written into a paged cache as they are made (bcp_kv_write), queries
are rotated (bcp_rope) and attend over the cache (bcp_kv_attend).  Sequences enter the batch one after the other, so
their lengths differ; one that has not begun has length 0 and its slot is negative.

    python examples/generate.py [--cache bf16|e4m3|int8] [--steps 64]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2407_20143_b200 as bcp  # noqa: E402
from workloads import fills  # noqa: E402
from workloads.configs import PARAMS_ONLY  # noqa: E402
from workloads.layouts import Parallelism, llama_model, reshard_case  # noqa: E402

LAYERS, HIDDEN, Q_HEADS, KV_HEADS, FFN, VOCAB = 2, 512, 8, 2, 1024, 1000
HEAD_DIM = HIDDEN // Q_HEADS
CACHES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def merged_parameters(device="cuda"):
    """Name -> bfloat16 tensor, views into the one target buffer that the reshard filled."""
    model = llama_model("llama-small", L=LAYERS, H=HIDDEN, nq=Q_HEADS, nkv=KV_HEADS, F=FFN, V=VOCAB, fused=True, tied=False)
    case = reshard_case("merge", model, Parallelism(tp=2), Parallelism(tp=1), PARAMS_ONLY, "normal", seed=7)
    saved = fills.fill_state(case.src, case.key_ids, "normal", case.seed, device)
    target = [torch.zeros(n, dtype=torch.uint8, device=device) for n in case.dst.buf_bytes]
    plan = bcp.bcp_plan(case.src.metas, case.src.buf_bytes, case.dst.metas, case.dst.buf_bytes)
    bcp.bcp_reshard(plan, saved, target)
    bcp.bcp_plan_device_status(plan)
    start = {}
    for m in case.dst.metas:  # a fused tensor has an entry for each of its blocks of rows, one behind the other
        start[m.fqn] = min(start.get(m.fqn, m.byte_offset), m.byte_offset)
    shapes = {m.fqn: m.global_shape for m in case.dst.metas}
    out = {}
    for name, at in start.items():
        n = 2 * int(torch.Size(shapes[name]).numel())
        out[name] = target[0][at:at + n].view(torch.bfloat16).view(shapes[name])
    return out


def norm(x, weight):
    y = x.float()
    return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-5) * (1.0 + weight.float())).to(x.dtype)


class Decoder:
    """One token per sequence and step over a paged cache."""

    def __init__(self, weights, max_seqs: int, max_tokens: int, cache: str = "e4m3", page_size: int = 16):
        self.w = weights
        pages = -(-max_tokens // page_size)
        self.rope = bcp.RopeTable.build(bcp.rope_frequencies(HEAD_DIM, base=500000.0), max_tokens)
        self.caches = [bcp.KvCache.empty(max_seqs * pages, KV_HEADS, page_size, HEAD_DIM, CACHES[cache]) for _ in range(LAYERS)]
        # pages are handed out in no particular order
        self.block_table = torch.randperm(max_seqs * pages, generator=torch.Generator().manual_seed(1)).int().view(max_seqs, pages).cuda()
        self.work = bcp.KvWorkspace(self.caches[0], Q_HEADS, max_seqs)
        self.rows = torch.arange(max_seqs, device="cuda")

    def step(self, tokens, positions):
        """Logits (float32) after one more token for every sequence; a position of -1: the sequence has not begun."""
        slots = self.caches[0].slots(self.block_table, self.rows, positions)
        lengths = (positions + 1).int()
        n = tokens.shape[0]
        x = self.w["embed_tokens.weight"][tokens]
        for i, cache in enumerate(self.caches):
            p = f"layers.{i}."
            qkv = (norm(x, self.w[p + "input_norm.weight"]) @ self.w[p + "attn.qkv.weight"].T).view(n, Q_HEADS + 2 * KV_HEADS, HEAD_DIM)
            q, k, v = qkv.split([Q_HEADS, KV_HEADS, KV_HEADS], 1)
            bcp.bcp_rope(q, self.rope, positions, out=q)
            bcp.bcp_kv_write(cache, k, v, slots, rope=self.rope, positions=positions)
            out, _ = bcp.bcp_kv_attend(cache, q, self.block_table, lengths, workspace=self.work)
            x = x + out.view(n, HIDDEN) @ self.w[p + "attn.o.weight"].T
            gate, up = (norm(x, self.w[p + "post_norm.weight"]) @ self.w[p + "mlp.gate_up.weight"].T).split(FFN, -1)
            x = x + (torch.nn.functional.silu(gate) * up) @ self.w[p + "mlp.down.weight"].T
        return (norm(x, self.w["final_norm.weight"]) @ self.w["lm_head.weight"].T).float()

    def check(self):
        self.rope.check()
        for c in self.caches:
            c.check()


def generate(decoder: Decoder, first_tokens, steps: int, stagger: int = 3):
    """Greedy generation; sequence b begins at step b * stagger with first_tokens[b].  Returns, per step, the tokens that
    went in, their positions and the logits that came out."""
    tokens, begin = first_tokens.clone(), torch.arange(len(first_tokens), device=first_tokens.device) * stagger
    trace = []
    for s in range(steps):
        positions = torch.where(begin <= s, s - begin, -1)
        logits = decoder.step(tokens, positions)
        trace.append((tokens, positions, logits))
        tokens = torch.where(positions >= 0, logits.argmax(-1), tokens)
    return trace


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--cache", choices=sorted(CACHES), default="e4m3")
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--sequences", type=int, default=8)
    a = ap.parse_args()
    decoder = Decoder(merged_parameters(), a.sequences, a.steps, a.cache)
    first = torch.arange(a.sequences, device="cuda") * 17 % VOCAB
    generate(decoder, first, min(a.steps, 4))
    torch.cuda.synchronize()
    t = time.perf_counter()
    trace = generate(decoder, first, a.steps)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t) * 1e3 / a.steps
    decoder.check()
    print(f"{a.sequences} sequences, {a.steps} steps, {a.cache} cache: {ms:.3f} ms a step")
    print("sequence 0:", torch.stack([x[0][0] for x in trace]).tolist())


if __name__ == "__main__":
    main()
