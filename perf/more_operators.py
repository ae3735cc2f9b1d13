"""Cases of the operators of batches that share work: rotary positions with several axes (images and video beside text),
attention of sequences that share a long prefix, and the verification of drafted tokens.  Each case has a plain form
(elementary torch operations, in 32 bits where outputs are computed numbers, in 64 where a token hangs on a border) and the call
a user makes of the library; `exact` gives the definition's value in 64 bits.

Head layouts and vocabularies are those of the model shapes the package's workloads describe (32 query / 8 key heads of 128; 16 heads
of 128; 128256, 50304, 50257 and 32768 tokens), sequence lengths and batch sizes are generic.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1, "int8": 1}
QMAX = {"e4m3": 448.0, "int8": 127.0}
SMALLEST_SCALE = 2.0 ** -96
#: pairs that go by each axis (time, height, width; or height, width), in parts of 16ths of the rotated pairs
SHARES = {2: (8, 8), 3: (4, 6, 6)}


def listed():
    return [
        # one decoding step of a batch that answers questions about videos: latency counts
        {"name": "axes-step", "op": "axes", "tokens": 48, "hq": 32, "hk": 8, "dim": 128, "rot": 128, "axes": 3, "mixed": False, "layout": "half",
         "type": "bf16", "context": 8192},
        # a prompt of 16k tokens, most of them patches of frames, the axes taking turns over the frequencies
        {"name": "axes-prompt", "op": "axes", "tokens": 16384, "hq": 32, "hk": 8, "dim": 128, "rot": 128, "axes": 3, "mixed": True, "layout": "half",
         "type": "bf16", "context": 32768},
        # training: the gradient of an image encoder's rotation by row and column, 32 bits, neighbouring pairs, odd number of patches
        {"name": "axes-gradient", "op": "axes_grad", "tokens": 8191, "hq": 16, "hk": 16, "dim": 128, "rot": 64, "axes": 2, "mixed": False,
         "layout": "pairs", "type": "f32", "context": 1024},
        # the frames of a long video go into the 8-bit cache, keys rotated on the way
        {"name": "axes-write", "op": "axes_write", "tokens": 30011, "heads": 8, "dim": 128, "rot": 128, "axes": 3, "mixed": False, "layout": "half",
         "type": "bf16", "format": "e4m3", "page": 64, "context": 32768},
        # drafted tokens of one sequence over its own cache: latency counts
        {"name": "shared-drafts", "op": "shared", "groups": 1, "seqs": 5, "prefix": 4096, "tail": 20, "ragged": False, "heads": 8, "group": 4,
         "dim": 128, "type": "bf16", "format": "bf16", "page": 16},
        # questions about one long document
        {"name": "shared-batch", "op": "shared", "groups": 1, "seqs": 64, "prefix": 32768, "tail": 600, "ragged": True, "heads": 8, "group": 4,
         "dim": 128, "type": "bf16", "format": "bf16", "page": 64},
        # a serving batch under several instructions, 8-bit cache, pages of an odd size, some sequences without a prefix
        {"name": "shared-several", "op": "shared", "groups": 5, "seqs": 70, "prefix": 9000, "tail": 900, "ragged": True, "heads": 8, "group": 4,
         "dim": 128, "type": "bf16", "format": "e4m3", "page": 24},
        # many samples of one prompt: bound by the products
        {"name": "shared-samples", "op": "shared", "groups": 1, "seqs": 256, "prefix": 32768, "tail": 512, "ragged": True, "heads": 8, "group": 4,
         "dim": 128, "type": "f16", "format": "f16", "page": 64},
        # four drafted tokens of a single sequence: latency counts
        {"name": "verify-one", "op": "verify", "seqs": 1, "drafts": 4, "vocab": 32768, "draft": "logits", "ragged": False, "mixed": False,
         "type": "bf16", "pad": 1},
        # a serving batch, each sequence with its own temperature
        {"name": "verify-batch", "op": "verify", "seqs": 64, "drafts": 4, "vocab": 128256, "draft": "logits", "ragged": False, "mixed": True,
         "type": "bf16", "pad": 64},
        # probabilities that a filter has cut to a few tokens, up to seven drafts looked up in the text, an odd vocabulary
        {"name": "verify-looked-up", "op": "verify", "seqs": 37, "drafts": 7, "vocab": 50257, "draft": "none", "ragged": True, "mixed": False,
         "type": "f32", "pad": 1},
        # no drafts: the next token of every sequence is sampled
        {"name": "verify-sample", "op": "verify", "seqs": 200, "drafts": 0, "vocab": 50304, "draft": "none", "ragged": False, "mixed": True,
         "type": "f16", "pad": 1},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["axes", "axes_grad", "axes_write", "shared", "shared", "shared", "verify", "verify", "verify"])
    if op.startswith("axes"):
        dim = rng.choice([64, 96, 128, 128, 256])
        rot = rng.choice([dim, dim, dim // 2, 32])
        case = {"op": op, "dim": dim, "rot": rot, "axes": rng.choice([2, 3, 3]), "mixed": rng.random() < 0.5, "layout": rng.choice(["half", "pairs"]),
                "context": rng.choice([1024, 8192, 40000])}
        if op == "axes_write":
            heads, typ = rng.choice([1, 2, 4, 8, 16]), rng.choice(["bf16", "f16"])
            return {**case, "tokens": _log(rng, 1, min(40000, 32768 * 1024 // (heads * dim))), "heads": heads, "type": typ,
                    "format": rng.choice([typ, "e4m3"]), "page": rng.choice([1, 7, 16, 24, 64, 100])}
        hk = rng.choice([1, 2, 4, 8, 16])
        hq = hk * rng.choice([1, 2, 4, 7])
        return {**case, "tokens": _log(rng, 1, min(40000, 16384 * 40 * 128 // ((hq + hk) * dim))), "hq": hq, "hk": hk,
                "type": rng.choice(["f32", "bf16", "f16"]) if op == "axes" else rng.choice(["f32", "bf16"])}
    if op == "shared":
        typ, dim = rng.choice(["bf16", "f16"]), rng.choice([64, 96, 128, 128, 128, 256])
        heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8, 16])
        groups = rng.choice([1, 1, 2, 3, 8])
        seqs = _log(rng, groups, 256)
        most = min(32768 * 1024 // (heads * dim * groups), 256 * 32 * 32768 * 128 // (seqs * heads * group * dim), 131072)
        return {"op": op, "groups": groups, "seqs": seqs, "prefix": _log(rng, 1, most), "tail": _log(rng, 1, min(2048, 131072 * 1024 // (heads * dim * seqs))),
                "ragged": rng.random() < 0.6, "heads": heads, "group": group, "dim": dim, "type": typ, "format": rng.choice([typ, typ, "e4m3", "int8"]),
                "page": rng.choice([1, 7, 16, 16, 24, 64, 100, 128])}
    vocab = rng.choice([1000, 32768, 50257, 50304, 128256, _log(rng, 2, 200000)])
    seqs, drafts = _log(rng, 1, 256), rng.choice([0, 1, 2, 3, 4, 5, 7, 12])
    seqs = max(1, min(seqs, 64 * 9 * 128256 // ((2 * drafts + 1) * vocab)))
    return {"op": op, "seqs": seqs, "drafts": drafts, "vocab": vocab, "draft": rng.choice(["logits", "logits", "none", "probabilities"]),
            "ragged": rng.random() < 0.5, "mixed": rng.random() < 0.5, "type": rng.choice(["bf16", "bf16", "f16", "f32"]), "pad": rng.choice([1, 1, 64])}


# ------------------------------------------------------------------------------------------------ inputs
def _axes_of_pairs(case):
    """The axis that each rotated pair goes by: parts in order, or (mixed) dealt out in turn while a part lasts."""
    n = case["rot"] // 2
    parts = [n * s // 16 for s in SHARES[case["axes"]]]
    parts[0] += n - sum(parts)
    if not case["mixed"]:
        return [a for a, m in enumerate(parts) for _ in range(m)]
    return [a for turn in range(n) for a, m in enumerate(parts) if turn < m]


def _frequencies(case):
    n = case["rot"] // 2
    return 10000.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n)


def _positions(case, g):
    """[axes, tokens]: patches of frames of 24 x 36 in the order of a video, text (all axes alike) between; 2 axes: patches of an image."""
    t = torch.arange(case["tokens"], device="cuda")
    first = torch.randint(0, max(1, case["context"] - case["tokens"] - 40), (1,), generator=g, device="cuda")
    frame, patch = t // 864, t % 864
    row, column = patch // 36, patch % 36
    if case["axes"] == 2:
        return torch.stack([row + 24 * (frame % 20), column]) % case["context"]
    text = (t // 50) % 10 == 0
    at = torch.stack([first + frame, first + row, first + column])
    return torch.where(text, first + t // 10, at) % case["context"]


def _quantised(x, fmt):
    """Rows of x (any shape, last dimension a row) in an 8-bit format, with a scale each."""
    scale = (x.abs().amax(-1) / QMAX[fmt]).clamp_min(SMALLEST_SCALE)
    y = x * (1.0 / scale)[..., None]
    y = y.round() if fmt == "int8" else y
    return y.clamp(-QMAX[fmt], QMAX[fmt]).to(TYPES[fmt]), scale


def _pages(case, n_pages, g, filled):
    """The key or value pages [pages, heads, page, dim] and, for 8-bit formats, their scales [pages, heads, page]."""
    shape = (n_pages, case["heads"], case["page"], case["dim"])
    fmt = case["format"]
    if not filled:
        return torch.zeros(shape, dtype=TYPES[fmt], device="cuda"), (torch.ones(shape[:3], device="cuda") if fmt in QMAX else None)
    x = torch.randn(shape, generator=g, device="cuda")
    return _quantised(x, fmt) if fmt in QMAX else (x.to(TYPES[fmt]), None)


def _tables(order, at, lengths, page):
    """A block table (int32, a row for each length, unused places 0) over order[at:], and the first entry that is left."""
    wide, rows = max(1, -(-max(lengths) // page)), []
    for n in lengths:
        m = -(-n // page)
        rows.append(torch.cat([order[at: at + m], order.new_zeros(wide - m)]))
        at += m
    return torch.stack(rows).int(), at


def _shared_inputs(st, case, g, r):
    groups, seqs, page = case["groups"], case["seqs"], case["page"]
    prefix, own_lengths, starts = [case["prefix"]] * groups, [case["tail"]] * seqs, [seqs * i // groups for i in range(groups + 1)]
    if case["ragged"]:
        prefix = [r.randint(max(1, case["prefix"] // 3), case["prefix"]) for _ in range(groups)]
        prefix[r.randrange(groups)] = case["prefix"]
        own_lengths = [r.randint(max(1, case["tail"] // 4), case["tail"]) for _ in range(seqs)]
        if seqs > 4:  # sequences that have just begun: one token, none
            own_lengths[1], own_lengths[3] = 1, 0
        if groups > 1:  # groups of other sizes; the first and the last sequences have no prefix
            spare = max(0, min(seqs // 16, 3))
            starts = [spare] + sorted(r.randint(spare, seqs - spare) for _ in range(groups - 1)) + [seqs - spare]
    n_pages = sum(-(-n // page) for n in prefix + own_lengths) + 2
    st["k_pages"], st["k_scale"] = _pages(case, n_pages, g, True)
    st["v_pages"], st["v_scale"] = _pages(case, n_pages, g, True)
    order = torch.randperm(n_pages, generator=g, device="cuda")
    st["prefix_table"], at = _tables(order, 0, prefix, page)
    st["block_table"], _ = _tables(order, at, own_lengths, page)
    for name, x in (("prefix_lengths", prefix), ("lengths", own_lengths), ("starts", starts)):
        st[name] = torch.tensor(x, dtype=torch.int32, device="cuda")
    st["widest"] = max(1, max(b - a for a, b in zip(starts, starts[1:])))
    # queries that prefer some tokens to others
    st["q"] = (2.0 * torch.randn(seqs, case["heads"] * case["group"], case["dim"], generator=g, device="cuda")).to(TYPES[case["type"]])
    st["scale"] = case["dim"] ** -0.5


def _sampled(logits, temperature, g):
    """A token of each row, drawn from softmax(logits / temperature)."""
    noise = -torch.log(-torch.log(torch.rand(logits.shape, generator=g, device="cuda").clamp(1e-7, 1 - 1e-6)))
    return (logits.float() + noise * temperature[:, None, None]).argmax(-1)


def _filtered(logits):
    """Probabilities of the 50 likeliest tokens."""
    top, at = logits.topk(min(50, logits.shape[-1]), -1)
    return torch.zeros_like(logits).scatter_(-1, at, torch.softmax(top, -1))


def _verify_inputs(st, case, g, r):
    b, k, v, typ = case["seqs"], case["drafts"], case["vocab"], TYPES[case["type"]]
    wide = -(-v // case["pad"]) * case["pad"]
    st["temperature"] = None
    t = torch.ones(b, device="cuda")
    if case["mixed"]:
        t = st["temperature"] = torch.tensor([r.choice([0.0, 0.3, 0.7, 1.0, 1.3]) for _ in range(b)], device="cuda")
    z = 3.0 * torch.randn(b, k + 1, wide, generator=g, device="cuda")
    near = (z[:, :k] + 0.6 * torch.randn(b, k, wide, generator=g, device="cuda"))
    st["probabilities"] = case["draft"] == "probabilities" or (case["draft"] == "none" and case["type"] == "f32")
    if st["probabilities"]:
        t, st["temperature"] = torch.ones_like(t), None
        z = torch.nn.functional.pad(_filtered(z[..., :v]), (0, wide - v))
        st["drafts"] = _sampled(near[..., :v].masked_fill(near[..., :v] < near[..., :v].amax(-1, keepdim=True) - 4.0, -1e9), t, g)
        near = torch.nn.functional.pad(_filtered(near[..., :v]), (0, wide - v))
    else:
        st["drafts"] = _sampled(near[..., :v], t, g) if k else torch.zeros(b, 0, dtype=torch.int64, device="cuda")
    st["target"] = z.to(typ)[..., :v]
    st["draft"] = None if case["draft"] == "none" else near.to(typ)[..., :v]
    if case["ragged"] and k:  # fewer drafts than there is room for
        n = torch.randint(0, k + 1, (b, 1), generator=g, device="cuda")
        st["drafts"] = torch.where(torch.arange(k, device="cuda") < n, st["drafts"], -1)
    st["uniform"] = torch.rand(b, k + 1, generator=g, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = random.Random(seed)
    op, typ = case["op"], TYPES[case["type"]]
    st = {"case": case}
    if op.startswith("axes"):
        t, d = case["tokens"], case["dim"]
        angle = torch.arange(case["context"], dtype=torch.float64, device="cuda")[:, None] * _frequencies(case)
        st["table"] = torch.stack([angle.cos(), angle.sin()], 1).float()
        st["pair_axes"] = torch.tensor(_axes_of_pairs(case), device="cuda")
        st["positions"] = _positions(case, g)
        # one fused projection gives queries, keys and values: strided views of it
        hq, hk = (case["heads"], case["heads"]) if op == "axes_write" else (case["hq"], case["hk"])
        wide = torch.randn(t, (hq + 2 * hk) * d, generator=g, device="cuda").to(typ)
        st["q"], st["k"] = wide[:, : hq * d].view(t, hq, d), wide[:, hq * d: (hq + hk) * d].view(t, hk, d)
        if op == "axes_write":
            page = case["page"]
            n_pages = -(-t // page) + 3
            st["v"] = wide[:, (hq + hk) * d:].view(t, hk, d)
            st["slots"] = (torch.randperm(n_pages, generator=g, device="cuda")[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)[:t].clone()
            if t > 8:  # padding of the batch
                st["slots"][torch.randint(0, t, (t // 16 + 1,), generator=g, device="cuda")] = -1
            st["k_pages"], st["k_scale"] = _pages(case, n_pages, g, False)
            st["v_pages"], st["v_scale"] = _pages(case, n_pages, g, False)
    elif op == "shared":
        _shared_inputs(st, case, g, r)
    else:
        _verify_inputs(st, case, g, r)
    if own:
        _handles(st)
    return st


def _handles(st):
    """What a program that decodes keeps from step to step: the handles over its tensors, the buffers of its outputs, the scratch memory."""
    import paper_2407_20143_b200 as bcp

    case, op = st["case"], st["case"]["op"]
    if "table" in st:
        st["rope"] = bcp.RopeTable(st["table"], layout=case["layout"], axes=_axes_of_pairs(case))
        st["out"] = (torch.empty_like(st["q"], memory_format=torch.contiguous_format), torch.empty_like(st["k"], memory_format=torch.contiguous_format))
    if "k_pages" in st:
        st["cache"] = bcp.KvCache(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
    if op == "shared":
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(st["q"].shape[:2], dtype=torch.float32, device="cuda")
        st["workspace"] = bcp.KvWorkspace(st["cache"], st["q"].shape[1], st["q"].shape[0], shared=True)
    if op == "verify":
        st["out"] = torch.empty((case["seqs"], case["drafts"] + 1), dtype=torch.int64, device="cuda")
        st["accepted"] = torch.empty(case["seqs"], dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------ the passes
def _rotate(x, table, pair_axes, positions, layout, transposed=False):
    """x [tokens, heads, dim] in 32 bits, pair i of each head turned by the angle of the position on its axis."""
    n = table.shape[2]
    pairs = torch.arange(n, device=x.device)
    at = positions[pair_axes].T
    c, s = table[at, 0, pairs][:, None], table[at, 1, pairs][:, None]
    s = -s if transposed else s
    turned, rest = x[..., : 2 * n], x[..., 2 * n:]
    if layout == "half":
        a, b = turned[..., :n], turned[..., n:]
        return torch.cat([a * c - b * s, b * c + a * s, rest], -1)
    a, b = turned[..., 0::2], turned[..., 1::2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), rest], -1)


def _put(pages, scales, x, page, off, fmt):
    """Rows x [tokens, heads, dim], in 32 bits, into the pages."""
    if fmt in QMAX:
        y, scale = _quantised(x, fmt)
        pages.view(torch.uint8)[page, :, off] = y.view(torch.uint8)
        scales[page, :, off] = scale
    else:
        pages[page, :, off] = x.to(pages.dtype)


def _values(pages, scales, page, off):
    """The rows of the pages at (page, off), any shape of the two, in 32 bits: [..., heads, dim]."""
    x = pages.view(torch.uint8)[page, :, off].view(pages.dtype).float() if pages.element_size() == 1 else pages[page, :, off].float()
    return x if scales is None else x * scales[page, :, off][..., None]


def _part(st, q, table, lengths):
    """Softmax over the tokens of each row of a table, not yet divided: largest score, sum, weighted values.  q [rows, n, query heads, dim]."""
    case, page = st["case"], st["case"]["page"]
    rows, n, _, d = q.shape
    heads, group = case["heads"], case["group"]
    pos = torch.arange(table.shape[1] * page, device=q.device)
    where, off = table.long()[:, pos // page], (pos % page).expand(rows, -1)
    k = _values(st["k_pages"], st["k_scale"], where, off)
    q = q.view(rows, n, heads, group, d).transpose(1, 2).reshape(rows, heads, n * group, d)
    score = torch.matmul(q, k.permute(0, 2, 3, 1)) * st["scale"]
    del k
    score = score.masked_fill(~(pos < lengths[:, None])[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = (score - torch.where(top == -math.inf, torch.zeros_like(top), top)).exp()
    out = torch.matmul(p, _values(st["v_pages"], st["v_scale"], where, off).permute(0, 2, 1, 3))
    back = lambda x: x.view(rows, heads, n, group, -1).transpose(1, 2).reshape(rows, n, heads * group, -1)  # noqa: E731
    return back(top), back(p.sum(-1, keepdim=True)), back(out)


def _plain_shared(st):
    case, q, starts = st["case"], st["q"].float(), st["starts"].long()
    b = q.shape[0]
    # the sequences of each group side by side; places behind a group's last sequence are computed and dropped
    wide = st["widest"]
    seq = (starts[:-1, None] + torch.arange(wide, device=q.device)).clamp_max(b - 1)
    first = _part(st, q[seq], st["prefix_table"], st["prefix_lengths"].long())
    rows = torch.arange(b, device=q.device)
    of = (torch.searchsorted(starts, rows, right=True) - 1).clamp(0, case["groups"] - 1)
    inside = ((rows >= starts[0]) & (rows < starts[-1]))[:, None, None]
    at = (rows - starts[of]).clamp(0, wide - 1)
    m1, l1, o1 = (x[of, at] for x in first)
    m1, l1, o1 = m1.masked_fill(~inside, -math.inf), l1.masked_fill(~inside, 0.0), o1.masked_fill(~inside, 0.0)
    m2, l2, o2 = (x[:, 0] for x in _part(st, q[:, None], st["block_table"], st["lengths"].long()))
    top = torch.maximum(m1, m2)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    w1, w2 = (m1 - top).exp(), (m2 - top).exp()
    total = l1 * w1 + l2 * w2
    out = (o1 * w1 + o2 * w2) / torch.where(total == 0, torch.ones_like(total), total)
    return out.to(st["q"].dtype), (total.log() + top)[..., 0]


def _lowest_largest(z):
    """The index of each row's largest value, the lowest of equal ones."""
    return torch.where(z == z.amax(-1, keepdim=True), torch.arange(z.shape[-1], device=z.device), z.shape[-1]).amin(-1)


def _weights(z, st):
    """The probabilities that rows z [sequences, rows, vocabulary] stand for, in 64 bits."""
    z = z.double()
    if st["probabilities"] or not z.shape[1]:
        return z
    if st["temperature"] is None:
        return torch.softmax(z, -1)
    t = st["temperature"].double()[:, None, None]
    greedy = torch.zeros_like(z).scatter_(-1, _lowest_largest(z)[..., None], 1.0)
    return torch.where(t == 0, greedy, torch.softmax(z / torch.where(t == 0, 1.0, t), -1))


def _plain_verify(st):
    drafts, u = st["drafts"], st["uniform"].double()
    b, k = drafts.shape
    v = st["target"].shape[2]
    p = _weights(st["target"], st)
    token = drafts.clamp(0, v - 1)[..., None]
    q = torch.zeros_like(p[:, :k]).scatter_(-1, token, 1.0) if st["draft"] is None else _weights(st["draft"], st)
    there = (drafts >= 0).long().cumprod(1)
    good = u[:, :k] * q.gather(-1, token)[..., 0] < p[:, :k].gather(-1, token)[..., 0]
    accepted = (good.long() * there).cumprod(1).sum(1)
    rows = torch.arange(b, device=u.device)
    weight = p[rows, accepted]
    if k:
        rest = (weight - q[rows, accepted.clamp_max(k - 1)]).clamp_min(0.0)
        use = (accepted < there.sum(1))[:, None] & (rest.sum(-1, keepdim=True) > 0)
        weight = torch.where(use, rest, weight)
    line = weight.cumsum(-1)
    found = (line <= u[:, k:] * line[:, -1:]).sum(-1)
    last = v - 1 - _lowest_largest((weight > 0).flip(-1).byte())
    new = torch.minimum(found, last)
    place = torch.arange(k + 1, device=u.device)
    tokens = torch.cat([drafts, drafts.new_full((b, 1), -1)], 1)
    tokens = torch.where(place < accepted[:, None], tokens, torch.where(place == accepted[:, None], new[:, None], -1))
    return tokens, accepted.int()


def _plain(st):
    case, op = st["case"], st["case"]["op"]
    if op in ("axes", "axes_grad"):
        return tuple(_rotate(x.float(), st["table"], st["pair_axes"], st["positions"], case["layout"], op == "axes_grad").to(x.dtype)
                     for x in (st["q"], st["k"]))
    if op == "axes_write":
        used = (st["slots"] >= 0).nonzero()[:, 0]
        slots = st["slots"][used]
        page, off = slots // case["page"], slots % case["page"]
        k = _rotate(st["k"][used].float(), st["table"], st["pair_axes"], st["positions"][:, used], case["layout"])
        _put(st["k_pages"], st["k_scale"], k, page, off, case["format"])
        _put(st["v_pages"], st["v_scale"], st["v"][used].float(), page, off, case["format"])
        return [st["k_pages"], st["v_pages"]] + ([st["k_scale"], st["v_scale"]] if case["format"] in QMAX else [])
    return _plain_shared(st) if op == "shared" else _plain_verify(st)


def run(st):
    if not own:
        return _plain(st)
    import paper_2407_20143_b200 as bcp

    op = st["case"]["op"]
    if op == "axes":
        return bcp.bcp_rope((st["q"], st["k"]), st["rope"], st["positions"], out=st["out"])
    if op == "axes_grad":
        return bcp.bcp_rope_backward((st["q"], st["k"]), st["rope"], st["positions"], out=st["out"])
    if op == "axes_write":
        bcp.bcp_kv_write(st["cache"], st["k"], st["v"], st["slots"], rope=st["rope"], positions=st["positions"])
        return [st["k_pages"], st["v_pages"]] + ([st["k_scale"], st["v_scale"]] if st["k_scale"] is not None else [])
    if op == "shared":
        return bcp.bcp_kv_attend_shared(st["cache"], st["q"], st["prefix_table"], st["prefix_lengths"], st["starts"], st["block_table"], st["lengths"],
                                        scale=st["scale"], out=st["out"], lse=st["lse"], workspace=st["workspace"])
    return bcp.bcp_verify_drafts(st["target"], st["drafts"], st["uniform"], draft=st["draft"], temperature=st["temperature"],
                                 probabilities=st["probabilities"], out=st["out"], accepted=st["accepted"])


# ------------------------------------------------------------------------------------------------ 64 bits
def _turned(x, st, sign):
    """The rotation as a product of complex numbers in 64 bits, an axis after the other."""
    case, table = st["case"], st["table"]
    n = table.shape[2]
    x = x.double()
    y = x.clone()
    for axis in range(case["axes"]):
        pairs = (st["pair_axes"] == axis).nonzero()[:, 0]
        rows = table[st["positions"][axis]][:, :, pairs].double()
        w = torch.complex(rows[:, 0], sign * rows[:, 1])[:, None]
        i, j = (pairs, pairs + n) if case["layout"] == "half" else (2 * pairs, 2 * pairs + 1)
        z = torch.complex(x[..., i], x[..., j]) * w
        y[..., i], y[..., j] = z.real, z.imag
    return y


def _exact_write(st, case):
    rows = {"k": _turned(st["k"], st, 1.0), "v": st["v"].double()}
    used = st["slots"] >= 0
    at = torch.div(st["slots"][used], case["page"], rounding_mode="floor"), st["slots"][used] % case["page"]
    pages, scales = [], []
    for name in "kv":
        full, x = st[name + "_pages"].double(), rows[name][used]
        if case["format"] in QMAX:
            scale = torch.clamp(x.abs().amax(-1) / QMAX[case["format"]], min=SMALLEST_SCALE)
            all_scales = st[name + "_scale"].double()
            all_scales[at[0], :, at[1]] = scale
            scales.append(all_scales)
            x = x / scale[..., None]
        full[at[0], :, at[1]] = x
        pages.append(full)
    return pages + scales


def _tokens_of(st, case, table, n):
    """Keys and values [heads, n, dim] of the first n tokens of a row of a block table."""
    pages, got = table[: -(-n // case["page"])].long(), []
    for name in "kv":
        x = st[name + "_pages"][pages].double()
        x = x * st[name + "_scale"][pages].double()[..., None] if st[name + "_scale"] is not None else x
        got.append(x.transpose(0, 1).reshape(case["heads"], -1, case["dim"])[:, :n])
    return got


def _exact_shared(st, case):
    starts, prefix, lengths = st["starts"].tolist(), st["prefix_lengths"].tolist(), st["lengths"].tolist()
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    of = {b: g for g in range(case["groups"]) for b in range(starts[g], starts[g + 1])}
    known = (None, None)
    for b, n in enumerate(lengths):
        g = of.get(b)
        if known[0] != g:
            known = g, None if g is None else _tokens_of(st, case, st["prefix_table"][g], prefix[g])
        rows = [x for x in (known[1], _tokens_of(st, case, st["block_table"][b], n) if n else None) if x]
        if not rows:
            continue
        q = st["q"][b].double().view(case["heads"], case["group"], case["dim"])
        score = torch.cat([q @ k.transpose(1, 2) for k, _ in rows], -1) * st["scale"]
        weight = torch.softmax(score, -1)
        parts = weight.split([k.shape[1] for k, _ in rows], -1)
        out[b] = sum(w @ v for w, (_, v) in zip(parts, rows)).flatten(0, 1)
        lse[b] = torch.logsumexp(score, -1).flatten()
    return out, lse


def _exact_verify(st, case):
    """One sequence after the other, a drafted token after the other."""
    k, v = case["drafts"], case["vocab"]
    t = [1.0] * case["seqs"] if st["temperature"] is None else st["temperature"].tolist()
    tokens = torch.full((case["seqs"], k + 1), -1, dtype=torch.int64)
    accepted = torch.zeros(case["seqs"], dtype=torch.int32)
    drafts, u = st["drafts"].tolist(), st["uniform"].tolist()

    def probabilities(z, b):
        z = z.double()
        if st["probabilities"]:
            return z
        if t[b] == 0:
            best = torch.zeros_like(z)
            best[(z == z.max()).nonzero()[0, 0]] = 1.0
            return best
        return ((z - z.max()) / t[b]).exp() / ((z - z.max()) / t[b]).exp().sum()

    for b in range(case["seqs"]):
        n = 0
        weight = probabilities(st["target"][b, 0], b)
        while n < k and drafts[b][n] >= 0:
            x = drafts[b][n]
            other = torch.zeros(v, dtype=torch.float64, device="cuda")
            if st["draft"] is None:
                other[x] = 1.0
            else:
                other = probabilities(st["draft"][b, n], b)
            if not u[b][n] * float(other[x]) < float(weight[x]):
                rest = (weight - other).clamp(min=0.0)
                weight = rest if float(rest.sum()) > 0 else weight
                break
            tokens[b, n] = x
            n += 1
            weight = probabilities(st["target"][b, n], b)
        line = weight.cumsum(0)
        at = int(torch.searchsorted(line, u[b][k] * line[-1], right=True))
        tokens[b, n] = min(at, int(weight.nonzero()[-1, 0]))
        accepted[b] = n
    return tokens.cuda(), accepted.cuda()


def exact(case, seed):
    """Values before they are rounded to the output's type."""
    st = prepare(case, seed)
    op = case["op"]
    if op in ("axes", "axes_grad"):
        return tuple(_turned(st[x], st, -1.0 if op == "axes_grad" else 1.0) for x in "qk")
    if op == "axes_write":
        return _exact_write(st, case)
    return _exact_shared(st, case) if op == "shared" else _exact_verify(st, case)


# ------------------------------------------------------------------------------------------------ floors
def work(case):
    """Every input read once and every output written once.  Lengths of ragged batches are taken at their mean."""
    op, es = case["op"], SIZE[case["type"]]
    if op == "verify":
        # the rows of all drafted tokens count, although those behind a rejected one need not be read
        b, k, v = case["seqs"], case["drafts"], case["vocab"]
        rows = b * (k + 1 + (k if case["draft"] != "none" else 0))
        return {"bytes": rows * v * es + b * (k * 8 + (k + 1) * 12 + 8), "flops": rows * v * 4}
    d = case["dim"]
    # a row of the rotation table has a cosine and a sine for every pair
    turn = case["tokens"] * 4 * case["rot"] + case["tokens"] * case["axes"] * 8 if op != "shared" else 0
    if op in ("axes", "axes_grad"):
        # tokens share rows: patches of a frame lie in a few dozen rows and columns
        turn = min(turn, case["tokens"] * case["axes"] * 8 + case["context"] * 4 * case["rot"])
        rows = case["tokens"] * (case["hq"] + case["hk"])
        return {"bytes": rows * d * 2 * es + turn, "flops": rows * 3 * case["rot"]}
    fmt = case["format"]
    row = d * SIZE[fmt] + (4 if fmt in QMAX else 0)
    if op == "axes_write":
        rows = case["tokens"] * case["heads"] * 2
        return {"bytes": rows * (row + d * es) + case["tokens"] * 8 + min(turn, case["tokens"] * case["axes"] * 8 + case["context"] * 4 * case["rot"]),
                "flops": rows * d * 2}
    n, prefix, tail = case["seqs"], case["prefix"], case["tail"]
    if case["ragged"]:
        prefix = prefix * 2 / 3 if case["groups"] > 1 else prefix
        tail = tail * 5 / 8
    tokens = prefix * case["groups"] + tail * n
    return {"bytes": tokens * case["heads"] * 2 * row + n * case["heads"] * case["group"] * (2 * d * es + 4) + n * 4,
            "flops": 4 * (prefix + tail) * n * case["heads"] * case["group"] * d}
