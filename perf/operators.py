"""Cases of the decoding operators: rotary positions, the paged key-value cache (written, read back) and
the attention of one new token over it.  Each case has a plain form (elementary torch operations in 32
bits) and the call a user makes of the library; `exact` gives the definition's value in 64 bits.

Head layouts are those of the model shapes the package's workloads describe (32 query / 8 key heads of
128; 16 heads of 128; 4 heads of 64), sequence lengths and batch sizes are generic.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1, "int8": 1}
QMAX = {"e4m3": 448.0, "int8": 127.0}
SMALLEST_SCALE = 2.0 ** -96


def listed():
    return [
        # one decoding step of a small batch: query and key heads rotated, latency counts
        {"name": "rope-decode", "op": "rope", "tokens": 16, "hq": 32, "hk": 8, "dim": 128, "rot": 128, "layout": "half", "type": "bf16",
         "context": 8192, "stretch": 1.0},
        # a prompt of 16k tokens, context stretched to four times its trained length
        {"name": "rope-prompt", "op": "rope", "tokens": 16384, "hq": 32, "hk": 8, "dim": 128, "rot": 128, "layout": "half", "type": "bf16",
         "context": 32768, "stretch": 4.0},
        # training: the gradient of a rotation of half of each head, neighbouring pairs, 32-bit gradients, odd number of tokens
        {"name": "rope-gradient", "op": "rope_grad", "tokens": 8191, "hq": 16, "hk": 16, "dim": 128, "rot": 64, "layout": "pairs", "type": "f32",
         "context": 8192, "stretch": 1.0},
        # one decoding step: 64 sequences each add a token to an 8-bit cache, keys rotated on the way
        {"name": "write-step", "op": "write", "tokens": 64, "heads": 8, "dim": 128, "rot": 128, "layout": "half", "type": "bf16", "format": "e4m3",
         "page": 16, "context": 8192},
        # a long prompt goes into the 8-bit cache
        {"name": "write-prompt", "op": "write", "tokens": 32768, "heads": 8, "dim": 128, "rot": 128, "layout": "half", "type": "bf16", "format": "e4m3",
         "page": 64, "context": 32768},
        # unquantised cache, pages of an odd size, partial rotation of neighbouring pairs, many heads
        {"name": "write-odd-pages", "op": "write", "tokens": 5001, "heads": 16, "dim": 128, "rot": 32, "layout": "pairs", "type": "f16", "format": "f16",
         "page": 13, "context": 8192},
        # the whole cache of some sequences read back, to continue a prompt in parts or to hand it on
        {"name": "read-long", "op": "read", "tokens": 65536, "heads": 8, "dim": 128, "type": "bf16", "format": "e4m3", "page": 16},
        # a few hundred tokens of a small model's 8-bit integer cache, with gaps
        {"name": "read-few", "op": "read", "tokens": 333, "heads": 4, "dim": 64, "type": "f16", "format": "int8", "page": 24},
        # a single sequence at the beginning of an answer: latency counts
        {"name": "attend-one", "op": "attend", "seqs": 1, "longest": 600, "ragged": False, "heads": 8, "group": 4, "dim": 128, "type": "bf16",
         "format": "bf16", "page": 16, "window": 0},
        # a serving batch over the 8-bit cache
        {"name": "attend-batch", "op": "attend", "seqs": 64, "longest": 4096, "ragged": True, "heads": 8, "group": 4, "dim": 128, "type": "bf16",
         "format": "e4m3", "page": 64, "window": 0},
        # one long document
        {"name": "attend-long", "op": "attend", "seqs": 1, "longest": 131072, "ragged": False, "heads": 8, "group": 4, "dim": 128, "type": "bf16",
         "format": "bf16", "page": 64, "window": 0},
        # as many key as query heads, integer cache, odd pages, a sliding window, sequences of no and of one token among them
        {"name": "attend-window", "op": "attend", "seqs": 37, "longest": 2500, "ragged": True, "heads": 16, "group": 1, "dim": 128, "type": "f16",
         "format": "int8", "page": 24, "window": 1000},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "rope_grad", "write", "read", "attend", "attend"])
    dim = rng.choice([64, 96, 128, 128, 256])
    layout = rng.choice(["half", "pairs"])
    rot = rng.choice([dim, dim, dim // 2, 32])
    if op in ("rope", "rope_grad"):
        hk = rng.choice([1, 2, 4, 8, 16])
        hq = hk * rng.choice([1, 2, 4, 7])
        most = 16384 * 40 * 128 // ((hq + hk) * dim)
        return {"op": op, "tokens": _log(rng, 1, min(40000, most)), "hq": hq, "hk": hk, "dim": dim, "rot": rot, "layout": layout,
                "type": rng.choice(["f32", "bf16", "f16"]) if op == "rope" else rng.choice(["f32", "bf16"]),
                "context": rng.choice([8192, 40000]), "stretch": rng.choice([1.0, 2.0, 8.0])}
    page = rng.choice([1, 7, 16, 16, 24, 32, 64, 100, 128])
    heads = rng.choice([1, 2, 4, 8, 16])
    typ = rng.choice(["bf16", "f16"])
    fmt = rng.choice([typ, "e4m3", "e4m3", "int8"])
    if op == "write":
        # an integer cache is written in cases of "read" too: what is compared here are floating values
        fmt = "e4m3" if fmt == "int8" else fmt
        return {"op": op, "tokens": _log(rng, 1, min(40000, 32768 * 1024 // (heads * dim))), "heads": heads, "dim": dim, "rot": rot, "layout": layout,
                "type": typ, "format": fmt, "page": page, "context": 40000}
    if op == "read":
        return {"op": op, "tokens": _log(rng, 1, min(100000, 65536 * 1024 // (heads * dim))), "heads": heads, "dim": dim, "type": typ, "format": fmt,
                "page": page}
    seqs = _log(rng, 1, 64)
    most = min(131072, 131072 * 1024 // (heads * dim * seqs) + 1)
    return {"op": op, "seqs": seqs, "longest": _log(rng, 1, most), "ragged": rng.random() < 0.6, "heads": heads, "group": rng.choice([1, 2, 4, 5, 8, 16]),
            "dim": dim, "type": typ, "format": fmt, "page": page, "window": rng.choice([0, 0, 0, 128, 1000])}


# ------------------------------------------------------------------------------------------------ inputs
def _table(context, rot, stretch):
    """Cosines and sines [context, 2, rot / 2]; slow frequencies divided by `stretch`, fast ones kept, a ramp between."""
    n = rot // 2
    f = 10000.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n)
    if stretch != 1.0:
        turns = context / stretch * f / (2 * math.pi)
        keep = ((turns - 1.0) / 3.0).clamp(0.0, 1.0)
        f = f * keep + f / stretch * (1.0 - keep)
    angle = torch.arange(context, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack([angle.cos(), angle.sin()], 1).float()


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


def _lengths(case, r):
    n, most = case["seqs"], case["longest"]
    if not case["ragged"]:
        return [most] * n
    got = [r.randint(max(1, most // 4), most) for _ in range(n)]
    got[r.randrange(n)] = most
    if n > 4:  # a sequence that has just begun, and one that has nothing yet
        got[1], got[3] = 1, 0
    return got


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = random.Random(seed)
    op, typ = case["op"], TYPES[case["type"]]
    st = {"case": case}
    if op in ("rope", "rope_grad"):
        hq, hk, d, t = case["hq"], case["hk"], case["dim"], case["tokens"]
        # one fused projection gives queries, keys and values: the first two are strided views of it
        wide = torch.randn(t, (hq + 2 * hk) * d, generator=g, device="cuda").to(typ)
        st["q"] = wide[:, : hq * d].view(t, hq, d)
        st["k"] = wide[:, hq * d: (hq + hk) * d].view(t, hk, d)
        st["table"] = _table(case["context"], case["rot"], case["stretch"])
        st["positions"] = torch.randint(0, case["context"], (t,), generator=g, device="cuda")
    elif op in ("write", "read"):
        h, d, t, page = case["heads"], case["dim"], case["tokens"], case["page"]
        n_pages = -(-t // page) + 3
        st["slots"] = (torch.randperm(n_pages, generator=g, device="cuda")[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)[:t].clone()
        if t > 8:  # padding of the batch
            st["slots"][torch.randint(0, t, (t // 16 + 1,), generator=g, device="cuda")] = -1
        st["k_pages"], st["k_scale"] = _pages(case, n_pages, g, op == "read")
        st["v_pages"], st["v_scale"] = _pages(case, n_pages, g, op == "read")
        if op == "write":
            wide = torch.randn(t, 2 * h * d, generator=g, device="cuda").to(typ)
            st["k"], st["v"] = wide[:, : h * d].view(t, h, d), wide[:, h * d:].view(t, h, d)
            st["table"] = _table(case["context"], case["rot"], 1.0)
            st["positions"] = torch.randint(0, case["context"], (t,), generator=g, device="cuda")
    else:
        lens, page = _lengths(case, r), case["page"]
        wide = max(1, -(-max(lens) // page))
        n_pages = sum(-(-n // page) for n in lens) + 2
        st["k_pages"], st["k_scale"] = _pages(case, n_pages, g, True)
        st["v_pages"], st["v_scale"] = _pages(case, n_pages, g, True)
        order = torch.randperm(n_pages, generator=g, device="cuda")
        table, at = [], 0
        for n in lens:
            m = -(-n // page)
            table.append(torch.cat([order[at: at + m], order.new_zeros(wide - m)]))
            at += m
        st["block_table"] = torch.stack(table).int()
        st["lengths"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        # queries that prefer some tokens to others
        st["q"] = (2.0 * torch.randn(case["seqs"], case["heads"] * case["group"], case["dim"], generator=g, device="cuda")).to(typ)
        st["scale"] = case["dim"] ** -0.5
    if own:
        _handles(st)
    return st


def _handles(st):
    """What a program that decodes keeps from step to step: the handles over its tensors, the buffers of its outputs, the scratch memory."""
    import paper_2407_20143_b200 as bcp

    case, op = st["case"], st["case"]["op"]
    if "table" in st:
        st["rope"] = bcp.RopeTable(st["table"], layout=case["layout"])
    if op in ("rope", "rope_grad"):
        st["out"] = (torch.empty_like(st["q"], memory_format=torch.contiguous_format), torch.empty_like(st["k"], memory_format=torch.contiguous_format))
    else:
        st["cache"] = bcp.KvCache(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
    if op == "read":
        shape = (case["tokens"], case["heads"], case["dim"])
        st["out"] = tuple(torch.empty(shape, dtype=TYPES[case["type"]], device="cuda") for _ in range(2))
    if op == "attend":
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(st["q"].shape[:2], dtype=torch.float32, device="cuda")
        st["workspace"] = bcp.KvWorkspace(st["cache"], st["q"].shape[1], st["q"].shape[0])


# ------------------------------------------------------------------------------------------------ the passes
def _rotate(x, table, positions, layout, transposed=False):
    """x [tokens, heads, dim] in 32 bits, the first rot dimensions of each head rotated."""
    n = table.shape[2]
    c, s = table[positions, 0][:, None], table[positions, 1][:, None]
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


def _plain_attend(st):
    case, q, lengths = st["case"], st["q"].float(), st["lengths"].long()
    b, hq, d = q.shape
    page, heads, group = case["page"], case["heads"], case["group"]
    pos = torch.arange(st["block_table"].shape[1] * page, device=q.device)
    where, off = st["block_table"].long()[:, pos // page], (pos % page).expand(b, -1)
    k = _values(st["k_pages"], st["k_scale"], where, off)
    score = torch.matmul(q.view(b, heads, group, d), k.permute(0, 2, 3, 1)) * st["scale"]
    del k
    keep = pos < lengths[:, None]
    if case["window"]:
        keep &= pos >= lengths[:, None] - case["window"]
    score = score.masked_fill(~keep[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = (score - top).exp()
    total = p.sum(-1, keepdim=True)
    v = _values(st["v_pages"], st["v_scale"], where, off)
    out = torch.matmul(p, v.permute(0, 2, 1, 3)) / torch.where(total == 0, torch.ones_like(total), total)
    return out.view(b, hq, d).to(st["q"].dtype), (total.log() + top).view(b, hq)


def _plain(st):
    case, op = st["case"], st["case"]["op"]
    if op in ("rope", "rope_grad"):
        return tuple(_rotate(x.float(), st["table"], st["positions"], case["layout"], op == "rope_grad").to(x.dtype) for x in (st["q"], st["k"]))
    if op == "write":
        used = (st["slots"] >= 0).nonzero()[:, 0]
        slots = st["slots"][used]
        page, off = slots // case["page"], slots % case["page"]
        k = _rotate(st["k"][used].float(), st["table"], st["positions"][used], case["layout"])
        _put(st["k_pages"], st["k_scale"], k, page, off, case["format"])
        _put(st["v_pages"], st["v_scale"], st["v"][used].float(), page, off, case["format"])
        return [st["k_pages"], st["v_pages"]] + ([st["k_scale"], st["v_scale"]] if case["format"] in QMAX else [])
    if op == "read":
        slots = st["slots"].clamp_min(0)
        page, off, there = slots // case["page"], slots % case["page"], (st["slots"] >= 0)[:, None, None]
        typ = TYPES[case["type"]]
        return tuple((_values(p, s, page, off) * there).to(typ) for p, s in ((st["k_pages"], st["k_scale"]), (st["v_pages"], st["v_scale"])))
    return _plain_attend(st)


def run(st):
    if not own:
        return _plain(st)
    import paper_2407_20143_b200 as bcp

    case, op = st["case"], st["case"]["op"]
    if op == "rope":
        return bcp.bcp_rope((st["q"], st["k"]), st["rope"], st["positions"], out=st["out"])
    if op == "rope_grad":
        return bcp.bcp_rope_backward((st["q"], st["k"]), st["rope"], st["positions"], out=st["out"])
    if op == "write":
        bcp.bcp_kv_write(st["cache"], st["k"], st["v"], st["slots"], rope=st["rope"], positions=st["positions"])
        return [st["k_pages"], st["v_pages"]] + ([st["k_scale"], st["v_scale"]] if case["format"] in QMAX else [])
    if op == "read":
        return bcp.bcp_kv_read(st["cache"], st["slots"], out=st["out"])
    return bcp.bcp_kv_attend(st["cache"], st["q"], st["block_table"], st["lengths"], scale=st["scale"], window=case["window"], out=st["out"],
                             lse=st["lse"], workspace=st["workspace"])


# ------------------------------------------------------------------------------------------------ 64 bits
def _turned(x, table, positions, layout, sign):
    """The rotation as a product of complex numbers in 64 bits."""
    n = table.shape[2]
    w = torch.complex(table[positions, 0].double(), sign * table[positions, 1].double())[:, None]
    x = x.double()
    y = x.clone()
    i = slice(0, n) if layout == "half" else slice(0, 2 * n, 2)
    j = slice(n, 2 * n) if layout == "half" else slice(1, 2 * n, 2)
    z = torch.complex(x[..., i], x[..., j]) * w
    y[..., i], y[..., j] = z.real, z.imag
    return y


def exact(case, seed):
    """Values before they are rounded to the output's type."""
    st = prepare(case, seed)
    op = case["op"]
    if op in ("rope", "rope_grad"):
        return tuple(_turned(st[x], st["table"], st["positions"], case["layout"], -1.0 if op == "rope_grad" else 1.0) for x in "qk")
    if op == "write":
        rows = {"k": _turned(st["k"], st["table"], st["positions"], case["layout"], 1.0), "v": st["v"].double()}
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
    if op == "read":
        got = []
        for name in "kv":
            flat = st[name + "_pages"].double()
            flat = flat * st[name + "_scale"].double()[..., None] if st[name + "_scale"] is not None else flat
            flat = flat.transpose(1, 2).reshape(-1, case["heads"], case["dim"])
            got.append(flat[st["slots"].clamp_min(0)] * (st["slots"] >= 0).double()[:, None, None])
        return tuple(got)
    outs, sums = [], []
    for b, n in enumerate(st["lengths"].tolist()):
        q = st["q"][b].double().view(case["heads"], case["group"], case["dim"])
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == 0:
            outs.append(torch.zeros_like(q).flatten(0, 1))
            sums.append(torch.full((case["heads"] * case["group"],), -math.inf, dtype=torch.float64, device=q.device))
            continue
        pages = st["block_table"][b, : -(-n // case["page"])].long()
        rows = []
        for name in "kv":
            x = st[name + "_pages"][pages].double()
            x = x * st[name + "_scale"][pages].double()[..., None] if st[name + "_scale"] is not None else x
            rows.append(x.transpose(0, 1).reshape(case["heads"], -1, case["dim"])[:, first:n])
        score = q @ rows[0].transpose(1, 2) * st["scale"]
        outs.append((torch.softmax(score, -1) @ rows[1]).flatten(0, 1))
        sums.append(torch.logsumexp(score, -1).flatten())
    return torch.stack(outs), torch.stack(sums)


# ------------------------------------------------------------------------------------------------ floors
def work(case):
    """Every input read once and every output written once.  Lengths of ragged batches are taken at their mean."""
    op, d, es = case["op"], case["dim"], SIZE[case["type"]]
    if op in ("rope", "rope_grad"):
        rows = case["tokens"] * (case["hq"] + case["hk"])
        return {"bytes": rows * d * 2 * es + case["tokens"] * (8 + 4 * case["rot"]), "flops": rows * 3 * case["rot"]}
    fmt = case["format"]
    row = d * SIZE[fmt] + (4 if fmt in QMAX else 0)
    if op in ("write", "read"):
        rows = case["tokens"] * case["heads"] * 2
        turn = case["tokens"] * 4 * case["rot"] if op == "write" else 0
        return {"bytes": rows * (row + d * es) + case["tokens"] * 8 + turn, "flops": rows * d * 2}
    n, most = case["seqs"], case["longest"]
    seen = (lambda x: min(x, case["window"])) if case["window"] else (lambda x: x)
    mean = seen(most) if not case["ragged"] else sum(seen(max(1, most // 4) + (most - max(1, most // 4)) * i / 16) for i in range(17)) / 17
    tokens = n * mean
    return {"bytes": tokens * case["heads"] * 2 * row + n * case["heads"] * case["group"] * (2 * d * es + 4) + n * 4,
            "flops": 4 * tokens * case["heads"] * case["group"] * d}
