"""Verification of drafted tokens against the definition in 64 bits, one sequence and one draft after the other.

A token hangs on a comparison of sums whose terms are binary32: a term exp((z - m) / T) has an exponent of at most 30 where it counts, off by four
roundings (4 * 2^-24 * 30), and 2^-22 of itself, together below 1e-5 of the weights' sum.  So the drawn place has to lie in the stretch of the token that
came out, widened by that much at either end, and where the place is farther than that from both ends the token is the definition's.  Where a draft's own
comparison is as close, the sequence is not compared; nearly all have wider margins, which is asserted."""
import math

import pytest
import torch

import paper_2407_20143_b200 as bcp
from paper_2407_20143_b200 import api

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
NEAR = 1e-5


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, seed, dtype=F32):
    return torch.randn(shape, generator=_gen(seed), device="cuda").to(dtype)


def _weights(z, t, probabilities):
    z = z.double()
    if probabilities:
        return z
    if t == 0:
        w = torch.zeros_like(z)
        w[int((z == z.max()).nonzero()[0, 0])] = 1.0
        return w
    e = ((z - z.max()) / t).exp()
    return e / e.sum()


def verify64(target, drafts, uniform, draft=None, temperature=None, probabilities=False):
    """(tokens, accepted, whether all drafts' comparisons are clear, the line and place of the next token), from CPU tensors."""
    b, rows, v = target.shape
    k = rows - 1
    tokens, accepted, sure, lines = [], [], [], []
    for i in range(b):
        t = 1.0 if temperature is None else float(temperature[i])
        n = 0
        while n < k and drafts[i, n] >= 0:
            n += 1
        out, ok, used = [], True, None
        for j in range(n):
            x, u = int(drafts[i, j]), float(uniform[i, j])
            p = _weights(target[i, j], t, probabilities)
            q = torch.zeros(v, dtype=torch.float64)
            if draft is not None:
                q = _weights(draft[i, j], t, probabilities)
            elif x < v:
                q[x] = 1.0
            px, qx = (float(p[x]), float(q[x])) if x < v else (0.0, 0.0)
            if t != 0:
                ok &= abs(u * qx - px) > NEAR * (u * qx + px) or px == 0 or x >= v
            if not (x < v and u * qx < px):
                used = (p - q).clamp(min=0)
                if float(used.sum()) == 0:
                    used = p
                break
            out.append(x)
        if used is None:
            used = _weights(target[i, n], t, probabilities)
        line = used.cumsum(0)
        place = float(uniform[i, k]) * float(line[-1])
        at = min(int(torch.searchsorted(line, torch.tensor(place, dtype=torch.float64), right=True)), int(used.nonzero()[-1, 0]))
        lines.append((line, place))
        tokens.append(out + [at] + [-1] * (k - len(out)))
        accepted.append(len(out))
        sure.append(ok)
    return torch.tensor(tokens), torch.tensor(accepted, dtype=torch.int32), torch.tensor(sure), lines


def assert_next(token, want, line, place):
    """The next token lies where it was drawn, and is the definition's unless the place is near an end of its stretch."""
    first, end = (float(line[token - 1]) if token else 0.0), float(line[token])
    assert end > first and first - NEAR <= place <= end + NEAR, (token, want, first, place, end)
    first, end = (float(line[want - 1]) if want else -1.0), float(line[want])
    assert token == want or not (place - first > NEAR and end - place > NEAR)


def assert_verified(target, drafts, uniform, least=0.9, **more):
    tokens, accepted = bcp.bcp_verify_drafts(target, drafts, uniform, **more)
    host = {k: x.cpu() if isinstance(x, torch.Tensor) else x for k, x in more.items()}
    want, many, sure, lines = verify64(target.cpu(), drafts.cpu(), uniform.cpu(), **host)
    assert float(sure.float().mean()) >= least
    assert torch.equal(accepted.cpu()[sure], many[sure])
    got, greedy = tokens.cpu(), host.get("temperature")
    for i in sure.nonzero()[:, 0].tolist():
        n = int(many[i])
        assert torch.equal(got[i, :n], want[i, :n]) and bool((got[i, n + 1:] == -1).all())
        if greedy is not None and float(greedy[i]) == 0:
            assert int(got[i, n]) == int(want[i, n])
        else:
            assert_next(int(got[i, n]), int(want[i, n]), *lines[i])
    return tokens, accepted


def _batch(b, k, v, seed, dtype=F32, near=0.5, certain=False, spread=2.0):
    """Logits, drafts mostly drawn from the drafts' logits, random numbers."""
    z = spread * _randn((b, k + 1, v), seed)
    q = z[:, :k] + near * _randn((b, k, v), seed + 1)
    noise = -torch.log(-torch.log(torch.rand((b, k, v), generator=_gen(seed + 2), device="cuda").clamp(1e-7, 1 - 1e-6)))
    drafts = (q + noise).argmax(-1) if k else torch.zeros((b, 0), dtype=torch.int64, device="cuda")
    return z.to(dtype), drafts, torch.rand((b, k + 1), generator=_gen(seed + 3), device="cuda"), None if certain else q.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("certain", [False, True])
@pytest.mark.parametrize("b,k,v", [(1, 4, 1000), (64, 3, 251), (7, 1, 50257), (3, 8, 32768), (2, 64, 300), (700, 2, 17), (40, 5, 2), (5, 2, 1),
                                   (1, 2, 128256), (20, 4, 9001)])
def test_drafts(cuda_device, dtype, certain, b, k, v):
    z, drafts, u, q = _batch(b, k, v, 1, dtype, certain=certain)
    assert_verified(z, drafts, u, draft=q)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("b,v", [(1, 1), (1, 5), (300, 1000), (33, 50304), (3, 200000), (1, 1 << 22)])
def test_sampling_without_drafts(cuda_device, dtype, b, v):
    z, drafts, u, _ = _batch(b, 0, v, 5, dtype)
    tokens, accepted = assert_verified(z, drafts, u)
    assert tokens.shape == (b, 1) and not accepted.any()


def test_temperatures_and_greedy(cuda_device):
    z, drafts, u, q = _batch(60, 4, 5003, 9, BF16)
    t = torch.tensor([0.0, 0.25, 0.9, 1.0, 1.7, 0.0], device="cuda").repeat(10)
    best = z.float().argmax(-1)
    drafts[:30] = torch.where(torch.rand((30, 4), generator=_gen(3), device="cuda") < 0.7, best[:30, :4], drafts[:30])
    z[5, 1] = z[5, 1].float().clamp(max=3.0).to(BF16)  # many equal largest: the lowest index counts
    drafts[5, 1] = int((z[5, 1] == z[5, 1].max()).nonzero()[0, 0])
    tokens, accepted = assert_verified(z, drafts, u, draft=q, temperature=t)
    assert int(accepted[::6].sum()) > 5
    assert_verified(z, drafts, u, temperature=t)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("certain", [False, True])
def test_probabilities_of_a_filter(cuda_device, dtype, certain):
    z, drafts, u, q = _batch(50, 5, 4001, 13)

    def cut(x):
        top, at = x.topk(20, -1)
        return torch.zeros_like(x).scatter_(-1, at, torch.softmax(top, -1)).to(dtype)

    assert_verified(cut(z), drafts, u, draft=None if certain else cut(q), probabilities=True)
    # weights need not add up to 1: an even row of threes
    tokens, _ = bcp.bcp_verify_drafts(torch.full((1, 1, 1000), 3.0, dtype=dtype, device="cuda"), drafts[:1, :0], torch.tensor([[0.3337]], device="cuda"),
                                      probabilities=True)
    assert int(tokens) == 333


def test_drafts_that_end_early_or_lie_past_the_vocabulary(cuda_device):
    z, drafts, u, q = _batch(40, 6, 700, 17, BF16, near=0.1)
    ends = torch.arange(40, device="cuda") % 7
    drafts = torch.where(torch.arange(6, device="cuda") < ends[:, None], drafts, -1)
    drafts[6, 3:] = torch.tensor([-5, 4, 4], device="cuda")  # what stands behind a negative one does not count
    drafts[13, 2] = 700
    drafts[20, 0] = 1 << 40
    q[0] = math.nan  # rows of drafts that are not there are not looked at
    z[0, 1:] = math.nan
    for draft in (q, None):
        _, accepted = assert_verified(z.nan_to_num(0.0) if draft is None else z, drafts, u, draft=draft)
        assert int(accepted[0]) == 0 and int(accepted[6]) <= 3 and int(accepted[13]) <= 2 and int(accepted[20]) == 0


@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 0), (5, 1), (24, 7), (8, 8)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_alignments(cuda_device, pad, shift, dtype):
    b, k, v = 6, 3, 1003
    z, drafts, u, q = _batch(b, k, v, 21, dtype)
    wide = torch.full((k + 1, b, v + pad + shift), math.nan, dtype=dtype, device="cuda")
    other = torch.full((b, 2 * k, v + 2 * pad + shift), math.nan, dtype=dtype, device="cuda")
    zs, qs = wide[:, :, shift:shift + v].transpose(0, 1), other[:, ::2, pad:pad + v]
    zs.copy_(z), qs.copy_(q)
    want = bcp.bcp_verify_drafts(z, drafts, u, draft=q)
    got = bcp.bcp_verify_drafts(zs, drafts, u, draft=qs)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert_verified(zs, drafts, u, draft=qs)
    # one row for all sequences and drafts
    assert_verified(z[:1, :1].expand(b, k + 1, v), drafts, u)


def test_masked_and_unusable_rows(cuda_device):
    inf = math.inf
    z, drafts, u, q = _batch(8, 1, 600, 25)
    z[0, :, 100:] = -inf                      # a mask; the draft lies outside
    drafts[0] = 300
    z[1, 0] = -inf                            # nothing is allowed
    z[2, 0, 77] = math.nan
    z[3, 0, 78] = inf
    q[4] = -inf                               # a draft's row without weight says no
    q[5, 0, 3] = math.nan
    z[6, 1], drafts[6], u[6, 0] = -inf, z[6, 0].argmax(), 0.0  # accepted, but nothing behind it
    z[7] = torch.finfo(F32).min               # the type's lowest value throughout: even
    q[7] = 0.0
    tokens, accepted = bcp.bcp_verify_drafts(z, drafts, u, draft=q)
    assert accepted.tolist()[:6] == [0] * 6 and int(accepted[6]) == 1
    assert tokens[1:4, 0].tolist() == [-1, -1, -1] and int(tokens[6, 1]) == -1 and 0 <= int(tokens[0, 0]) < 100
    for i in (0, 4, 5, 7):
        p, t = z[i].cpu(), u[i:i + 1].cpu()
        other = q[i:i + 1].cpu() if i in (0, 7) else torch.full((1, 1, 600), 0.0)
        other[0, 0] = p[0] if i in (4, 5) else other[0, 0]  # nothing is left of p - q: p itself is drawn from
        x = drafts[i:i + 1].cpu()
        t[0, 0] = 1.0 if i in (4, 5) else t[0, 0]
        want, many, sure, lines = verify64(p[None], x, t, draft=other)
        n = int(many[0])  # an even row against an even row is accepted
        assert (sure[0] or i in (4, 5)) and int(accepted[i]) == n == int(i == 7) and int(tokens[i, 1 - n]) == (int(x) if n else -1)
        assert_next(int(tokens[i, n]), int(want[0, n]), *lines[0])
    greedy, many = bcp.bcp_verify_drafts(z, drafts, u, draft=q, temperature=torch.zeros(8, device="cuda"))
    assert int(greedy[1, 0]) == -1 and int(greedy[3, 0]) == 78 and int(greedy[7, 0]) == (0 if int(drafts[7]) else int(drafts[7]))


def test_edges_of_the_random_numbers(cuda_device):
    p = torch.tensor([0.0, 0.25, 0.0, 0.5, 0.25, 0.0], device="cuda").view(1, 1, 6)
    below = 1.0 - 2.0 ** -24
    for u, want in ((0.0, 1), (0.2499999, 1), (0.25, 3), (0.7499999, 3), (0.75, 4), (below, 4)):
        tokens, _ = bcp.bcp_verify_drafts(p, torch.zeros((1, 0), dtype=torch.int64, device="cuda"), torch.tensor([[u]], device="cuda"), probabilities=True)
        assert int(tokens) == want
    # u q < p is strict: u = 0 accepts what p allows at all
    two = p.expand(1, 2, 6)
    for x, u, ok in ((0, 0.0, 0), (1, 0.0, 1), (1, 0.25, 0), (1, 0.2499999, 1), (3, 0.5, 0)):
        _, accepted = bcp.bcp_verify_drafts(two, torch.tensor([[x]], device="cuda"), torch.tensor([[u, 0.5]], device="cuda"), probabilities=True)
        assert int(accepted) == ok


def test_tokens_are_distributed_as_the_target(cuda_device):
    # 2^17 sequences of one draft over 5 tokens: each frequency within six standard deviations of p
    n, p, q = 1 << 17, torch.tensor([0.1, 0.45, 0.05, 0.3, 0.1]), torch.tensor([0.3, 0.1, 0.3, 0.3, 0.0])
    drafts = torch.multinomial(q.cuda(), n, replacement=True, generator=_gen(1))[:, None]
    u = torch.rand((n, 2), generator=_gen(2), device="cuda")
    target = torch.stack([p, torch.tensor([0.2] * 5)]).cuda()[None].expand(n, 2, 5)
    tokens, _ = bcp.bcp_verify_drafts(target, drafts, u, draft=q.cuda()[None, None].expand(n, 1, 5), probabilities=True)
    seen = torch.bincount(tokens[:, 0], minlength=5).double().cpu() / n
    assert bool(((seen - p).abs() <= 6 * (p * (1 - p) / n).sqrt()).all())


def test_streams_graphs_and_outputs(cuda_device):
    z, drafts, u, q = _batch(9, 3, 2000, 29, BF16)
    out, accepted = torch.empty((9, 4), dtype=torch.int64, device="cuda"), torch.empty(9, dtype=torch.int32, device="cuda")
    version = out._version
    got = bcp.bcp_verify_drafts(z, drafts, u, draft=q, out=out, accepted=accepted)
    assert got[0] is out and got[1] is accepted and out._version > version
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bcp.bcp_verify_drafts(z, drafts, u, draft=q, out=out, accepted=accepted)
    z2, drafts2, u2, q2 = _batch(9, 3, 2000, 33, BF16)
    for x, y in ((z, z2), (drafts, drafts2), (u, u2), (q, q2)):
        x.copy_(y)
    graph.replay()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    tokens, many = bcp.bcp_verify_drafts(z2, drafts2, u2, draft=q2, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(tokens, out) and torch.equal(many, accepted)
    none = bcp.bcp_verify_drafts(z[:0], drafts[:0], u[:0])
    assert none[0].shape == (0, 4) and none[1].shape == (0,)


@pytest.mark.parametrize("b,v", [(1, 40001), (5, 128256), (70, 33000)])
def test_clusters_of_every_size_in_graphs_and_on_two_streams(cuda_device, b, v):
    # 16, 8 or fewer CTAs a sequence; two captured calls without anything between them, two streams at once
    z, drafts, u, q = _batch(b, 3, v, 41, BF16)
    want = bcp.bcp_verify_drafts(z, drafts, u, draft=q)
    out, torch_graph = [], torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(torch_graph):
        out = [bcp.bcp_verify_drafts(z, drafts, u, draft=q) for _ in range(2)]
    torch_graph.replay()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    out += [bcp.bcp_verify_drafts(z, drafts, u, draft=q, stream=streams[i % 2]) for i in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[0]) and torch.equal(y, want[1]) for x, y in out)


def test_refusals(cuda_device):
    z, drafts, u, q = _batch(3, 2, 50, 37)
    bcp.bcp_verify_drafts(z, drafts, u, draft=q)
    t = torch.ones(3, device="cuda")
    calls = [dict(target=z[0]), dict(target=z.double()), dict(target=z.cpu()), dict(target=z.transpose(1, 2)), dict(draft=q.bfloat16()), dict(draft=q[:, :1]),
             dict(draft=q[..., :49]), dict(drafts=drafts.int()), dict(drafts=drafts[:, :1]), dict(drafts=drafts.T.contiguous().T), dict(uniform=u[:, :2]),
             dict(uniform=u.double()), dict(temperature=t.double()), dict(temperature=t[:2]), dict(temperature=t, probabilities=True),
             dict(out=torch.empty((3, 3), device="cuda")), dict(accepted=torch.empty(3, dtype=torch.int64, device="cuda")), dict(target=None),
             dict(target=z.clone().requires_grad_())]
    for c in calls:
        a = {"target": z, "drafts": drafts, "uniform": u, "draft": q, **c}
        with pytest.raises(bcp.BcpError) as e:
            bcp.bcp_verify_drafts(**a)
        assert e.value.code in (api.ERR_INVALID, api.ERR_MISMATCH)
    many = torch.zeros((1, 66, 4), device="cuda")
    with pytest.raises(bcp.BcpError):
        bcp.bcp_verify_drafts(many, torch.zeros((1, 65), dtype=torch.int64, device="cuda"), torch.zeros((1, 66), device="cuda"))
