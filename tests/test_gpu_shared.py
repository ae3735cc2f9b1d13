"""Attention over shared prefixes against the definition in 64 bits: every sequence attends over its group's prefix and its own tokens together.

Tolerances.  A score is a sum of head_dim exact products in binary32 in an order that the matrix unit chooses, then scaled (d / 2 + 4 roundings bound both);
exp2 adds 2^-21.  A weight is rounded to binary16 (2^-11; own tokens over 8-bit caches too) or to two bfloat16 numbers (2^-16), sums of n tokens carry at most
n binary32 roundings, and weights below 2^-30 of the largest may vanish; the result is rounded once, by half a step."""
import math

import pytest
import torch

import paper_2407_20143_b200 as bcp
from paper_2407_20143_b200 import api

pytestmark = pytest.mark.gpu

BF16, F16, F32, E4M3, I8 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn, torch.int8
U = {t: torch.finfo(t).eps / 2 for t in (BF16, F16, F32)}
TINY = {BF16: 2.0 ** -133, F16: 2.0 ** -25}
F32_EPS = 2.0 ** -24


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, seed, dtype=F32):
    return torch.randn(shape, generator=_gen(seed), device="cuda").to(dtype)


def _cache(n_pages, heads, page, dim, fmt, seed=1, tokens_first=False):
    """A cache of random vectors whose rows a mask can be set to NaN in; tokens_first: heads of a token side by side."""
    scales = (None, None)
    if tokens_first:
        k, v = (torch.zeros((n_pages, page, heads, dim), dtype=fmt, device="cuda").transpose(1, 2) for _ in range(2))
        if fmt in (E4M3, I8):
            scales = tuple(torch.zeros((n_pages, heads, page), device="cuda") for _ in range(2))
        cache = bcp.KvCache(k, v, *scales)
    else:
        cache = bcp.KvCache.empty(n_pages, heads, page, dim, fmt)
    t = n_pages * page
    bcp.bcp_kv_write(cache, _randn((t, heads, dim), seed), _randn((t, heads, dim), seed + 1), torch.arange(t, device="cuda"))
    return cache


def _tables(prefix, lengths, page, seed):
    """Tables over shuffled pages; entries past an end point nowhere."""
    used = [-(-n // page) for n in prefix + lengths]
    order = torch.randperm(sum(used) + 1, generator=torch.Generator().manual_seed(seed)).tolist()

    def table(counts):
        t = torch.full((len(counts), max(1, max(counts, default=0))), -1, dtype=torch.int32)
        for i, n in enumerate(counts):
            t[i, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
        return t.cuda()

    return table(used[:len(prefix)]), table(used[len(prefix):]), sum(used) + 1


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _rows(cache, table, n):
    """Keys and values [heads, tokens, dim] in 64 bits of the first n tokens of a row of a table, without those whose page is outside the cache."""
    pos = torch.arange(min(n, table.numel() * cache.page_size), device="cuda")
    where, off = table.long()[pos // cache.page_size], pos % cache.page_size
    there = (where >= 0) & (where < cache.n_pages)
    where, off, got = where[there], off[there], []
    for pages, scales in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        flat = pages.view(torch.uint8)[where, :, off].view(pages.dtype) if pages.element_size() == 1 else pages[where, :, off]
        x = flat.float().double()
        got.append((x * scales[where, :, off].double()[..., None] if scales is not None else x).transpose(0, 1))
    return got


def assert_attended(out, lse, cache, q, prefix_table, prefix, starts, table, lengths, scale=None):
    n, hq, d = q.shape
    group, scale = hq // cache.n_heads, d ** -0.5 if scale is None else scale
    prefixes = [_rows(cache, prefix_table[g], max(0, m)) for g, m in enumerate(prefix)]
    weights = 2.0 ** -16 if cache.k.dtype == BF16 else U[F16]
    assert not out.isnan().any()
    for b in range(n):
        rows = [_rows(cache, table[b], max(0, lengths[b]))]
        of = [g for g in range(len(prefix)) if starts[g] <= b < starts[g + 1]]
        if of:
            rows.insert(0, prefixes[of[0]])
        k, v = (torch.cat([r[i] for r in rows], 1).repeat_interleave(group, 0) for i in range(2))
        tokens = k.shape[1]
        if not tokens:
            assert not out[b].any() and bool((lse[b] == -math.inf).all())
            continue
        qb = q[b].double()
        s = torch.einsum("hd,htd->ht", qb, k) * scale
        p = torch.softmax(s, -1)
        want, sums, mass = torch.einsum("ht,htd->hd", p, v), torch.logsumexp(s, -1), torch.einsum("ht,htd->hd", p, v.abs())
        size = (torch.einsum("hd,htd->ht", qb.abs(), k.abs()) * abs(scale)).amax(-1)
        score = (d / 2 + 4) * F32_EPS * size + 2.0 ** -21 + 4 * F32_EPS * sums.abs()
        tol = (weights + 4 * score[:, None] + tokens * F32_EPS) * mass * 1.01 + U[out.dtype] * want.abs() + tokens * 2.0 ** -30 * mass.amax(-1, keepdim=True) + TINY[out.dtype]
        off = (out[b].double() - want).abs()
        assert bool((off <= tol).all()), (b, float((off / tol).max()), float(off.max()))
        off = (lse[b].double() - sums).abs()
        assert bool((off <= 4 * score + tokens * F32_EPS).all()), (b, float(off.max()))


def _poison(cache, table, n):
    """NaN in what follows the first n tokens on their last page."""
    page = cache.page_size
    if n <= 0 or n % page == 0:
        return
    last = int(table[n // page])
    for x in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        if x is not None and x.element_size() > 1:
            x[last, :, n % page:] = math.nan


CASES = [  # prefix lengths, starts, own lengths, heads, group, dim, page
    ([1], [0, 1], [0], 1, 1, 64, 1),
    ([128], [0, 2], [1, 5], 1, 4, 128, 16),
    ([300], [0, 3], [0, 40, 17], 2, 4, 128, 16),
    ([257, 0, 129, 5], [1, 3, 4, 4, 7], [3, 0, 70, 9, 0, 33, 1, 80], 2, 5, 96, 13),
    ([1000], [0, 40], [7] * 40, 2, 4, 64, 24),
    ([777, 64], [0, 33, 34], [5] * 36, 1, 8, 128, 100),
    ([500], [0, 17], [20] * 17, 1, 16, 128, 64),
    ([260, 131], [0, 2, 9], [11] * 9, 2, 3, 256, 24),
    ([700], [0, 30], [2] * 30, 1, 9, 144, 7),
    ([90, 400], [0, 1, 3], [6, 0, 200], 4, 1, 16, 32),
    ([350], [0, 3], [9, 0, 1], 1, 130, 128, 64),
    ([5], [0, 70], [0] * 70, 3, 4, 80, 128),
    ([2500, 2049, 100], [0, 5, 9, 60], [13] * 60, 2, 7, 112, 16),
]


@pytest.mark.parametrize("fmt,dtype", [(BF16, BF16), (F16, F16), (E4M3, BF16), (E4M3, F16), (I8, BF16), (I8, F16)])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}p{max(c[0])}-{len(c[2])}s-{c[3]}x{c[4]}x{c[5]}-p{c[6]}")
def test_shared(cuda_device, case, fmt, dtype):
    prefix, starts, lengths, heads, group, dim, page = case
    prefix_table, table, n_pages = _tables(prefix, lengths, page, 5)
    cache = _cache(n_pages, heads, page, dim, fmt, tokens_first=page == 16)
    for t, n in [*zip(prefix_table, prefix), *zip(table, lengths)]:
        _poison(cache, t, n)
    q = _randn((len(lengths), heads * group, dim), 9, dtype) * 2
    args = (prefix_table, _int(prefix), _int(starts), table, _int(lengths))
    out, lse = bcp.bcp_kv_attend_shared(cache, q, *args)
    cache.check()
    assert_attended(out, lse, cache, q, prefix_table, prefix, starts, table, lengths)
    # the same bits again, with one workspace for several calls
    work = bcp.KvWorkspace(cache, heads * group, len(lengths), shared=True)
    for _ in range(3):
        again, lse2 = bcp.bcp_kv_attend_shared(cache, q, *args, workspace=work)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("fmt", [BF16, F16, E4M3])
@pytest.mark.parametrize("seqs,group,prefix", [(1, 1, 40000), (3, 4, 30000), (64, 4, 20000), (100, 8, 9000), (256, 1, 5001)])
def test_long_prefixes(cuda_device, fmt, seqs, group, prefix):
    lengths, starts = [3] * seqs, [0, seqs]
    prefix_table, table, n_pages = _tables([prefix], lengths, 64, 5)
    cache = _cache(n_pages, 2, 64, 128, fmt)
    q = _randn((seqs, 2 * group, 128), 9, F16 if fmt == F16 else BF16) * 2
    out, lse = bcp.bcp_kv_attend_shared(cache, q, prefix_table, _int([prefix]), _int(starts), table, _int(lengths))
    cache.check()
    assert_attended(out, lse, cache, q, prefix_table, [prefix], starts, table, lengths)


def test_many_groups(cuda_device):
    r = torch.Generator().manual_seed(3)
    prefix = torch.randint(0, 200, (700,), generator=r).tolist()
    starts = [0, *torch.randint(0, 900, (699,), generator=r).sort().values.tolist(), 900]
    lengths = torch.randint(0, 30, (900,), generator=r).tolist()
    prefix_table, table, n_pages = _tables(prefix, lengths, 16, 5)
    cache = _cache(n_pages, 1, 16, 64, BF16)
    q = _randn((900, 2, 64), 9, BF16) * 2
    out, lse = bcp.bcp_kv_attend_shared(cache, q, prefix_table, _int(prefix), _int(starts), table, _int(lengths))
    cache.check()
    assert_attended(out, lse, cache, q, prefix_table, prefix, starts, table, lengths)


@pytest.mark.parametrize("fmt", [BF16, F16, I8])
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0, 1e-30])
def test_scales_of_scores(cuda_device, fmt, scale):
    prefix_table, table, n_pages = _tables([500], [40] * 6, 16, 5)
    cache = _cache(n_pages, 2, 16, 64, fmt)
    q = _randn((6, 8, 64), 9, F16 if fmt == F16 else BF16)
    out, lse = bcp.bcp_kv_attend_shared(cache, q, prefix_table, _int([500]), _int([0, 6]), table, _int([40] * 6), scale=scale)
    assert_attended(out, lse, cache, q, prefix_table, [500], [0, 6], table, [40] * 6, scale)


@pytest.mark.parametrize("fmt", [BF16, F16, E4M3])
@pytest.mark.parametrize("rising", [False, True])
def test_peaked_and_rising_scores(cuda_device, fmt, rising):
    # scores rise by 0.1 (in all by 180) or lie 60 apart: references move at nearly every tile, or what came before counts nothing
    n, dim = 1800, 64
    prefix_table, table, n_pages = _tables([n], [30] * 40, 16, 5)
    cache = _cache(n_pages, 1, 16, dim, fmt)
    k = 0.01 * _randn((n, 1, dim), 3)
    at = torch.arange(n, device="cuda", dtype=F32)
    k[:, 0, 0] = at * 0.1 if rising else 60.0 * (at % 7 == 3)
    pages = prefix_table[0].long()
    slots = (pages[:, None] * 16 + torch.arange(16, device="cuda")).reshape(-1)[:n]
    bcp.bcp_kv_write(cache, k, _randn((n, 1, dim), 4), slots)
    q = torch.zeros((40, 4, dim), device="cuda")
    q[:, :, 0] = torch.linspace(-1, 1, 160, device="cuda").view(40, 4)
    q = q.to(F16 if fmt == F16 else BF16)
    out, lse = bcp.bcp_kv_attend_shared(cache, q, prefix_table, _int([n]), _int([0, 40]), table, _int([30] * 40), scale=1.0)
    assert_attended(out, lse, cache, q, prefix_table, [n], [0, 40], table, [30] * 40, 1.0)


@pytest.mark.parametrize("fmt", [E4M3, I8])
@pytest.mark.parametrize("least,most", [(2.0 ** -40, 2.0 ** 40), (2.0 ** -80, 2.0 ** -70), (1.0, 2.0 ** 100), (2.0 ** -96, 2.0 ** -90)])
def test_scales_of_values_far_apart(cuda_device, fmt, least, most):
    n = 900
    prefix_table, table, n_pages = _tables([n], [10] * 12, 16, 5)
    cache = _cache(n_pages, 2, 16, 64, fmt)
    span = torch.rand(cache.v_scale.shape, generator=_gen(7), device="cuda", dtype=torch.float64)
    cache.v_scale.copy_(least * (most / least) ** span)
    q = _randn((12, 8, 64), 9, BF16)
    out, lse = bcp.bcp_kv_attend_shared(cache, q, prefix_table, _int([n]), _int([0, 12]), table, _int([10] * 12))
    assert_attended(out, lse, cache, q, prefix_table, [n], [0, 12], table, [10] * 12)


@pytest.mark.parametrize("fmt", [BF16, F16, E4M3])
def test_values_that_are_not_finite(cuda_device, fmt):
    prefix_table, table, n_pages = _tables([200], [5] * 4, 16, 5)
    cache = _cache(n_pages, 2, 16, 64, fmt)
    page, off = int(prefix_table[0, 3]), 7
    if fmt == E4M3:
        cache.v_scale[page, 1, off] = math.nan
    else:
        cache.v[page, 1, off, 5] = math.nan
        cache.v[page, 1, off, 6] = math.inf
    q = _randn((4, 8, 64), 9, F16 if fmt == F16 else BF16)
    out, lse = bcp.bcp_kv_attend_shared(cache, q, prefix_table, _int([200]), _int([0, 3]), table, _int([5] * 4))
    hit = torch.zeros_like(out, dtype=torch.bool)
    if fmt == E4M3:
        hit[:3, 4:] = True
    else:
        hit[:3, 4:, 5:7] = True
        assert bool((out[:3, 4:, 6] == math.inf).all()) and bool(out[:3, 4:, 5].isnan().all())
    assert bool(out[~hit].isfinite().all()) and not out[hit].isfinite().any() and bool(lse.isfinite().all())


def test_bad_pages_lengths_and_starts(cuda_device):
    prefix, lengths, starts = [100, 40], [20, 3, 0, 9], [0, 2, 4]
    prefix_table, table, n_pages = _tables(prefix, lengths, 16, 5)
    cache = _cache(n_pages, 2, 16, 64, BF16)
    q = _randn((4, 4, 64), 9, BF16)
    # pages outside the cache: their tokens are left out
    bad = prefix_table.clone()
    bad[0, 2], bad[0, 4], bad[1, 0] = n_pages, -1, 1 << 30
    out, lse = bcp.bcp_kv_attend_shared(cache, q, bad, _int(prefix), _int(starts), table, _int(lengths))
    with pytest.raises(bcp.BcpError) as e:
        cache.check()
    assert e.value.code == api.ERR_BOUNDS and "page" in str(e.value)
    assert_attended(out, lse, cache, q, bad, prefix, starts, table, lengths)
    # a prefix of no tokens at all, all pages missing
    nowhere = torch.full_like(bad, -1)
    out, lse = bcp.bcp_kv_attend_shared(cache, q, nowhere, _int(prefix), _int(starts), table, _int(lengths))
    with pytest.raises(bcp.BcpError):
        cache.check()
    assert_attended(out, lse, cache, q, nowhere, prefix, starts, table, lengths)
    # lengths past the table count as the table's, negative ones as none
    for given, as_if in (([1 << 30, 40], [112, 40]), ([-5, 40], [0, 40])):
        full = torch.where(prefix_table < 0, 0, prefix_table)
        out, lse = bcp.bcp_kv_attend_shared(cache, q, full, _int(given), _int(starts), table, _int(lengths))
        if given[0] > 0:
            with pytest.raises(bcp.BcpError) as e:
                cache.check()
            assert "length" in str(e.value)
        else:
            cache.check()
        assert_attended(out, lse, cache, q, full, as_if, starts, table, lengths)
    # starts outside the sequences are cut off; a group that ends before it starts has none
    for given, as_if in (([-3, 2, 9], [0, 2, 4]), ([1, 1, 3], [1, 1, 3]), ([4, 4, 4], [4, 4, 4])):
        out, lse = bcp.bcp_kv_attend_shared(cache, q, prefix_table, _int(prefix), _int(given), table, _int(lengths))
        if given[0] < 0:
            with pytest.raises(bcp.BcpError):
                cache.check()
        else:
            cache.check()
        assert_attended(out, lse, cache, q, prefix_table, prefix, as_if, table, lengths)
    bcp.bcp_kv_attend_shared(cache, q, prefix_table, _int(prefix), _int([3, 1, 2]), table, _int(lengths))
    with pytest.raises(bcp.BcpError):
        cache.check()


def test_starts_that_claim_every_sequence_again_and_again(cuda_device):
    # 300,000 prefixes of 16 tiles, half of which claim all of 65,536 sequences (1024 tiles of rows): 2.4e9 steps, more than the kernel counts; no prefix is used and
    # the status says so
    cache = _cache(130, 1, 16, 64, BF16)
    n, groups = 65536, 300000
    starts = torch.tensor([0, n] * (groups // 2) + [0], dtype=torch.int32, device="cuda")
    prefix_table = torch.arange(125, dtype=torch.int32, device="cuda").expand(groups, -1).contiguous()
    q, table = _randn((n, 4, 64), 9, BF16), torch.full((n, 1), 127, dtype=torch.int32, device="cuda")
    out, _ = bcp.bcp_kv_attend_shared(cache, q, prefix_table, _int([2000] * groups), starts, table, _int([9] * n))
    with pytest.raises(bcp.BcpError) as e:
        cache.check()
    assert "length" in str(e.value)
    assert_attended(out[:3], bcp.bcp_kv_attend(cache, q[:3], table[:3], _int([9] * 3))[1], cache, q[:3], prefix_table[:0], [], [], table[:3], [9] * 3)


def test_one_workspace_for_calls_of_different_shapes(cuda_device):
    cache = _cache(60, 2, 16, 128, E4M3)
    work = bcp.KvWorkspace(cache, 8, 50, shared=True)
    r = torch.Generator().manual_seed(2)
    for seqs, prefix in ((50, [300, 77]), (3, [500]), (7, [0, 0, 0]), (50, [16]), (1, [640]), (50, [300, 77])):
        starts = [0, *torch.randint(0, seqs + 1, (len(prefix) - 1,), generator=r).sort().values.tolist(), seqs]
        prefix_table = torch.randint(0, 60, (len(prefix), 40), generator=r, dtype=torch.int32).cuda()
        table = torch.randint(0, 60, (seqs, 3), generator=r, dtype=torch.int32).cuda()
        lengths = torch.randint(0, 49, (seqs,), generator=r).tolist()
        q = _randn((seqs, 8, 128), 9, BF16)
        out, lse = bcp.bcp_kv_attend_shared(cache, q, prefix_table, _int(prefix), _int(starts), table, _int(lengths), workspace=work)
        assert_attended(out, lse, cache, q, prefix_table, prefix, starts, table, lengths)
        plain, lse1 = bcp.bcp_kv_attend(cache, q, table, _int(lengths), workspace=work)  # the plain call between
        fresh, lse2 = bcp.bcp_kv_attend(cache, q, table, _int(lengths))
        assert torch.equal(plain, fresh) and torch.equal(lse1, lse2)


def test_without_prefixes_it_is_the_plain_attention(cuda_device):
    _, table, n_pages = _tables([], [20, 0, 300], 16, 5)
    cache = _cache(n_pages, 2, 16, 64, BF16)
    q, lengths = _randn((3, 4, 64), 9, BF16), _int([20, 0, 300])
    want = bcp.bcp_kv_attend(cache, q, table, lengths)
    none = torch.zeros((0, 0), dtype=torch.int32, device="cuda")
    got = bcp.bcp_kv_attend_shared(cache, q, none, _int([]), _int([0]), table, lengths)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    empty = bcp.bcp_kv_attend_shared(cache, q[:0], none, _int([]), _int([0]), table[:0], lengths[:0])
    assert empty[0].shape == (0, 4, 64)


def test_strided_queries_and_outputs(cuda_device):
    prefix_table, table, n_pages = _tables([150], [9] * 5, 16, 5)
    cache = _cache(n_pages, 2, 16, 64, BF16)
    wide = _randn((5, 3 * 8 * 64 + 4), 9, BF16)
    q = wide[:, 4:4 + 8 * 64].view(5, 8, 64)
    holder = torch.full((8, 5, 128), 7.0, dtype=BF16, device="cuda")
    out = holder[:, :, 64:].transpose(0, 1)
    got, lse = bcp.bcp_kv_attend_shared(cache, q, prefix_table, _int([150]), _int([0, 5]), table, _int([9] * 5), out=out)
    assert got is out and bool((holder[:, :, :64] == 7).all())
    assert_attended(out, lse, cache, q, prefix_table, [150], [0, 5], table, [9] * 5)


def test_streams_and_graphs(cuda_device):
    prefix_table, table, n_pages = _tables([700], [30] * 20, 16, 5)
    cache = _cache(n_pages, 2, 16, 128, BF16)
    q, args = _randn((20, 8, 128), 9, BF16), (prefix_table, _int([700]), _int([0, 20]), table, _int([30] * 20))
    out, lse = torch.empty_like(q), torch.empty((20, 8), device="cuda")
    work = bcp.KvWorkspace(cache, 8, 20, shared=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(2):
            bcp.bcp_kv_attend_shared(cache, q, *args, out=out, lse=lse, workspace=work)
    for seed, n, seqs in ((10, 700, 20), (11, 333, 13), (12, 0, 5)):  # what stands on the device counts, not what was captured
        q.copy_(_randn((20, 8, 128), seed, BF16)), args[1].fill_(n), args[2][1:].fill_(seqs)
        graph.replay()
        assert_attended(out, lse, cache, q, prefix_table, [n], [0, seqs], table, [30] * 20)
    # two streams with a workspace each
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for i in range(6):
        got.append(bcp.bcp_kv_attend_shared(cache, q, *args, stream=streams[i % 2]))
    torch.cuda.synchronize()
    assert all(torch.equal(x, out) and torch.equal(y, lse) for x, y in got)


@pytest.mark.parametrize("page", [64, 7])
def test_offsets_past_32_bits(cuda_device, page):
    # the last pages of a cache whose elements lie beyond 2^32; boxes and copies
    n_pages = (1 << 32) // (page * 128) + 40
    k, v = (torch.zeros((n_pages, 1, page, 128), dtype=I8, device="cuda") for _ in range(2))
    cache = bcp.KvCache(k, v, *(torch.zeros((n_pages, 1, page), device="cuda") for _ in range(2)))
    last = torch.arange(n_pages - 40, n_pages, device="cuda")
    slots = (last[:, None] * page + torch.arange(page, device="cuda")).flatten()
    bcp.bcp_kv_write(cache, _randn((len(slots), 1, 128), 1), _randn((len(slots), 1, 128), 2), slots)
    table = last[torch.randperm(40, generator=torch.Generator().manual_seed(1)).cuda()].int()
    prefix_table, own, lengths = table[None, :30], table[30:].view(5, 2), [page + 3] * 5
    q = _randn((5, 4, 128), 9, BF16)
    out, lse = bcp.bcp_kv_attend_shared(cache, q, prefix_table, _int([30 * page - 5]), _int([0, 5]), own, _int(lengths))
    cache.check()
    assert_attended(out, lse, cache, q, prefix_table, [30 * page - 5], [0, 5], own, lengths)


def test_small_work_between_other_kernels(cuda_device):
    # queries, lengths and pages are written by kernels right before, outputs read right behind, without anything waiting between
    prefix_table, table, n_pages = _tables([300], [30] * 9, 16, 5)
    cache = _cache(n_pages, 2, 16, 128, BF16)
    work, got = bcp.KvWorkspace(cache, 8, 9, shared=True), []
    lengths, prefix = _int([0] * 9), _int([0])
    for i in range(20):
        q = _randn((9, 8, 128), 100 + i, BF16)
        lengths.fill_(1 + i), prefix.fill_(15 * i)
        out, lse = bcp.bcp_kv_attend_shared(cache, q, prefix_table, prefix, _int([0, 9]), table, lengths, workspace=work)
        got.append((q, out * 1, lse * 1))
        out.zero_()
    for i, (q, out, lse) in enumerate(got):
        assert_attended(out, lse, cache, q, prefix_table, [15 * i], [0, 9], table, [1 + i] * 9)


def test_refusals(cuda_device):
    prefix_table, table, n_pages = _tables([150], [9] * 5, 16, 5)
    cache = _cache(n_pages, 2, 16, 64, BF16)
    q = _randn((5, 8, 64), 9, BF16)
    good = dict(cache=cache, q=q, prefix_table=prefix_table, prefix_lengths=_int([150]), starts=_int([0, 5]), block_table=table, lengths=_int([9] * 5))
    bcp.bcp_kv_attend_shared(**good)
    small = bcp.KvWorkspace(cache, 8, 5)
    for c in (dict(q=q.half()), dict(q=q.float()), dict(q=q[:4]), dict(q=q[:, :3]), dict(prefix_table=prefix_table.long()), dict(prefix_table=prefix_table[0]),
              dict(prefix_lengths=_int([150, 1])), dict(starts=_int([0])), dict(starts=torch.tensor([0, 5], device="cuda")), dict(block_table=table[:4]),
              dict(lengths=_int([9] * 4)), dict(scale=math.inf), dict(workspace=small), dict(q=q.clone().requires_grad_()),
              dict(out=torch.empty((5, 8, 64), device="cuda")), dict(prefix_table=prefix_table.cpu()), dict(lse=torch.empty((5, 7), device="cuda"))):
        with pytest.raises(bcp.BcpError):
            bcp.bcp_kv_attend_shared(**{**good, **c})
    cache.check()
