"""Rotary positions, the paged key-value cache and the attention over it, against plain forms in 64 bits.

Tolerances are bounds of the arithmetic the header describes: U[t] is half a unit in the last place of a
type, relative; a value that is computed in binary32 and rounded once is within U[t] of itself plus a few
binary32 roundings of the terms it is summed from.
"""
import math

import numpy as np
import pytest
import torch

import paper_2407_20143_b200 as bcp
from paper_2407_20143_b200 import api

pytestmark = pytest.mark.gpu

BF16, F16, F32, E4M3, I8 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn, torch.int8
U = {t: torch.finfo(t).eps / 2 for t in (BF16, F16, F32)}  # 2^-8, 2^-11, 2^-24
TINY = {BF16: 2.0 ** -133, F16: 2.0 ** -25, F32: 2.0 ** -149}  # half the smallest subnormal
QMAX = {E4M3: 448.0, I8: 127.0}
F32_EPS = 2.0 ** -24


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, seed, dtype=F32):
    return torch.randn(shape, generator=_gen(seed), device="cuda").to(dtype)


# ------------------------------------------------------------------ rotary positions
def rotate64(x, table, positions, layout, transposed=False):
    """x [tokens, heads, dim] on the CPU in 64 bits; rows of positions outside the table are zero."""
    x, table, positions = x.double().cpu(), table.double().cpu(), positions.cpu()
    n = table.shape[2]
    ok = (positions >= 0) & (positions < table.shape[0])
    p = positions.clamp(0, table.shape[0] - 1)
    c, s = table[p, 0][:, None], table[p, 1][:, None] * (-1.0 if transposed else 1.0)
    y = x.clone()
    i, j = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    size = x.abs()
    size[..., i] = size[..., j] = x[..., i].abs() + x[..., j].abs()
    return y * ok[:, None, None], size * ok[:, None, None]


def assert_rotated(got, x, table, positions, layout, transposed=False):
    want, size = rotate64(x, table, positions, layout, transposed)
    factor = max(1.0, float(table.abs().max()))
    tol = U[got.dtype] * want.abs() * 1.0001 + 4 * F32_EPS * factor * size + TINY[got.dtype]
    bad = (got.double().cpu() - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), float((got.double().cpu() - want).abs().max()))


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("tokens,hq,hk,dim,rot", [(1, 1, 1, 64, 64), (5, 4, 2, 128, 128), (67, 7, 1, 96, 32), (33, 3, 3, 256, 256),
                                                  (9, 2, 1, 80, 20), (11, 5, 2, 30, 6), (4, 6, 3, 2, 2), (3, 32, 8, 128, 126)])
def test_rope(cuda_device, layout, dtype, tokens, hq, hk, dim, rot):
    table = bcp.RopeTable.build(bcp.rope_frequencies(rot), 300, layout=layout)
    positions = torch.randint(0, 300, (tokens,), generator=_gen(1), device="cuda")
    q, k = _randn((tokens, hq, dim), 2, dtype), _randn((tokens, hk, dim), 3, dtype)
    yq, yk = bcp.bcp_rope((q, k), table, positions)
    assert_rotated(yq, q, table.table, positions, layout)
    assert_rotated(yk, k, table.table, positions, layout)
    gq = bcp.bcp_rope_backward(q, table, positions)  # one tensor alone
    assert_rotated(gq, q, table.table, positions, layout, transposed=True)
    table.check()


@pytest.mark.parametrize("shift", [0, 1, 4])
def test_rope_strides_and_in_place(cuda_device, shift):
    # heads of a fused projection, tokens apart by more than they are long, rows off the 16-byte boundaries by `shift` elements
    t, hq, hk, dim = 21, 6, 2, 64
    table = bcp.RopeTable.build(bcp.rope_frequencies(dim), 64)
    positions = torch.randint(0, 64, (t,), generator=_gen(1), device="cuda")
    wide = _randn((t, (hq + 2 * hk) * dim + 8), 2, BF16)
    before = wide.clone()
    q = wide[:, shift:shift + hq * dim].view(t, hq, dim)
    k = wide[:, shift + hq * dim:shift + (hq + hk) * dim].view(t, hk, dim)
    q0, k0 = q.clone(), k.clone()
    turned = torch.empty((hq, t, dim), dtype=BF16, device="cuda").transpose(0, 1)  # heads outermost
    bcp.bcp_rope(q, table, positions, out=turned)
    assert_rotated(turned, q0, table.table, positions, "half")
    got = bcp.bcp_rope((q, k), table, positions, out=(q, k))
    assert got[0] is q and got[1] is k
    assert_rotated(q, q0, table.table, positions, "half")
    assert_rotated(k, k0, table.table, positions, "half")
    assert torch.equal(wide[:, shift + (hq + hk) * dim:], before[:, shift + (hq + hk) * dim:]) and torch.equal(wide[:, :shift], before[:, :shift])
    # one vector for all heads and tokens
    one = _randn((1, 1, dim), 5, BF16).expand(t, hq, dim)
    assert_rotated(bcp.bcp_rope(one, table, positions), one, table.table, positions, "half")


def test_rope_positions_out_of_the_table(cuda_device):
    table = bcp.RopeTable.build(bcp.rope_frequencies(32), 10, layout="pairs")
    x = _randn((6, 3, 48), 2)
    x[1] = math.nan  # what stands in a padding row does not matter
    positions = torch.tensor([0, -1, 9, 10, -(1 << 40), 1 << 40], device="cuda")
    y = bcp.bcp_rope(x, table, positions)
    assert_rotated(y, torch.nan_to_num(x), table.table, positions, "pairs")
    assert not y[[1, 3, 4, 5]].any()
    with pytest.raises(bcp.BcpError) as e:
        table.check()
    assert e.value.code == api.ERR_BOUNDS and "position" in str(e.value)
    table.check()  # cleared
    bcp.bcp_rope(x[:2].contiguous(), table, positions[:2])
    table.check()  # padding is no error


def test_rope_no_tokens(cuda_device):
    table = bcp.RopeTable.build(bcp.rope_frequencies(32), 10)
    y = bcp.bcp_rope(torch.empty((0, 3, 32), device="cuda"), table, torch.empty(0, dtype=torch.int64, device="cuda"))
    assert y.shape == (0, 3, 32)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_rope_gradient(cuda_device, layout):
    t, h, hk, dim, rot = 7, 3, 2, 48, 32
    table = bcp.RopeTable.build(bcp.rope_frequencies(rot, scaling="linear", factor=4.0), 50, layout=layout, attention_factor=1.3)
    positions = torch.randint(0, 50, (t,), generator=_gen(1), device="cuda")
    x, xk = _randn((t, h, dim), 2).requires_grad_(), _randn((t, hk, dim), 3).requires_grad_()
    w, wk = _randn((t, h, dim), 4), _randn((t, hk, dim), 5)
    y, yk = bcp.rope((x, xk), table, positions)
    ((y * w).sum() + (yk * wk).sum()).backward()
    assert_rotated(x.grad, w, table.table, positions, layout, transposed=True)
    assert_rotated(xk.grad, wk, table.table, positions, layout, transposed=True)
    # against differences: the map is linear, so a quotient over +-1 has no truncation error, only the
    # roundings of the two outputs (dim terms each)
    for i in (0, 100, 555, t * h * dim - 1):
        step = torch.zeros(t * h * dim, device="cuda")
        step[i] = 1.0
        step = step.view(t, h, dim)
        up, down = (bcp.bcp_rope(x.detach() + s * step, table, positions).double() for s in (1, -1))
        quotient = float(((up - down) * w.double()).sum() / 2)
        tol = 4 * F32_EPS * 2 * 1.3 * float((x.detach().abs() + 1).max()) * 2 * float(w.abs().max()) * 2
        assert abs(quotient - float(x.grad.flatten()[i])) <= tol
    # a gradient that is one number expanded
    z = x.detach().clone().requires_grad_()
    bcp.rope(z, table, positions).sum().backward()
    assert_rotated(z.grad, torch.ones_like(w), table.table, positions, layout, transposed=True)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_rope_gradient_of_a_gradient(cuda_device, layout):
    t, h, dim, rot = 7, 3, 48, 32
    table = bcp.RopeTable.build(bcp.rope_frequencies(rot), 50, layout=layout, attention_factor=1.3)
    positions = torch.randint(0, 50, (t,), generator=_gen(1), device="cuda")
    x, w = _randn((t, h, dim), 2).requires_grad_(), _randn((t, h, dim), 4)
    first = (bcp.rope(x, table, positions) ** 2 * w).sum()
    g, = torch.autograd.grad(first, x, create_graph=True)
    (first + (g ** 2).sum()).backward()
    # J = 2 R^T w R is symmetric: the gradient is J x + 2 J J x
    turn = lambda v, back=False: rotate64(v, table.table, positions, layout, back)  # noqa: E731
    w64 = w.double().cpu()
    through = lambda v: 2 * turn(w64 * turn(v)[0], True)[0]  # noqa: E731
    want = through(x.detach()) + 2 * through(through(x.detach()))
    # Every rotation rounds its terms (4 in binary32, of the sums of magnitudes that it adds), the products in between once or twice:
    # 24 roundings along the longest way, of the same chain in magnitudes.
    size = lambda v: 2 * 1.3 ** 2 * turn(w64.abs() * turn(v)[1])[1]  # noqa: E731
    s1 = size(x.detach())
    tol = 24 * F32_EPS * (s1 + 2 * size(s1))
    assert bool(((x.grad.double().cpu() - want).abs() <= tol).all())


def test_rope_long_positions_keep_their_angle(cuda_device):
    # 64-bit angles: at position 200,000 a binary32 product of position and frequency is off by up to 0.01
    f = bcp.rope_frequencies(64, base=500000.0, scaling="bands", factor=8.0, trained=8192)
    table = bcp.RopeTable.build(f, 200001)
    x = torch.zeros((1, 1, 64), device="cuda")
    x[..., :32] = 1.0
    y = bcp.bcp_rope(x, table, torch.tensor([200000], device="cuda"))[0, 0].cpu().double()
    for i, w in enumerate(f):
        assert abs(float(y[i]) - math.cos(200000 * w)) < 2e-7 and abs(float(y[32 + i]) - math.sin(200000 * w)) < 2e-7


# ------------------------------------------------------------------ cache
def _grid_e4m3():
    v = torch.arange(0, 127, dtype=torch.uint8).view(E4M3).double().numpy()  # 0 .. 448, ascending; index = bit pattern
    assert v[-1] == 448.0 and np.all(np.diff(v) > 0)
    return v


def quantise64(x, fmt):
    """(values, scales) of rows x (float32) as the header defines them; the products in binary32 as well."""
    x = x.float().cpu().numpy()
    top = np.abs(x).max(-1)
    scale = np.maximum(top / np.float32(QMAX[fmt]), np.float32(2.0 ** -96)).astype(np.float32)
    y = (x * (np.float32(1.0) / scale)[..., None]).astype(np.float32).astype(np.float64)
    if fmt == I8:
        q = np.clip(np.rint(y), -127, 127)
    else:
        grid = _grid_e4m3()
        a = np.minimum(np.abs(y), 448.0)
        hi = np.clip(np.searchsorted(grid, a), 1, 126)
        lo = hi - 1
        down, up = a - grid[lo], grid[hi] - a
        take_hi = (up < down) | ((up == down) & (hi % 2 == 0))
        q = np.copysign(np.where(take_hi, grid[hi], grid[lo]), y)
    return q, scale


def _cache(n_pages, heads, page, dim, fmt, layout="heads", fill=None):
    """A cache whose memory is poisoned, in one of three orders."""
    shape = {"heads": (n_pages, heads, page, dim), "tokens": (n_pages, page, heads, dim), "joined": (n_pages, 2, heads, page, dim)}[layout]
    if layout == "joined":
        both = torch.zeros(shape, dtype=torch.uint8 if fmt in QMAX else fmt, device="cuda")
        k, v = both[:, 0], both[:, 1]
    else:
        k, v = (torch.zeros(shape, dtype=torch.uint8 if fmt in QMAX else fmt, device="cuda") for _ in range(2))
        if layout == "tokens":
            k, v = k.transpose(1, 2), v.transpose(1, 2)
    if fmt in QMAX:
        k.fill_(0x7F), v.fill_(0x7F)  # NaN in e4m3
        k, v = k.view(fmt), v.view(fmt)
        return bcp.KvCache(k, v, *(torch.full((n_pages, heads, page), math.nan, device="cuda") for _ in range(2)))
    k.fill_(math.nan), v.fill_(math.nan)
    return bcp.KvCache(k, v)


def _some_slots(n, total, seed, skip=()):
    s = torch.randperm(total, generator=torch.Generator().manual_seed(seed))[:n].cuda()
    for i in skip:
        s[i] = -1
    return s


def _rows(pages, slots, page):
    x = pages.float() if pages.element_size() > 1 else pages.float()
    return x.transpose(1, 2).reshape(-1, pages.shape[1], pages.shape[3])[slots.cpu()] if not x.is_cuda else \
        x.transpose(1, 2).reshape(-1, pages.shape[1], pages.shape[3])[slots].cpu()


@pytest.mark.parametrize("layout", ["heads", "tokens", "joined"])
@pytest.mark.parametrize("fmt", [BF16, F16, E4M3, I8])
@pytest.mark.parametrize("tokens,heads,dim,page", [(1, 1, 16, 1), (37, 5, 128, 13), (6, 2, 256, 16), (50, 3, 80, 7), (19, 8, 64, 64)])
def test_write_then_read(cuda_device, layout, fmt, tokens, heads, dim, page):
    n_pages = -(-tokens // page) + 2
    cache = _cache(n_pages, heads, page, dim, fmt, layout)
    k0, v0 = cache.k.clone(), cache.v.clone()
    k, v = _randn((tokens, heads, dim), 1, BF16), _randn((tokens, heads, dim), 2, BF16) * 3
    if tokens > 4:
        k[2, 0] = 0  # a vector of zeros
        v[3, heads - 1, dim - 1] = 1000.0  # one element far above the others
    slots = _some_slots(tokens, n_pages * page, 3, skip=(4,) if tokens > 4 else ())
    bcp.bcp_kv_write(cache, k, v, slots)
    cache.check()
    used = slots >= 0
    for pages, scales, x in ((cache.k, cache.k_scale, k), (cache.v, cache.v_scale, v)):
        got = _rows(pages, slots[used], page)
        if fmt in QMAX:
            q, s = quantise64(x[used], fmt)
            assert np.array_equal(got.numpy(), q)
            assert np.array_equal(scales.transpose(1, 2).reshape(-1, heads)[slots[used]].cpu().numpy(), s)
        else:
            assert torch.equal(got, x[used].to(fmt).float().cpu())
    # nothing else was touched
    left = torch.ones(n_pages * page, dtype=torch.bool, device="cuda")
    left[slots[used]] = False
    for pages, was in ((cache.k, k0), (cache.v, v0)):
        a, b = (p.contiguous().view(torch.uint8).view(n_pages, heads, page, -1).transpose(1, 2).reshape(n_pages * page, -1)[left] for p in (pages, was))
        assert torch.equal(a, b)
    for dtype in (BF16, F16, F32):
        rk, rv = bcp.bcp_kv_read(cache, slots, dtype=dtype)
        for got, pages, scales in ((rk, cache.k, cache.k_scale), (rv, cache.v, cache.v_scale)):
            want = _rows(pages, slots[used], page)
            if scales is not None:
                want = want * scales.transpose(1, 2).reshape(-1, heads)[slots[used]].cpu()[..., None]
            assert torch.equal(got[used].cpu(), want.to(dtype)) and not got[~used].any()


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fmt", [F16, E4M3, I8])
@pytest.mark.parametrize("dim,rot", [(128, 128), (96, 32), (64, 12), (256, 250)])
def test_write_rotates_keys(cuda_device, layout, dtype, fmt, dim, rot):
    t, h, page = 23, 3, 8
    cache = _cache(6, h, page, dim, fmt)
    table = bcp.RopeTable.build(bcp.rope_frequencies(rot), 99, layout=layout)
    positions = torch.randint(0, 99, (t,), generator=_gen(4), device="cuda")
    positions[5] = 99
    slots = _some_slots(t, 48, 3, skip=(2,))
    k, v = _randn((t, h, dim), 1, dtype), _randn((t, h, dim), 2, dtype)
    bcp.bcp_kv_write(cache, k, v, slots, rope=table, positions=positions)
    with pytest.raises(bcp.BcpError, match="position"):
        cache.check()
    used = (slots >= 0) & (torch.arange(t, device="cuda") != 5)
    rk, rv = bcp.bcp_kv_read(cache, slots, dtype=F32)
    want, size = rotate64(k, table.table, positions, layout)
    want, size, got = want[used.cpu()], size[used.cpu()], rk[used].double().cpu()
    if fmt in QMAX:
        # half a step of the format above a value that is itself a few binary32 roundings off
        top = want.abs().amax(-1, keepdim=True)
        step = top / 127 * 0.5 if fmt == I8 else torch.maximum(want.abs() * 2.0 ** -4, top / 448 * 2.0 ** -10)
        tol = step * 1.001 + 8 * F32_EPS * (size + top)
        assert bool(((rv[used].double() - v[used].double()).abs().cpu() <= v[used].double().abs().cpu().amax(-1, keepdim=True) * (0.5 / 127 if fmt == I8 else 2.0 ** -4) * 1.001).all())
    else:
        tol = U[fmt] * want.abs() * 1.0001 + 4 * F32_EPS * size + TINY[fmt]
        assert torch.equal(rv[used], v[used].to(fmt).float())
    assert bool(((got - want).abs() <= tol).all())
    left = rk[~used & (slots >= 0)]  # the token whose position is not in the table was not written
    assert bool(left.isnan().all())


@pytest.mark.parametrize("fmt", [E4M3, I8])
def test_vectors_that_are_not_finite(cuda_device, fmt):
    cache = _cache(1, 2, 8, 32, fmt)
    k = _randn((4, 2, 32), 1)
    k[1, 0, 7], k[2, 1, 31], k[3, 0, 0] = math.nan, math.inf, 3.0e38
    slots = torch.arange(4, device="cuda")
    bcp.bcp_kv_write(cache, k, k, slots)
    rk, rv = bcp.bcp_kv_read(cache, slots, dtype=F32)
    for r in (rk, rv):
        nan = torch.zeros((4, 2), dtype=torch.bool, device="cuda")
        nan[1, 0] = nan[2, 1] = True
        assert torch.equal(r.isnan().all(-1), nan) and torch.equal(r.isnan().any(-1), nan)
        assert float(r[3, 0, 0]) == pytest.approx(3.0e38, rel=1e-6)
    # vectors near the smallest numbers: the scale stops at 2^-96
    tiny = torch.full((1, 2, 32), 2.0 ** -96 * 3, device="cuda")
    tiny[0, 1] = 1e-42
    bcp.bcp_kv_write(cache, tiny, tiny, slots[:1])
    rk, _ = bcp.bcp_kv_read(cache, slots[:1], dtype=F32)
    assert torch.equal(rk[0, 0], tiny[0, 0]) and not rk[0, 1].any()


def test_slots_out_of_the_cache(cuda_device):
    cache = _cache(3, 2, 5, 32, BF16)
    k = _randn((4, 2, 32), 1, BF16)
    slots = torch.tensor([14, 15, 1 << 40, -7], device="cuda")
    bcp.bcp_kv_write(cache, k, k, slots)
    with pytest.raises(bcp.BcpError) as e:
        cache.check()
    assert e.value.code == api.ERR_BOUNDS and "slot" in str(e.value)
    assert int((~cache.k.isnan()).sum()) == 2 * 32
    rk, rv = bcp.bcp_kv_read(cache, slots)
    assert torch.equal(rk[0], k[0]) and not rk[1:].any() and not rv[1:].any()
    with pytest.raises(bcp.BcpError, match="slot"):
        cache.check()


def test_slots_of_padding_and_of_positions_past_the_table(cuda_device):
    cache = _cache(4, 2, 5, 32, BF16)
    table = torch.tensor([[2, 0], [3, -1]], dtype=torch.int32, device="cuda")
    rows = torch.tensor([0, 0, 0, 1, 1, 0], device="cuda")
    positions = torch.tensor([0, 9, -1, 4, 5, -7], device="cuda")
    k = _randn((6, 2, 32), 1, BF16)
    slots = cache.slots(table, rows, positions)
    assert slots.tolist() == [10, 4, -1, 19, -1, -1]
    bcp.bcp_kv_write(cache, k, k, slots)
    cache.check()  # padding is no error
    assert int((~cache.k.isnan()).sum()) == 3 * 2 * 32
    rk, _ = bcp.bcp_kv_read(cache, slots)
    assert torch.equal(rk[[0, 1, 3]], k[[0, 1, 3]]) and not rk[[2, 4, 5]].any()
    past = cache.slots(table, torch.tensor([0, 2], device="cuda"), torch.tensor([10, 0], device="cuda"))
    bcp.bcp_kv_write(cache, k[:2], k[:2], past)
    with pytest.raises(bcp.BcpError, match="slot"):
        cache.check()
    assert int((~cache.k.isnan()).sum()) == 3 * 2 * 32


@pytest.mark.parametrize("shift", [0, 1])
def test_write_and_read_strided(cuda_device, shift):
    t, h, dim = 9, 5, 48
    cache = _cache(2, h, 16, dim, E4M3)
    wide = _randn((t, 3 * h * dim + 16), 1, BF16)
    k, v = wide[:, shift:shift + h * dim].view(t, h, dim), wide[:, shift + h * dim:shift + 2 * h * dim].view(t, h, dim)
    slots = torch.arange(t, device="cuda")
    bcp.bcp_kv_write(cache, k, v, slots)
    q, _ = quantise64(k, E4M3)
    assert np.array_equal(_rows(cache.k, slots, 16).numpy(), q)
    out = torch.full((t, 3 * h * dim + 16), 7.0, dtype=F16, device="cuda")
    ok, ov = out[:, shift:shift + h * dim].view(t, h, dim), out[:, shift + 2 * h * dim:shift + 3 * h * dim].view(t, h, dim)
    bcp.bcp_kv_read(cache, slots, out=(ok, ov))
    rk, rv = bcp.bcp_kv_read(cache, slots, dtype=F16)
    assert torch.equal(ok, rk) and torch.equal(ov, rv)
    assert bool((out[:, shift + h * dim:shift + 2 * h * dim] == 7).all()) and bool((out[:, shift + 3 * h * dim:] == 7).all())


# ------------------------------------------------------------------ attention
def attend64(cache, q, block_table, lengths, scale, window):
    """(out, lse, sum p |v|, largest sum |q k| scale) on the CPU in 64 bits."""
    n, hq, d = q.shape
    group, page = hq // cache.n_heads, cache.page_size
    out, lse, mass, size = torch.zeros(n, hq, d, dtype=torch.float64), torch.full((n, hq), -math.inf, dtype=torch.float64), None, None
    mass, size = torch.zeros(n, hq, d, dtype=torch.float64), torch.zeros(n, hq, dtype=torch.float64)
    values = []
    for pages, scales in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x = pages.float().double()
        values.append((x * scales.double()[..., None] if scales is not None else x).cpu())
    for b in range(n):
        length = min(max(0, int(lengths[b])), block_table.shape[1] * page)
        pos = torch.arange(max(0, length - window) if window else 0, length)
        where = block_table[b].cpu().long()[pos // page]
        there = (where >= 0) & (where < cache.n_pages)
        pos, where = pos[there], where[there]
        if not len(pos):
            continue
        k, v = (x[where, :, pos % page].repeat_interleave(group, 1) for x in values)
        qb = q[b].double().cpu()
        s = torch.einsum("hd,thd->ht", qb, k) * scale
        p = torch.softmax(s, -1)
        out[b], lse[b] = torch.einsum("ht,thd->hd", p, v), torch.logsumexp(s, -1)
        mass[b] = torch.einsum("ht,thd->hd", p, v.abs())
        size[b] = (torch.einsum("hd,thd->ht", qb.abs(), k.abs()) * abs(scale)).amax(-1)
    return out, lse, mass, size


def assert_attended(out, lse, cache, q, block_table, lengths, scale, window):
    want, sums, mass, size = attend64(cache, q, block_table, lengths, scale, window)
    # A score is a sum of head_dim exact products in binary32, whose order the matrix unit chooses, then scaled
    # (d/2 + 4 roundings bound both); exp2 adds 2^-21.  The weights are rounded to bfloat16 (16-bit bfloat16
    # caches) or binary16 (all others; at most 2^-30 of the largest is lost below), the result to its type.
    score = (q.shape[2] / 2 + 4) * F32_EPS * size + 2.0 ** -21 + 4 * F32_EPS * sums.abs().nan_to_num(0, 0, 0)
    weights = U[BF16] if cache.k.dtype == BF16 else U[F16]
    tokens = int(lengths.max()) if lengths.numel() else 0
    tol = (weights + 4 * score[..., None] + tokens * F32_EPS) * mass * 1.01 + U[out.dtype] * want.abs() + tokens * 2.0 ** -30 * mass.amax(-1, keepdim=True) + TINY[out.dtype]
    off = (out.double().cpu() - want).abs()
    assert bool((off <= tol).all()), (float((off / tol).max()), float(off.max()))
    empty = sums == -math.inf
    assert torch.equal(lse.double().cpu() == -math.inf, empty) and not out.cpu()[empty].any()
    off = (lse.double().cpu() - sums)[~empty].abs()
    assert bool((off <= 4 * score[~empty] + tokens * F32_EPS).all()), float(off.max())


def _filled(n_pages, heads, page, dim, fmt, layout="heads", seed=1):
    cache = _cache(n_pages, heads, page, dim, fmt, layout)
    t = n_pages * page
    k, v = _randn((t, heads, dim), seed), _randn((t, heads, dim), seed + 1)
    bcp.bcp_kv_write(cache, k, v, torch.arange(t, device="cuda"))
    return cache


def _batch(lengths, page, seed, n_pages=None):
    """A block table over shuffled pages; entries past a sequence's end point nowhere."""
    used = [-(-n // page) for n in lengths]
    n_pages = n_pages or sum(used) + 1
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((len(lengths), max(1, max(used))), -1, dtype=torch.int32)
    for b, n in enumerate(used):
        table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    return table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), n_pages


CASES = [  # lengths, heads, group, dim, page, window, layout
    ([1], 1, 1, 64, 1, 0, "heads"),
    ([16], 1, 8, 128, 16, 0, "heads"),
    ([0, 1, 63, 64, 65, 15, 17], 2, 4, 128, 16, 0, "tokens"),
    ([600], 8, 4, 128, 16, 0, "heads"),
    ([333, 0, 5, 1000], 3, 5, 96, 13, 0, "joined"),
    ([100, 777], 2, 16, 64, 100, 0, "heads"),
    ([250, 31], 1, 24, 128, 7, 0, "tokens"),
    ([129, 500, 2], 2, 12, 256, 24, 0, "heads"),
    ([70, 4], 4, 3, 16, 32, 0, "heads"),
    ([400, 90, 0, 100, 101, 1], 2, 7, 128, 24, 100, "heads"),
    ([5000], 1, 1, 128, 64, 1, "heads"),
    ([200, 3000], 4, 9, 48, 16, 1000, "tokens"),
]


@pytest.mark.parametrize("fmt,dtype", [(BF16, BF16), (F16, F16), (E4M3, BF16), (E4M3, F16), (I8, BF16), (I8, F16)])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{max(c[0])}-{c[1]}x{c[2]}x{c[3]}-p{c[4]}-w{c[5]}-{c[6]}")
def test_attend(cuda_device, case, fmt, dtype):
    lengths, heads, group, dim, page, window, layout = case
    table, lens, n_pages = _batch(lengths, page, 5)
    cache = _filled(n_pages, heads, page, dim, fmt, layout)
    # tokens past each end hold NaN, as do the pages no sequence has
    for b, n in enumerate(lengths):
        if n % page:
            last = int(table[b, n // page])
            for x in (cache.k, cache.v):
                if x.element_size() > 1:
                    x[last, :, n % page:] = math.nan
            if cache.k_scale is not None:
                cache.k_scale[last, :, n % page:] = math.nan
                cache.v_scale[last, :, n % page:] = math.nan
    q = _randn((len(lengths), heads * group, dim), 9, dtype) * 2
    scale = dim ** -0.5
    out, lse = bcp.bcp_kv_attend(cache, q, table, lens, window=window)
    cache.check()
    assert_attended(out, lse, cache, q, table, lens, scale, window)
    # the same bits again, with one workspace for several calls
    work = bcp.KvWorkspace(cache, heads * group, len(lengths))
    for _ in range(3):
        again, lse2 = bcp.bcp_kv_attend(cache, q, table, lens, scale=scale, window=window, workspace=work)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("fmt", [BF16, E4M3])
def test_attend_long(cuda_device, fmt):
    table, lens, n_pages = _batch([40000, 3], 64, 5)
    cache = _filled(n_pages, 2, 64, 128, fmt)
    q = _randn((2, 8, 128), 9, BF16)
    out, lse = bcp.bcp_kv_attend(cache, q, table, lens)
    assert_attended(out, lse, cache, q, table, lens, 128 ** -0.5, 0)


@pytest.mark.parametrize("fmt", [F16, I8])
def test_attend_many_sequences(cuda_device, fmt):
    g = torch.Generator().manual_seed(7)
    lengths = torch.randint(0, 90, (700,), generator=g).tolist()
    table, lens, n_pages = _batch(lengths, 16, 5)
    cache = _filled(n_pages, 1, 16, 64, fmt)
    q = _randn((700, 4, 64), 9, F16)
    out, lse = bcp.bcp_kv_attend(cache, q, table, lens)
    assert_attended(out, lse, cache, q, table, lens, 64 ** -0.5, 0)


@pytest.mark.parametrize("fmt", [F16, E4M3])
def test_attend_peaked_and_rising_scores(cuda_device, fmt):
    # scores that rise along the sequence make the running reference move at every step; a peak of e^60 over the rest
    n, dim = 700, 64
    cache = _cache(n // 16 + 1, 1, 16, dim, fmt)
    k, v = _randn((n, 1, dim), 1) * 0.1, _randn((n, 1, dim), 2)
    k[:, 0, 0] = torch.linspace(-30, 30, n, device="cuda")
    bcp.bcp_kv_write(cache, k, v, torch.arange(n, device="cuda"))
    table = torch.arange(n // 16 + 1, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    q = _randn((1, 8, dim), 3, F16) * 0.1
    q[0, :, 0] = torch.tensor([8.0, -8.0, 4.0, -4.0, 2.0, 1.0, 0.0, -1.0], device="cuda")
    for scale in (1.0, -0.5, 0.0):
        out, lse = bcp.bcp_kv_attend(cache, q, table, lens, scale=scale)
        assert_attended(out, lse, cache, q, table, lens, scale, 0)


@pytest.mark.parametrize("fmt", [E4M3, I8])
def test_attend_scales_far_apart(cuda_device, fmt):
    # value vectors from 2^-40 to 2^40: the weights carry the scales' exponents, whichever token dominates
    n, dim = 100, 64
    cache = _cache(7, 1, 16, dim, fmt)
    k, v = _randn((n, 1, dim), 1), _randn((n, 1, dim), 2)
    v *= torch.pow(2.0, torch.linspace(-40, 40, n, device="cuda"))[:, None, None]
    v[50] = 0.0
    k[:, 0, 0] = torch.linspace(30, -30, n, device="cuda")  # the smallest values have the largest scores
    bcp.bcp_kv_write(cache, k, v, torch.arange(n, device="cuda"))
    cache.v_scale[50 // 16, 0, 50 % 16] = 0.0  # another program may scale a vector of zeros by zero
    table = torch.arange(7, dtype=torch.int32, device="cuda")[None]
    q = torch.zeros((1, 3, dim), dtype=BF16, device="cuda")
    q[0, 0, 0], q[0, 1, 0], q[0, 2, 0] = 1.0, -1.0, 0.25
    for length in (100, 51, 1):
        lens = torch.tensor([length], dtype=torch.int32, device="cuda")
        out, lse = bcp.bcp_kv_attend(cache, q, table, lens, scale=1.0)
        assert_attended(out, lse, cache, q, table, lens, 1.0, 0)


@pytest.mark.parametrize("fmt", [E4M3, I8])
@pytest.mark.parametrize("top", [2.0 ** 45, 2.0 ** 100, 3.0e38])
@pytest.mark.parametrize("n,zeros", [(1 + 16, [0]), (60, [5, 20, 59]), (3000, list(range(10))), (3000, list(range(2990, 3000))), (20000, [11000])])
def test_attend_vectors_of_zeros_that_dominate(cuda_device, fmt, top, n, zeros):
    # Tokens whose values are zero (scale 2^-96) have the largest scores by far, the others' values are near the largest numbers:
    # what the zeros weigh has to stay in the denominator, whichever come first and whichever part of the sequence they are in.
    dim, page = 64, 16
    cache = _cache(-(-n // page), 1, page, dim, fmt)
    k, v = _randn((n, 1, dim), 1) * 0.1, _randn((n, 1, dim), 2).clamp(-3, 3) * (top / 3)
    k[zeros, 0, 0], v[zeros] = 30.0, 0.0
    bcp.bcp_kv_write(cache, k, v, torch.arange(n, device="cuda"))
    table = torch.arange(-(-n // page), dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    q = _randn((1, 4, dim), 3, BF16) * 0.1
    q[0, :, 0] = torch.tensor([1.0, 0.5, 0.0, -1.0])
    out, lse = bcp.bcp_kv_attend(cache, q, table, lens, scale=1.0)
    assert_attended(out, lse, cache, q, table, lens, 1.0, 0)


@pytest.mark.parametrize("fmt", [F16, E4M3])
def test_attend_values_that_are_not_finite(cuda_device, fmt):
    table, lens, n_pages = _batch([40, 40], 16, 5)
    cache = _filled(n_pages, 2, 16, 64, fmt)
    q = _randn((2, 4, 64), 9, F16)
    page = int(table[0, 1])
    (cache.v_scale if fmt == E4M3 else cache.v)[page, 1, 3] = math.nan
    out, _ = bcp.bcp_kv_attend(cache, q, table, lens)
    assert bool(out[0, 2:].isnan().all()) and not out[0, :2].isnan().any() and not out[1].isnan().any()
    q[1, 0, 5] = math.nan
    out, lse = bcp.bcp_kv_attend(cache, q, table, lens)
    assert bool(out[1, 0].isnan().all()) and bool(lse[1, 0].isnan()) and not out[1, 1:].isnan().any()
    # keys of minus infinity weigh nothing; a row of nothing else has no mass
    if fmt == F16:
        q = torch.ones((2, 4, 64), dtype=F16, device="cuda")
        cache.v[page, 1, 3] = 0
        cache.k[page, 0, 5] = -math.inf
        out, lse = bcp.bcp_kv_attend(cache, q, table, lens)
        assert not out.isnan().any() and not lse.isinf().any()
        cache.k[:] = -math.inf
        out, lse = bcp.bcp_kv_attend(cache, q, table, lens)
        assert not out.any() and bool((lse == -math.inf).all())


@pytest.mark.parametrize("heads,group,dim,n", [(1, 4, 64, 300), (2, 16, 128, 2000), (1, 3, 256, 90)])
def test_attend_weights_over_bfloat16_caches(cuda_device, heads, group, dim, n):
    # Values that nearly cancel: neighbours are each other's negative, and their keys differ a little.  A weight reaches the product as the
    # sum of two bfloat16 numbers, the second, below 2^-7 of it, rounded to nearest: 2^-16, where one alone would be off by 2^-8.
    page = 16
    cache = _cache(-(-n // page), heads, page, dim, BF16)
    k, v = _randn((n, heads, dim), 1), _randn((n, heads, dim), 2, BF16)
    k[1::2], v[1::2] = k[0::2] * 1.004, -v[0::2]
    bcp.bcp_kv_write(cache, k.to(BF16), v, torch.arange(n, device="cuda"))
    table = torch.arange(-(-n // page), dtype=torch.int32, device="cuda")[None]
    q, scale = _randn((1, heads * group, dim), 3, BF16), dim ** -0.5
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    out, _ = bcp.bcp_kv_attend(cache, q, table, lens)
    want, sums, mass, size = attend64(cache, q, table, lens, scale, 0)
    # scores and exponentials as for any attention (rounded the same way for both neighbours or not)
    score = (dim / 2 + 4) * F32_EPS * size + 2.0 ** -21 + 4 * F32_EPS * sums.abs()
    tol = (1.01 * 2.0 ** -16 + 4 * score[..., None] + n * F32_EPS) * mass + U[BF16] * want.abs()
    assert bool(((out.double().cpu() - want).abs() <= tol).all())


def test_attend_infinite_values_stay_infinite(cuda_device):
    table, lens, n_pages = _batch([40, 40], 16, 5)
    cache = _filled(n_pages, 2, 16, 64, BF16)
    q = _randn((2, 4, 64), 9, BF16)
    q[0, 0] = 0  # equal weights, that are exact in few bits
    page = int(table[0, 1])
    cache.v[page, :, 3, 7], cache.v[page, :, 4, 9] = math.inf, -math.inf
    out, _ = bcp.bcp_kv_attend(cache, q, table, lens)
    assert bool((out[0, :, 7] == math.inf).all()) and bool((out[0, :, 9] == -math.inf).all())
    out[0, :, 7] = out[0, :, 9] = 0
    assert bool(out.isfinite().all())


def test_one_workspace_for_calls_of_different_shapes(cuda_device):
    # batches of one size after another, another head layout between them: what a call leaves must not disturb the next
    work, cases = None, []
    for i, (lengths, heads, group, dim, fmt) in enumerate([([500, 30, 700, 0, 64] * 12, 4, 8, 128, F16), ([9000], 2, 4, 128, F16),
                                                           ([40000, 5], 1, 16, 128, F16), ([300] * 9, 2, 3, 64, I8)]):
        table, lens, n_pages = _batch(lengths, 16, 5 + i)
        cache = _filled(n_pages, heads, 16, dim, fmt, seed=i)
        q = _randn((len(lengths), heads * group, dim), 9 + i, F16)
        cases.append((cache, q, table, lens, bcp.bcp_kv_attend(cache, q, table, lens)))
        w = bcp.KvWorkspace(cache, heads * group, len(lengths))
        work = w if work is None or w.bytes > work.bytes else work
    for order in ([0, 1, 2, 3], [3, 0, 2, 1], [1, 0, 3, 2]):
        for i in order * 2:
            cache, q, table, lens, (want, want_lse) = cases[i]
            out, lse = bcp.bcp_kv_attend(cache, q, table, lens, workspace=work)
            assert torch.equal(out, want) and torch.equal(lse, want_lse)
            few, _ = bcp.bcp_kv_attend(cache, q[:1], table[:1], lens[:1], workspace=work)
            assert_attended(few, _, cache, q[:1], table[:1], lens[:1], q.shape[2] ** -0.5, 0)


def test_attend_reports_bad_pages_and_lengths(cuda_device):
    table, lens, n_pages = _batch([40, 64], 16, 5)
    cache = _filled(n_pages, 2, 16, 64, BF16)
    q = _randn((2, 4, 64), 9, BF16)
    table[0, 1], table[1, 3] = n_pages, -5
    lens[1] = 65
    out, lse = bcp.bcp_kv_attend(cache, q, table, lens)
    with pytest.raises(bcp.BcpError) as e:
        cache.check()
    assert e.value.code == api.ERR_BOUNDS and "page" in str(e.value) and "length" in str(e.value)
    assert_attended(out, lse, cache, q, table, lens, 64 ** -0.5, 0)
    lens[:] = torch.tensor([-3, 2 ** 31 - 1], dtype=torch.int32)
    out, lse = bcp.bcp_kv_attend(cache, q, table, lens)
    assert_attended(out, lse, cache, q, table, lens.clamp(max=64), 64 ** -0.5, 0)
    with pytest.raises(bcp.BcpError, match="length"):
        cache.check()


def test_attend_strided_queries_and_outputs(cuda_device):
    table, lens, n_pages = _batch([40, 64, 7], 16, 5)
    cache = _filled(n_pages, 2, 16, 64, BF16)
    wide = _randn((3, 4 * 64 + 36), 9, BF16)
    q = wide[:, 4:4 + 256].view(3, 4, 64)
    out = torch.zeros((4, 3, 64), dtype=BF16, device="cuda").transpose(0, 1)
    table = torch.cat([table, table], 1)[:, :table.shape[1]]  # rows of the table apart by more than its width
    got, lse = bcp.bcp_kv_attend(cache, q, table, lens, out=out)
    assert got is out
    assert_attended(out, lse, cache, q, table, lens, 64 ** -0.5, 0)
    same, _ = bcp.bcp_kv_attend(cache, q[:, :1].expand(3, 4, 64), table, lens)  # one query for all heads
    assert_attended(same, _, cache, q[:, :1].expand(3, 4, 64), table, lens, 64 ** -0.5, 0)


@pytest.mark.parametrize("fmt", [I8])
def test_offsets_past_32_bits(cuda_device, fmt):
    # 2^32 elements and more on either side of the cache; the sequence lies in its first and last pages
    heads, page, dim = 8, 64, 128
    n_pages = (1 << 32) // (heads * page * dim) + 4
    k, v = (torch.empty((n_pages, heads, page, dim), dtype=fmt, device="cuda") for _ in range(2))
    cache = bcp.KvCache(k, v, *(torch.empty((n_pages, heads, page), device="cuda") for _ in range(2)))
    where = [0, n_pages - 1, n_pages - 2, n_pages // 2 + 1]
    table = torch.tensor([where], dtype=torch.int32, device="cuda")
    lens = torch.tensor([4 * page - 3], dtype=torch.int32, device="cuda")
    t = 4 * page
    slots = cache.slots(table, torch.zeros(t, dtype=torch.int64, device="cuda"), torch.arange(t, device="cuda"))
    x, y = _randn((t, heads, dim), 1, BF16), _randn((t, heads, dim), 2, BF16)
    bcp.bcp_kv_write(cache, x, y, slots)
    rk, rv = bcp.bcp_kv_read(cache, slots)
    small = bcp.KvCache.empty(4, heads, page, dim, fmt)
    bcp.bcp_kv_write(small, x, y, torch.arange(t, device="cuda"))
    sk, sv = bcp.bcp_kv_read(small, torch.arange(t, device="cuda"))
    assert torch.equal(rk, sk) and torch.equal(rv, sv)
    q = _randn((1, 16, dim), 3, BF16)
    got = bcp.bcp_kv_attend(cache, q, table, lens)
    want = bcp.bcp_kv_attend(small, q, torch.arange(4, dtype=torch.int32, device="cuda")[None], lens)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    cache.check()


def test_streams_and_graphs(cuda_device):
    table, lens, n_pages = _batch([300, 64, 7], 16, 5)
    cache = _filled(n_pages, 2, 16, 64, E4M3)
    rot = bcp.RopeTable.build(bcp.rope_frequencies(64), 512)
    work = bcp.KvWorkspace(cache, 8, 3)
    q, k, v = _randn((3, 8, 64), 9, BF16), _randn((3, 2, 64), 10, BF16), _randn((3, 2, 64), 11, BF16)
    positions, rows = (lens - 1).long(), torch.arange(3, device="cuda")
    slots = cache.slots(table, rows, positions)
    turned, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((3, 8), device="cuda")

    def step(stream=None):
        bcp.bcp_rope(q, rot, positions, out=turned, stream=stream)
        bcp.bcp_kv_write(cache, k, v, slots, rope=rot, positions=positions, stream=stream)
        bcp.bcp_kv_attend(cache, turned, table, lens, out=out, lse=lse, workspace=work, stream=stream)

    step()
    torch.cuda.synchronize()
    want, want_lse = out.clone(), lse.clone()
    assert_attended(out, lse, cache, turned, table, lens, 64 ** -0.5, 0)
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        out.zero_()
        torch.cuda.synchronize()
        step(stream)
        side.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    # outputs that the calls allocate belong to the stream they run on
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
    got, _ = bcp.bcp_kv_attend(cache, turned, table, lens, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    q.mul_(0.5)  # new inputs in the same places, other lengths
    lens.copy_(torch.tensor([299, 1, 0], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    assert_attended(out, lse, cache, turned, table, lens, 64 ** -0.5, 0)
    cache.check()


@pytest.mark.parametrize("fmt", [BF16, E4M3, I8])
def test_calls_in_a_row_see_what_the_ones_before_wrote(cuda_device, fmt):
    # Steps without any wait between their kernels, on lines of memory that the kernels before have read: tokens
    # join the pages (and rows of scales) that the last attention went over, a page table and the lengths change in
    # place.  The same steps with a synchronisation after every call give the reference.
    n, heads, group, dim, page, steps = 5, 2, 4, 64, 16, 60
    table0, lens0, n_pages = _batch([20 + steps] * n, page, 5)
    rot = bcp.RopeTable.build(bcp.rope_frequencies(dim), 128)
    work_of = lambda c: bcp.KvWorkspace(c, heads * group, n)  # noqa: E731
    q, k, v = (_randn((steps, n, h, dim), i, BF16 if fmt == BF16 else F16) for i, h in ((1, heads * group), (2, heads), (3, heads)))
    positions = (torch.arange(steps, device="cuda")[:, None] + 20).expand(steps, n).contiguous()
    rows = torch.arange(n, device="cuda")

    def run(wait):
        cache = _filled(n_pages, heads, page, dim, fmt)
        work, table, lens = work_of(cache), table0.clone(), lens0.clone()
        slots = [cache.slots(table0, rows, positions[s]) for s in range(steps)]
        tables = [table0.clone() for _ in range(steps)]
        for s in range(steps):
            tables[s][:, 0] = tables[s][:, 0].roll(s)  # sequences exchange their first pages
        lengths = [(positions[s] + 1).int() for s in range(steps)]
        outs = [torch.empty_like(q[0]) for _ in range(steps)]
        sums = [torch.empty((n, heads * group), device="cuda") for _ in range(steps)]
        back = [(torch.empty((n, heads, dim), dtype=F32, device="cuda"), torch.empty((n, heads, dim), dtype=F32, device="cuda")) for _ in range(steps)]
        turned = torch.empty_like(q[0])
        torch.cuda.synchronize()
        sync = torch.cuda.synchronize if wait else (lambda: None)
        for s in range(steps):
            bcp.bcp_rope(q[s], rot, positions[s], out=turned)
            sync()
            bcp.bcp_kv_write(cache, k[s], v[s], slots[s], rope=rot, positions=positions[s])
            sync()
            bcp.bcp_kv_read(cache, slots[s], out=back[s])
            sync()
            table.copy_(tables[s])
            lens.copy_(lengths[s])
            sync()
            bcp.bcp_kv_attend(cache, turned, table, lens, out=outs[s], lse=sums[s], workspace=work)
            sync()
            bcp.bcp_kv_attend(cache, turned, tables[s], lengths[s], out=outs[s], lse=sums[s], workspace=work)
            sync()
        torch.cuda.synchronize()
        cache.check()
        return outs, sums, back

    want = run(True)
    for _ in range(4):
        got = run(False)
        for w, x in zip(want[:2], got[:2]):
            assert all(torch.equal(a, b) for a, b in zip(w, x))
        assert all(torch.equal(a, b) for w, x in zip(want[2], got[2]) for a, b in zip(w, x))


def test_two_streams_with_a_workspace_each(cuda_device):
    table, lens, n_pages = _batch([2000, 64, 700], 16, 5)
    cache = _filled(n_pages, 2, 16, 128, BF16)
    q = _randn((3, 8, 128), 9, BF16)
    want, _ = bcp.bcp_kv_attend(cache, q, table, lens)
    streams = [torch.cuda.Stream() for _ in range(2)]
    works = [bcp.KvWorkspace(cache, 8, 3) for _ in range(2)]
    outs = [[torch.empty_like(q) for _ in range(20)] for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        for s, w, o in zip(streams, works, outs):
            bcp.bcp_kv_attend(cache, q, table, lens, out=o[i], workspace=w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for o in outs for x in o)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("call", ["rope", "rope_pair", "write", "write_rotated", "read", "attend"])
def test_inputs_of_another_stream_are_not_reused_too_early(cuda_device, call, raw):
    # Tensors that the current stream owns are handed to work on a stream that is still busy, and dropped: their memory must not be
    # given to new tensors of the current stream before that work is done.
    side = torch.cuda.Stream()
    stream = side.cuda_stream if raw else side
    table, lens, n_pages = _batch([300, 64, 7], 16, 5)
    cache = _filled(n_pages, 2, 16, 64, E4M3)
    rot = bcp.RopeTable.build(bcp.rope_frequencies(64), 512)
    work = bcp.KvWorkspace(cache, 8, 3)
    row = lambda i, h=2: _randn((3, h, 64), i, BF16)  # noqa: E731
    index = lambda: torch.tensor([1, 20, 3], device="cuda")  # noqa: E731
    given = {"rope": lambda: [row(1), index()], "rope_pair": lambda: [row(1, 8), row(2), index()], "write": lambda: [row(1), row(2), index()],
             "write_rotated": lambda: [row(1), row(2), index(), index()], "read": lambda: [index(), row(1), row(2)],
             "attend": lambda: [row(1, 8), row(2, 8), table.clone(), lens.clone(), torch.empty((3, 8), device="cuda")]}[call]
    made = given()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)  # a tenth of a second
    if call == "rope":
        bcp.bcp_rope(made[0], rot, made[1], stream=stream)
    elif call == "rope_pair":
        bcp.bcp_rope(made[:2], rot, made[2], out=made[:2], stream=stream)
    elif call == "write":
        bcp.bcp_kv_write(cache, *made, stream=stream)
    elif call == "write_rotated":
        bcp.bcp_kv_write(cache, made[0], made[1], made[2], rope=rot, positions=made[3], stream=stream)
    elif call == "read":
        bcp.bcp_kv_read(cache, made[0], out=(made[1], made[2]), stream=stream)
    else:
        bcp.bcp_kv_attend(cache, made[0], made[2], made[3], out=made[1], lse=made[4], workspace=work, stream=stream)
    was = {x.data_ptr() for x in made}
    del made
    again = given()
    busy = not side.query()
    side.synchronize()
    assert busy and not was & {x.data_ptr() for x in again}


def test_calls_that_name_the_capturing_stream(cuda_device):
    # tensors are recorded on a stream that is being captured, some of them from the capture's own pool
    table, lens, n_pages = _batch([300, 64, 7], 16, 5)
    cache = _filled(n_pages, 2, 16, 64, E4M3)
    rot = bcp.RopeTable.build(bcp.rope_frequencies(64), 512)
    work = bcp.KvWorkspace(cache, 8, 3)
    q, k, v = _randn((3, 8, 64), 9, BF16), _randn((3, 2, 64), 10, BF16), _randn((3, 2, 64), 11, BF16)
    positions, rows = (lens - 1).long(), torch.arange(3, device="cuda")

    def step(stream=None):
        slots = cache.slots(table, rows, positions)
        turned = bcp.bcp_rope(q, rot, positions, stream=stream)
        bcp.bcp_kv_write(cache, k, v, slots, rope=rot, positions=positions, stream=stream)
        return (*bcp.bcp_kv_attend(cache, turned, table, lens, workspace=work, stream=stream), bcp.bcp_kv_read(cache, slots, stream=stream)[0])

    want = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(torch.cuda.current_stream())
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    cache.check()


def test_workspace_zeroed_on_the_stream_that_uses_it(cuda_device):
    table, lens, n_pages = _batch([2000, 64, 700], 16, 5)
    cache = _filled(n_pages, 2, 16, 128, BF16)
    q = _randn((3, 8, 128), 9, BF16)
    want, _ = bcp.bcp_kv_attend(cache, q, table, lens)
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        with torch.cuda.stream(side):
            junk = torch.full((bcp.KvWorkspace(cache, 8, 3).bytes,), 255, dtype=torch.uint8, device="cuda")  # what the memory may hold
        torch.cuda.synchronize()
        del junk
        torch.cuda._sleep(200_000_000)  # zeroes on this stream would come too late
        got, _ = bcp.bcp_kv_attend(cache, q, table, lens, workspace=bcp.KvWorkspace(cache, 8, 3, stream=stream), stream=stream)
        side.synchronize()
        assert torch.equal(got, want)
        torch.cuda.synchronize()


def test_status_keeps_bits_that_are_set_while_it_is_read(cuda_device):
    # a bad slot on one stream, a bad page on another, somewhere around the moment in which the status is read and cleared
    table, lens, n_pages = _batch([40], 16, 5)
    cache = _filled(n_pages, 2, 16, 64, BF16)
    table[0, 1] = n_pages
    x, slots = _randn((1, 2, 64), 1, BF16), torch.tensor([n_pages * 16], device="cuda")
    q, out, lse = _randn((1, 4, 64), 9, BF16), torch.empty((1, 4, 64), dtype=BF16, device="cuda"), torch.empty((1, 4), device="cuda")
    work, side = bcp.KvWorkspace(cache, 4, 1), torch.cuda.Stream()
    torch.cuda.synchronize()

    def read():
        try:
            cache.check()
        except bcp.BcpError as e:
            return str(e)
        return ""

    for i in range(500):
        with torch.cuda.stream(side):
            torch.cuda._sleep(1 + 211 * i % 120_000)  # up to some 60 us
        bcp.bcp_kv_attend(cache, q, table, lens, out=out, lse=lse, workspace=work, stream=side.cuda_stream)
        bcp.bcp_kv_write(cache, x, x, slots)
        seen = read()
        torch.cuda.synchronize()
        seen += read()
        assert "slot" in seen and "page" in seen, (i, seen)
    assert read() == ""


def test_tensors_that_require_gradients(cuda_device):
    cache = _cache(3, 2, 16, 64, BF16)
    rot = bcp.RopeTable.build(bcp.rope_frequencies(64), 32)
    x, slots = _randn((4, 2, 64), 1, BF16), torch.arange(4, device="cuda")
    g = x.clone().requires_grad_()
    lens, table = torch.ones(4, dtype=torch.int32, device="cuda"), torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    calls = [
        lambda a: bcp.bcp_rope(a, rot, slots),
        lambda a: bcp.bcp_rope((x, a), rot, slots)[1],
        lambda a: bcp.bcp_rope_backward(a, rot, slots),
        lambda a: bcp.bcp_rope(x, rot, slots, out=a * 1),
        lambda a: bcp.bcp_kv_write(cache, a, x, slots),
        lambda a: bcp.bcp_kv_write(cache, x, a, slots, rope=rot, positions=slots),
        lambda a: bcp.bcp_kv_read(cache, slots, out=(x.clone(), a * 1))[1],
        lambda a: bcp.bcp_kv_attend(cache, a, table, lens)[0],
        lambda a: bcp.bcp_kv_attend(cache, x, table, lens, lse=(a * 1).float().sum(-1))[1],
    ]
    for i, call in enumerate(calls):
        with pytest.raises(bcp.BcpError, match="requires a gradient"):
            call(g)
            pytest.fail(f"call {i} was accepted")
        want = call(x)
        for mode in (torch.no_grad, torch.inference_mode):
            with mode():
                got = call(g)
            assert want is None or torch.equal(got, want)
    leaf = bcp.rope(g, rot, slots)  # the differentiable form takes it
    leaf.float().sum().backward()
    assert g.grad is not None


def test_outputs_count_as_written(cuda_device):
    # autograd keeps values for the backward pass: a call that overwrites them has to be noticed
    cache = _cache(3, 2, 16, 64, F16)
    rot = bcp.RopeTable.build(bcp.rope_frequencies(64), 32)
    slots = torch.arange(4, device="cuda")
    lens, table = torch.ones(4, dtype=torch.int32, device="cuda"), torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    x = [_randn((4, 2, 64), i, F16) for i in range(4)]
    sums = torch.zeros((4, 2), device="cuda")
    calls = [
        (x[0], lambda: bcp.bcp_rope(x[0], rot, slots, out=x[0])),
        (x[1], lambda: bcp.bcp_rope((x[0], x[1]), rot, slots, out=(x[0], x[1]))),
        (cache.k, lambda: bcp.bcp_kv_write(cache, x[0], x[1], slots)),
        (cache.v, lambda: bcp.bcp_kv_write(cache, x[0], x[1], slots, rope=rot, positions=slots)),
        (x[2], lambda: bcp.bcp_kv_read(cache, slots, out=(x[2], x[3]))),
        (x[3], lambda: bcp.bcp_kv_read(cache, slots, out=(x[2], x[3]))),
        (x[2], lambda: bcp.bcp_kv_attend(cache, x[0], table, lens, out=x[2], lse=sums)),
        (sums, lambda: bcp.bcp_kv_attend(cache, x[0], table, lens, out=x[2], lse=sums)),
    ]
    for kept, call in calls:
        a = torch.ones_like(kept).requires_grad_()
        y = (a * kept).float().sum()
        version = kept._version
        call()
        assert kept._version > version
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


def test_python_refusals(cuda_device):
    cache = _cache(3, 2, 16, 64, E4M3)
    rot = bcp.RopeTable.build(bcp.rope_frequencies(64), 32)
    x, slots = _randn((4, 2, 64), 1, BF16), torch.arange(4, device="cuda")
    lens, table = torch.ones(4, dtype=torch.int32, device="cuda"), torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    bad = [
        lambda: bcp.bcp_rope(x.cpu(), rot, slots),
        lambda: bcp.bcp_rope(x, rot, slots.int()),
        lambda: bcp.bcp_rope(x, rot, slots[:3]),
        lambda: bcp.bcp_rope(x[..., :32].contiguous(), rot, slots),  # shorter than the rotation
        lambda: bcp.bcp_rope(x[..., ::2], rot, slots),
        lambda: bcp.bcp_rope(x.double(), rot, slots),
        lambda: bcp.bcp_rope(x, rot, slots, out=torch.empty_like(x.float())),
        lambda: bcp.bcp_rope(x, rot, slots, out=x[:, :1].expand(4, 2, 64)),
        lambda: bcp.bcp_kv_write(cache, x, x[:, :1], slots),
        lambda: bcp.bcp_kv_write(cache, x, x.float(), slots),
        lambda: bcp.bcp_kv_write(cache, x, x, slots, rope=rot),
        lambda: bcp.bcp_kv_write(cache, x[..., :48].contiguous(), x, slots),
        lambda: bcp.bcp_kv_read(cache, slots.int()),
        lambda: bcp.bcp_kv_read(cache, slots, dtype=torch.float64),
        lambda: bcp.bcp_kv_attend(cache, x.float(), table, lens),
        lambda: bcp.bcp_kv_attend(cache, torch.cat([x, x[:, :1]], 1), table, lens),
        lambda: bcp.bcp_kv_attend(cache, x, table.long(), lens),
        lambda: bcp.bcp_kv_attend(cache, x, table, lens.long()),
        lambda: bcp.bcp_kv_attend(cache, x, table, lens, scale=math.nan),
        lambda: bcp.bcp_kv_attend(cache, x, table, lens, window=-1),
        lambda: bcp.bcp_kv_attend(cache, x, table, lens, workspace=bcp.KvWorkspace(cache, 2, 4), out=x.float()),
        lambda: bcp.bcp_kv_attend(_cache(1, 2, 16, 64, F16), x, table, lens),
        lambda: bcp.bcp_kv_attend(cache, _randn((900, 200, 64), 1, BF16), torch.zeros((900, 1), dtype=torch.int32, device="cuda"),
                                  torch.zeros(900, dtype=torch.int32, device="cuda"), workspace=bcp.KvWorkspace(cache, 2, 1)),
        lambda: bcp.KvCache(cache.k, cache.v),
        lambda: bcp.KvCache(cache.k, cache.v[:2], cache.k_scale, cache.v_scale),
        lambda: bcp.KvCache(cache.k.float(), cache.v.float()),
        lambda: bcp.RopeTable(rot.table.double()),
        lambda: bcp.RopeTable(rot.table, layout="other"),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(bcp.BcpError):
            f()
            pytest.fail(f"call {i} was accepted")
    cache.check()
    rot.check()
