"""Rotary positions with several axes against the definition in 64 bits: pair i of a head turned by the angle of the position on its
axis.  Tolerances: a value is computed in binary32 from two products (at most four roundings of the size of its terms) and rounded once to
its type, by at most half a step (torch.finfo(t).eps / 2); e4m3 elements 2^-4, and half a step of their smallest numbers, 2^-10 * scale."""
import pytest
import torch

import paper_2407_20143_b200 as bcp
from paper_2407_20143_b200 import api

pytestmark = pytest.mark.gpu

BF16, F16, F32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
U = {t: torch.finfo(t).eps / 2 for t in (BF16, F16, F32)}
TINY = {BF16: 2.0 ** -133, F16: 2.0 ** -25, F32: 2.0 ** -149}
F32_EPS = 2.0 ** -24


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, seed, dtype=F32):
    return torch.randn(shape, generator=_gen(seed), device="cuda").to(dtype)


def _positions(axes, tokens, most, seed):
    return torch.randint(0, most, (axes, tokens), generator=_gen(seed), device="cuda")


def turned64(x, table, axes, positions, layout, transposed=False):
    """x [tokens, heads, dim] in 64 bits, and the size of what each element is summed from."""
    x, table, positions = x.double().cpu(), table.double().cpu(), positions.cpu()
    y, size = x.clone(), x.abs()
    n = table.shape[2]
    inside = ((positions >= 0) & (positions < table.shape[0])).all(0)
    for i, a in enumerate(axes):
        row = table[positions[a].clamp(0, table.shape[0] - 1)]
        c, s = row[:, 0, i][:, None], row[:, 1, i][:, None] * (-1.0 if transposed else 1.0)
        u, v = (i, n + i) if layout == "half" else (2 * i, 2 * i + 1)
        y[..., u], y[..., v] = x[..., u] * c - x[..., v] * s, x[..., v] * c + x[..., u] * s
        size[..., u] = size[..., v] = x[..., u].abs() + x[..., v].abs()
    return y * inside[:, None, None], size * inside[:, None, None]


def assert_turned(got, x, table, positions, transposed=False):
    want, size = turned64(x, table.table, table.axes, positions, table.layout, transposed)
    tol = U[got.dtype] * want.abs() * 1.0001 + 4 * F32_EPS * size + TINY[got.dtype]
    bad = (got.double().cpu() - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), float((got.double().cpu() - want).abs().max()))


SHAPES = [  # tokens, query heads, key heads, dim, pairs of each axis
    (1, 1, 1, 64, (8, 12, 12)), (5, 4, 2, 128, (16, 24, 24)), (67, 7, 1, 96, (5, 11)), (33, 3, 3, 256, (32, 32, 32, 32)), (9, 2, 1, 80, (3, 4, 3)),
    (11, 5, 2, 30, (1, 2)), (4, 6, 3, 2, (1,)), (3, 32, 8, 128, (21, 21, 21)), (2000, 16, 4, 128, (24, 20, 20)), (700, 40, 1, 64, (16, 16)),
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("tokens,hq,hk,dim,pairs", SHAPES)
def test_axes(cuda_device, interleaved, layout, dtype, tokens, hq, hk, dim, pairs):
    table = bcp.RopeTable.build(bcp.rope_frequencies(2 * sum(pairs)), 300, layout=layout, axes=bcp.rope_axes(pairs, interleaved))
    positions = _positions(len(pairs), tokens, 300, 1)
    q, k = _randn((tokens, hq, dim), 2, dtype), _randn((tokens, hk, dim), 3, dtype)
    yq, yk = bcp.bcp_rope((q, k), table, positions)
    assert_turned(yq, q, table, positions)
    assert_turned(yk, k, table, positions)
    assert_turned(bcp.bcp_rope_backward(q, table, positions), q, table, positions, transposed=True)
    table.check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_same_position_on_every_axis_is_the_rotation_by_that_position(cuda_device, dtype):
    f, at = bcp.rope_frequencies(64), torch.randint(0, 90, (41,), generator=_gen(4), device="cuda")
    x = _randn((41, 3, 96), 5, dtype)
    plain = bcp.bcp_rope(x, bcp.RopeTable.build(f, 90), at)
    axes = bcp.RopeTable.build(f, 90, axes=bcp.rope_axes((10, 11, 11), True))
    assert torch.equal(plain, bcp.bcp_rope(x, axes, at.expand(3, -1)))  # rows without a stride between them


def test_strides_of_positions_and_in_place(cuda_device):
    table = bcp.RopeTable.build(bcp.rope_frequencies(64), 64, axes=bcp.rope_axes((16, 16)))
    many = _positions(5, 50, 64, 1)
    wide = _randn((21, 6 * 64 + 8), 2, BF16)
    for shift in (0, 1, 8):
        x = wide.clone()[:, shift:shift + 6 * 64].view(21, 6, 64)
        before, at = x.clone(), many[1:4:2, 7:28]
        assert bcp.bcp_rope(x, table, at, out=x) is x
        assert_turned(x, before, table, at)


def test_positions_out_of_the_table(cuda_device):
    table = bcp.RopeTable.build(bcp.rope_frequencies(32), 10, axes=bcp.rope_axes((4, 8, 4)))
    x = _randn((6, 2, 48), 3)
    padding = torch.tensor([[0, -1, 3, 9, 2, 5], [1, 4, -(1 << 40), 9, 2, -1], [2, 1 << 40, 3, 9, -7, 12]], device="cuda")
    y = bcp.bcp_rope(x, table, padding)  # a negative position anywhere: padding, whatever the others
    assert_turned(y, x, table, padding)
    assert not y[[1, 2, 4, 5]].any() and y[[0, 3]].any()
    table.check()
    for axis in range(3):
        past = torch.zeros((3, 6), dtype=torch.int64, device="cuda")
        past[axis, 4] = 10
        y = bcp.bcp_rope(x, table, past)
        assert_turned(y, x, table, past)
        with pytest.raises(bcp.BcpError) as e:
            table.check()
        assert e.value.code == api.ERR_BOUNDS and "position" in str(e.value)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_gradient_against_the_formula_and_differences(cuda_device, layout):
    table = bcp.RopeTable.build(bcp.rope_frequencies(32), 50, layout=layout, axes=bcp.rope_axes((4, 6, 6), True))
    positions = _positions(3, 13, 50, 6)
    q, k = _randn((13, 4, 48), 7).requires_grad_(), _randn((13, 2, 48), 8).requires_grad_()
    gq, gk = _randn((13, 4, 48), 9), _randn((13, 2, 48), 10)
    yq, yk = bcp.rope((q, k), table, positions)
    (yq * gq).sum().add((yk * gk).sum()).backward()
    assert_turned(q.grad, gq, table, positions, transposed=True)
    assert_turned(k.grad, gk, table, positions, transposed=True)
    # the map is linear: a difference along d is the map of d, and the gradient's product with d is the same number
    d = _randn((13, 4, 48), 11)
    step = (bcp.bcp_rope((q + d).detach(), table, positions).double() - yq.detach().double() * 1.0)
    a, b = float((step * gq.double()).sum()), float((q.grad.double() * d.double()).sum())
    assert abs(a - b) <= 16 * F32_EPS * float((step.abs() * gq.double().abs()).sum() + (yq.detach().double().abs() * gq.double().abs()).sum())
    # one side without gradient, an expanded gradient, a gradient of a gradient
    x = _randn((13, 4, 48), 12).requires_grad_()
    first, = torch.autograd.grad((bcp.rope(x, table, positions) ** 2).sum(), x, create_graph=True)
    first.sum().backward()
    assert torch.allclose(x.grad, torch.full_like(x, 2.0), atol=1e-5)  # the rotation keeps lengths: sum of squares of x


@pytest.mark.parametrize("fmt", [BF16, F16, E4M3, torch.int8])
@pytest.mark.parametrize("dim,pairs,interleaved", [(128, (16, 24, 24), False), (128, (24, 20, 20), True), (96, (8, 8), False), (64, (3, 2, 1), True),
                                                   (256, (40, 44, 44), True)])
def test_write_rotates_keys_by_their_axes(cuda_device, fmt, dim, pairs, interleaved):
    tokens, heads, page = 61, 3, 7
    table = bcp.RopeTable.build(bcp.rope_frequencies(2 * sum(pairs)), 90, axes=bcp.rope_axes(pairs, interleaved))
    cache = bcp.KvCache.empty(12, heads, page, dim, fmt)
    positions = _positions(len(pairs), tokens, 90, 1)
    k, v = _randn((tokens, heads, dim), 2, BF16), _randn((tokens, heads, dim), 3, BF16)
    slots = torch.randperm(84, generator=_gen(4), device="cuda")[:tokens]
    slots[5] = -1
    bcp.bcp_kv_write(cache, k, v, slots, rope=table, positions=positions)
    table.check(), cache.check()
    got, values = bcp.bcp_kv_read(cache, slots, dtype=F32)
    want, size = turned64(k, table.table, table.axes, positions, "half")
    for x, w, around in ((got, want, size), (values, v.double().cpu(), v.double().cpu().abs())):
        top = w.abs().amax(-1, keepdim=True) * 1.0001
        step = {BF16: U[BF16] * w.abs(), F16: U[F16] * w.abs() + TINY[F16], E4M3: 2.0 ** -4 * w.abs() + top / 448 * 2.0 ** -10,
                torch.int8: top / 127 / 2}[fmt]
        off = (x.double().cpu() - w).abs()
        off[5] = 0
        assert bool((off <= 1.001 * step + 8 * F32_EPS * (around + top)).all())
    assert not got[5].any()


def test_write_skips_positions_out_of_the_table(cuda_device):
    table = bcp.RopeTable.build(bcp.rope_frequencies(32), 10, axes=bcp.rope_axes((8, 8)))
    cache = bcp.KvCache.empty(2, 1, 4, 32, BF16)
    x = _randn((3, 1, 32), 1, BF16)
    positions = torch.tensor([[1, 2, 10], [3, -1, 4]], device="cuda")
    bcp.bcp_kv_write(cache, x, x, torch.tensor([0, 1, 2], device="cuda"), rope=table, positions=positions)
    with pytest.raises(bcp.BcpError):
        cache.check()
    k, v = bcp.bcp_kv_read(cache, torch.tensor([0, 1, 2], device="cuda"))
    assert k[0].any() and v[0].any() and not k[1:].any() and not v[1:].any()


def test_captured_and_on_another_stream(cuda_device):
    table = bcp.RopeTable.build(bcp.rope_frequencies(64), 100, axes=bcp.rope_axes((16, 16)))
    x, at, out = _randn((30, 4, 64), 1, BF16), _positions(2, 30, 100, 2), torch.empty((30, 4, 64), dtype=BF16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bcp.bcp_rope(x, table, at, out=out)
    x.copy_(_randn((30, 4, 64), 3, BF16)), at.copy_(_positions(2, 30, 100, 4))
    graph.replay()
    assert_turned(out, x, table, at)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    y = bcp.bcp_rope(x, table, at, stream=stream)
    stream.synchronize()
    assert torch.equal(y, out)


def test_refusals(cuda_device):
    table = bcp.RopeTable.build(bcp.rope_frequencies(32), 10, axes=bcp.rope_axes((8, 8)))
    x = _randn((4, 1, 32), 1)
    zeros = torch.zeros((2, 4), dtype=torch.int64, device="cuda")
    for positions in (zeros[0], zeros[:, :3], zeros.int(), zeros.cpu(), torch.zeros((3, 4), dtype=torch.int64, device="cuda"),
                      torch.zeros((4, 2), dtype=torch.int64, device="cuda").T, [0, 1, 2, 3]):
        with pytest.raises(bcp.BcpError):
            bcp.bcp_rope(x, table, positions)
    with pytest.raises(bcp.BcpError):  # a table without axes takes one position a token
        bcp.bcp_rope(x, bcp.RopeTable(table.table), zeros)
    for axes in ([0] * 15, [0] * 15 + [4], [0] * 15 + [-1], [0] * 17):
        with pytest.raises(bcp.BcpError):
            bcp.RopeTable(table.table, axes=axes)
    bcp.bcp_rope(x, table, zeros)
    bcp.bcp_rope(x[:0], table, zeros[:, :0])
