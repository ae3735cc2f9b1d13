"""Autograd side of the decoding operators without a GPU: the kernel's call is replaced by the same rotation in plain torch, which
fills its output from outside the graph as the kernel does."""
from types import SimpleNamespace

import pytest
import torch

from paper_2407_20143_b200 import decode

TOKENS, HEADS, DIM, ROT = 5, 3, 10, 6


class Kernel:
    """Stands in for the binding: rotates x into out, seen by autograd as little as the kernel is."""

    def __init__(self, table):
        self.table, self.calls = table, []

    def rope(self, address, device, x, x2, out, out2, positions, transpose, stream):
        self.calls.append(transpose)
        for a, b in ((x, out), (x2, out2)):
            if a is not None:
                b.detach().copy_(turned(a.detach(), self.table, positions, transpose))


def turned(x, table, positions, transpose=False):
    n = table.shape[2]
    c, s = table[positions, 0][:, None], table[positions, 1][:, None] * (-1.0 if transpose else 1.0)
    a, b = x[..., :n], x[..., n:2 * n]
    return torch.cat([a * c - b * s, b * c + a * s, x[..., 2 * n:]], -1)


@pytest.fixture
def stand_in(monkeypatch):
    g = torch.Generator().manual_seed(3)
    angle = torch.rand((20, ROT // 2), generator=g, dtype=torch.float64) * 6
    table = 1.2 * torch.stack([angle.cos(), angle.sin()], 1)
    kernel = Kernel(table)
    monkeypatch.setattr(decode, "_b", kernel)
    return kernel, SimpleNamespace(address=0, device=-1), torch.tensor([3, 0, 19, 7, 7])


def _x(seed, heads=HEADS):
    return torch.randn((TOKENS, heads, DIM), generator=torch.Generator().manual_seed(seed), dtype=torch.float64).requires_grad_()


def test_gradients_of_every_order(stand_in):
    kernel, handle, positions = stand_in
    assert torch.autograd.gradcheck(lambda x: decode.rope(x, handle, positions), (_x(1),))
    assert torch.autograd.gradgradcheck(lambda x: decode.rope(x, handle, positions) ** 3, (_x(1),))
    assert torch.autograd.gradgradcheck(lambda x, y: tuple(t ** 2 for t in decode.rope((x, y), handle, positions)), (_x(1), _x(2, 1)))


def test_a_penalty_on_the_gradient(stand_in):
    # a loss with the square of its own gradient, against the same with a rotation that autograd sees through
    kernel, handle, positions = stand_in

    def loss(rotate, x):
        first = (rotate(x) ** 3).sum()
        g, = torch.autograd.grad(first, x, create_graph=True)
        return first + (g ** 2).sum()

    x, y = _x(4), _x(4)
    loss(lambda t: decode.rope(t, handle, positions), x).backward()
    loss(lambda t: turned(t, kernel.table, positions), y).backward()
    assert torch.allclose(x.grad, y.grad, rtol=1e-12, atol=1e-12)


def test_only_the_gradients_that_are_asked_for(stand_in, monkeypatch):
    kernel, handle, positions = stand_in
    pairs, rope = [], kernel.rope
    monkeypatch.setattr(kernel, "rope", lambda *a: (pairs.append(a[3] is not None), rope(*a)))
    x, y = _x(1), _x(2, 1)
    a, b = decode.rope((x, y), handle, positions)
    b.sum().backward()  # the first output is not used
    assert pairs == [True, False] and x.grad is None and torch.equal(y.grad, turned(torch.ones_like(y), kernel.table, positions, True).detach())
    y.requires_grad_(False)  # the second input needs none
    a, b = decode.rope((x, y), handle, positions)
    (a.sum() + (b * 2).sum()).backward()
    assert pairs == [True, False, True, False] and torch.equal(x.grad, turned(torch.ones_like(x), kernel.table, positions, True).detach())
