"""Activations of rows in 32 bits, to a few of their own units at any size of the argument."""
import pytest
import torch

import paper_1907_01729_amd as sk

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def sigmoid(x):
    return 1 / (1 + torch.exp(-x))


def arguments():
    """Single numbers under one scale each: a kept row of one number is that number, up to its scale's rounding."""
    x = torch.cat((torch.linspace(-80, 80, 1999), torch.randn(1000, generator=torch.Generator().manual_seed(1))))
    return x.cuda()[:, None]


def test_silu():
    """exp to one unit in the last place (two of 2^-24), and a sum, a quotient and a product rounded once each: 5."""
    x = arguments()
    y = sk.sinkhorn_activation(x, "silu").cpu().double()
    want = x.cpu().double() * sigmoid(x.cpu().double())
    assert bool(((y - want).abs() <= 6 * U * want.abs()).all())


def test_gradient_of_silu():
    """d = p (1 + x (1 - p)), p to 4 units as above: 1 - p is off by 4 units of p and one of its own, x (1 - p) and the sum
    by one each; then two products."""
    x = arguments().requires_grad_()
    got, = torch.autograd.grad(sk.sinkhorn_activation(x, "silu"), x, torch.ones_like(x))
    v = sk.sinkhorn_unpack(sk.sinkhorn_pack(x.detach(), 128)).cpu().double()
    p = sigmoid(v)
    q = 1 - p
    want = p * (1 + v * q)
    off = 7 * U * want.abs() + p * U * (v.abs() * (5 * p + 3 * q) + 1 + (v * q).abs())
    assert bool(((got.cpu().double() - want).abs() <= off).all())


def test_gradient_of_gelu():
    """p + x phi(x): phi's exp to two units and x^2 / 2 times two of its argument's, constant and products a unit each; p
    by the complementary error function to eight units, and x^2 of them for its argument's rounding."""
    x = arguments()[:2000].clamp(-12, 12).requires_grad_()
    got, = torch.autograd.grad(sk.sinkhorn_activation(x, "gelu"), x, torch.ones_like(x))
    v = sk.sinkhorn_unpack(sk.sinkhorn_pack(x.detach(), 128)).cpu().double()
    p = 0.5 * torch.special.erfc(-v * 0.5 ** 0.5)
    f = torch.exp(-0.5 * v * v) * 0.3989422804014327
    want = p + v * f
    off = U * ((v * f).abs() * (v * v + 6) + p * (8 + 2 * v * v) + want.abs()) + 2.0 ** -140
    assert bool(((got.cpu().double() - want).abs() <= off).all())
