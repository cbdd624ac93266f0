"""Hooks on saved tensors that give the same values back with other strides: the routed layer's and the losses' gradients
are the same to the last bit."""
import pytest
import torch

import paper_1907_01729_amd as sk

pytestmark = pytest.mark.gpu


def make(*shape, seed, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda().requires_grad_()


def _spaced(t):
    s = t.new_zeros(*t.shape, 2)
    s[..., 0] = t
    return s


HOOKS = {
    "transposed": (lambda t: t.mT.contiguous() if t.dim() > 1 else t, lambda t: t.mT if t.dim() > 1 else t),
    "spaced": (_spaced, lambda s: s[..., 0]),
    "expanded": (lambda t: (t[:1].clone() if t.dim() and t.shape[0] and bool((t == t[:1]).all()) else t, t.shape),
                 lambda s: s[0].expand(s[1])),
}


def route():
    logits = make(50, 12, seed=1)
    return (logits,), lambda: [v for v in sk.sinkhorn_route(logits, 2) if v.requires_grad]


def layer(gathered):
    T, E, k, K, N = 60, 4, 2, 72, 40
    r = sk.sinkhorn_route(make(T, E, seed=1).detach(), k)
    x, w = make(T if gathered else T * k, K, seed=2, dtype=torch.bfloat16), make(E, N, K, seed=3, dtype=torch.bfloat16)
    return (x, w), lambda: (sk.sinkhorn_expert_product(x, w, r.offsets, *((r.tokens, r.slots) if gathered else ())),)


def gathered():
    return layer(True)


def in_order():
    return layer(False)


def combine():
    r = sk.sinkhorn_route(make(60, 4, seed=1).detach(), 2)
    z, w = make(120, 40, seed=2, dtype=torch.bfloat16), r.weights.clone().requires_grad_()
    return (z, w), lambda: (sk.sinkhorn_expert_combine(z, w, r.slots, r.offsets),)


def masses(B, d, seed):
    return torch.softmax(make(B, d, seed=seed).detach(), 1).requires_grad_()


def loss(sharp=False):
    mu, nu, C = masses(3, 20, 1), masses(3, 30, 2), make(20, 30, seed=3).detach().abs().requires_grad_(not sharp)
    return (mu, nu) if sharp else (mu, nu, C), lambda: (sk.sinkhorn_loss(mu, nu, C, 0.1, 50, sharp=sharp),)


def sharp_loss():
    return loss(True)


def points_loss():
    mu, nu, X, Y = masses(3, 20, 1), masses(3, 30, 2), make(20, 2, seed=3), make(30, 2, seed=4)
    return (mu, nu, X, Y), lambda: (sk.sinkhorn_loss_points(mu, nu, X, Y, 0.1, 50),)


@pytest.mark.parametrize("hook", HOOKS)
@pytest.mark.parametrize("call", [route, gathered, in_order, combine, loss, sharp_loss, points_loss])
def test_other_strides(call, hook):
    leaves, run = call()
    y = run()
    g = [make(*t.shape, seed=9 + i).detach().to(t.dtype) for i, t in enumerate(y)]
    want = torch.autograd.grad(y, leaves, g)
    seen = []
    pack, unpack = HOOKS[hook]
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (seen.append(t.dtype), pack(t))[1], unpack):
        y = run()
    got = torch.autograd.grad(y, leaves, g)
    assert seen
    for u, v in zip(got, want):
        assert u.shape == v.shape and torch.equal(u, v)
