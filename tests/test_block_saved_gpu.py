"""Hooks on saved tensors that give the same values back with other strides, and at other addresses: the gradients are
the same to the last bit."""
import pytest
import torch

import paper_1907_01729_amd as sk
from routed_util import order_of

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def make(*shape, seed, dtype=BF16):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda().requires_grad_()


def _spaced(t):
    s = t.new_zeros(*t.shape, 2)
    s[..., 0] = t
    return s


def _shifted(t):
    s = t.new_zeros(t.numel() + 1)
    s[1:] = t.reshape(-1)
    return s, t.shape


HOOKS = {
    "transposed": (lambda t: t.mT.contiguous() if t.dim() > 1 else t, lambda t: t.mT if t.dim() > 1 else t),
    "spaced": (_spaced, lambda s: s[..., 0]),
    "shifted": (_shifted, lambda s: s[0][1:].view(s[1])),
    "expanded": (lambda t: (t[:1].clone() if t.dim() and t.shape[0] and bool((t == t[:1]).all()) else t, t.shape),
                 lambda s: s[0].expand(s[1])),
}


def norms():
    x, w, b = make(37, 72, seed=1), make(72, seed=2), make(72, seed=3)
    return (x, w, b), lambda: (sk.sinkhorn_norm(x, sk.Norm(w, b, 1e-5, True)),)


def block_ends(T=37, same=False):
    h, residual, gate = make(T, 72, seed=1), make(T, 72, seed=2), make(T, 72, seed=3)
    if same:  # rows that are alike come back as one row
        h, residual, gate = (t.detach()[:1].repeat(T, 1).requires_grad_() for t in (h, residual, gate))
    p = [make(72, seed=4 + i) for i in range(4)]
    return (h, residual, gate, *p), lambda: sk.sinkhorn_residual_norm(h, residual, gate, 0.7, sk.Norm(*p[:2]),
                                                                      sk.Norm(*p[2:]))


def equal_block_ends():
    return block_ends(same=True)


def activations():
    x = make(37, 2 * 200, seed=1)
    return (x,), lambda: (sk.sinkhorn_activation(x, "silu", True),)


def kept(gathered, activation, gated):
    T, E, k, K, N = 90, 3, 2, 136, 40
    offsets, tokens, slots = (t.cuda() for t in order_of(
        torch.rand(T, E, generator=torch.Generator().manual_seed(5)).topk(k, 1).indices.int(), E))
    if not gathered:
        T, tokens, slots = T * k, None, None
    x, w = make(T, K * (1 + gated), seed=1), make(E, N, K, seed=2)
    return (x, w), lambda: (sk.sinkhorn_expert_product_kept(x, w, offsets, tokens, slots, activation, gated),)


def kept_plain():
    return kept(True, "none", False)


def kept_gathered():
    return kept(True, "gelu", False)


def kept_gated():
    return kept(False, "silu", True)


@pytest.mark.parametrize("hook", HOOKS)
@pytest.mark.parametrize("call", [norms, block_ends, equal_block_ends, activations, kept_plain, kept_gathered, kept_gated])
def test_other_strides(call, hook):
    leaves, run = call()
    y = run()
    g = [make(*t.shape, seed=9 + i).detach() for i, t in enumerate(y)]
    want = torch.autograd.grad(y, leaves, g)
    seen = []
    pack, unpack = HOOKS[hook]
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (seen.append(t.dtype), pack(t))[1], unpack):
        y = run()
    got = torch.autograd.grad(y, leaves, g)
    assert seen
    for u, v in zip(got, want):
        assert u.shape == v.shape and torch.equal(u, v)
