"""Forward-mode differentiation of the routed layers' operators: they have no such derivative, and who asks for one gets
an error, not a result without a tangent (which would pass for a derivative of zero)."""
import pytest
import torch
import torch.autograd.forward_ad as fwad

import paper_1907_01729_amd as sk

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(*shape, dtype=torch.float32):
    return torch.randn(*shape, generator=gen(sum(shape)), device="cuda").to(dtype)


LOGITS = randn(6, 8) if torch.cuda.is_available() else None


def calls():
    """(call, its differentiable inputs) of each operator."""
    r = sk.sinkhorn_route(LOGITS, 2)
    x, w = randn(6, 16, dtype=torch.bfloat16), randn(8, 24, 16, dtype=torch.bfloat16)
    z, residual = randn(12, 10), randn(6, 10)
    return {
        "route": (lambda l: sk.sinkhorn_route(l, 2), (LOGITS,)),
        "product": (lambda a, b: sk.sinkhorn_expert_product(a, b, r.offsets, r.tokens, r.slots), (x, w)),
        "combine": (lambda a, b, c: sk.sinkhorn_expert_combine(a, b, r.slots, r.offsets, residual=c, p=0.1, seed=1),
                    (z, r.weights, residual)),
        "dropout": (lambda a, b: sk.sinkhorn_dropout(a, 0.1, 1, residual=b), (z, z + 1)),
    }


@pytest.mark.parametrize("name", ["route", "product", "combine", "dropout"])
@pytest.mark.parametrize("grad", [True, False])
def test_a_tangent_is_refused(name, grad):
    call, inputs = calls()[name]
    want = call(*inputs)
    with torch.set_grad_enabled(grad):
        for i in range(len(inputs)):
            with fwad.dual_level():
                dual = [fwad.make_dual(t, torch.ones_like(t)) if j == i else t for j, t in enumerate(inputs)]
                with pytest.raises(RuntimeError, match="forward mode AD"):
                    call(*dual)
        with fwad.dual_level():  # inputs without a tangent run as ever
            got = call(*inputs)
    for a, b in zip(want if name == "route" else (want,), got if name == "route" else (got,)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", ["route", "product", "combine", "dropout"])
def test_a_tangent_of_an_incoming_gradient_is_refused(name):
    call, inputs = calls()[name]
    leaves = [t.clone().requires_grad_() for t in inputs]
    outputs = call(*leaves)
    outputs = [outputs.weights, outputs.balance, outputs.z_loss] if name == "route" else [outputs]
    ones = [torch.ones_like(o) for o in outputs]
    want = torch.autograd.grad(outputs, leaves, ones, retain_graph=True)
    for i in range(len(outputs)):
        with fwad.dual_level():
            dual = [fwad.make_dual(t, torch.ones_like(t)) if j == i else t for j, t in enumerate(ones)]
            with pytest.raises(RuntimeError, match="forward mode AD"):
                torch.autograd.grad(outputs, leaves, dual, retain_graph=True)
            got = torch.autograd.grad(outputs, leaves, ones, retain_graph=True)
        for a, b in zip(want, got):
            assert torch.equal(a, b)
