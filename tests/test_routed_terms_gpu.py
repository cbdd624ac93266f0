"""The router's gradient by output, each against its own term of the formula with its own bound."""
import pytest
import torch

import paper_1907_01729_amd as sk
import routed_terms

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,k", routed_terms.SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient_of_each_output(T, E, k, dtype):
    logits, mask, renormalize, want, gw, gb, gz = routed_terms.case(T, E, k, dtype)
    dev = logits.cuda().requires_grad_()
    r = sk.sinkhorn_route(dev, k, mask=mask.cuda(), renormalize=renormalize)
    assert torch.equal(r.experts.cpu(), want["experts"])
    terms = routed_terms.terms(logits, k, want, mask, renormalize, gw, gb, gz)
    for name, incoming in (("weights", gw), ("balance", torch.tensor(gb)), ("z_loss", torch.tensor(gz))):
        got, = torch.autograd.grad(getattr(r, name), (dev,), incoming.cuda(), retain_graph=True)
        value, bound = terms[name]
        off = ~((got.double().cpu() - value).abs() <= bound)
        assert not off.any(), (name, int(off.sum()), got.cpu()[off][:4], value[off][:4], bound[off][:4])
