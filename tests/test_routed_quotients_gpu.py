"""The router's divisions, where nothing else rounds: equal logits, whose exponentials are 1 and whose sum is whole."""
import pytest
import torch

import paper_1907_01729_amd as sk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [1, 130])
def test_weights_of_equal_logits_are_rounded_once(tokens):
    for E in range(1, 1025):
        r = sk.sinkhorn_route(torch.full((tokens, E), 1.5, device="cuda"), 1, renormalize=False)
        assert (r.weights == torch.tensor(1.0) / E).all(), E
    for k in range(1, 17):
        r = sk.sinkhorn_route(torch.zeros(tokens, 40, device="cuda"), k)
        assert (r.weights == torch.tensor(1.0) / k).all(), k


@pytest.mark.parametrize("E", [3, 7, 25, 49, 100, 231, 511, 1000])
def test_gradient_of_equal_logits(E):
    """Raw weights, one slot at expert 0: d_e = p (delta_e0 - p) with p = 1 / E: the quotient, a product or two and a
    difference: at most three roundings of p^2, two of p."""
    l = torch.zeros(5, E, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(sk.sinkhorn_route(l, 1, renormalize=False).weights.sum(), (l,))
    p = 1.0 / E
    want = torch.full((5, E), -p * p, dtype=torch.float64)
    want[:, 0] += p
    size = torch.full((5, E), p * p, dtype=torch.float64)
    size[:, 0] += p
    assert ((g.double().cpu() - want).abs() <= 4 * 2.0 ** -24 * size).all()
