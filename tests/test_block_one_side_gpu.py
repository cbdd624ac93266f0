"""A block's end whose next norm has no gradient: rows that are not finite, or whose norm is not, leave that norm's weight
and bias a gradient of zero."""
import math

import pytest
import torch

import paper_1907_01729_amd as sk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [60, 4096, 8200, 20000])
@pytest.mark.parametrize("center", [False, True])
def test_no_gradient_through_the_next_norm(N, center):
    gen = torch.Generator().manual_seed(N)
    h, residual, w, b, g = (torch.randn(*s, generator=gen).cuda() for s in ((9, N), (9, N), (N,), (N,), (9, N)))
    residual[2, 5], residual[3, N - 1], residual[4, 0] = math.inf, -math.inf, math.nan
    residual[6], h[6] = 0.0, 0.0  # with eps = 0 its inverse is infinite
    for t in (h, w, b):
        t.requires_grad_()
    out, _ = sk.sinkhorn_residual_norm(h, residual, scale=0.5, before=sk.Norm(w, b, 0.0, center))
    gh, gw, gb = torch.autograd.grad(out, (h, w, b), g)
    assert torch.equal(gh, g) and not gw.any() and not gb.any()
