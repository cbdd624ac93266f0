"""Rows of more than 2^24 pairs in order: a layer's second product has as many rows as its first."""
import pytest
import torch

import paper_1907_01729_amd as sk
import routed_util as ref
from routed_util import rounding

pytestmark = pytest.mark.gpu

E32 = 2.0 ** -24  # unit roundoff of 32 bits


@pytest.mark.parametrize("rows", [(1 << 24) + 16, 3 * ((1 << 23) + 5)])
def test_rows_in_order(rows):
    K, N, E = 16, 8, 3
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, K, generator=g, device="cuda").bfloat16().requires_grad_()
    w = torch.randn(E, N, K, generator=g, device="cuda").bfloat16().requires_grad_()
    offsets = torch.tensor([0, rows // 3, rows - 500, rows - 100], dtype=torch.int32, device="cuda")
    gy = torch.zeros(rows, N, device="cuda", dtype=torch.bfloat16)
    some = torch.cat([torch.arange(0, 200), torch.arange(rows // 3 - 100, rows // 3 + 100),
                      torch.arange(rows - 600, rows - 100)]).cuda()  # the others' gradients are zeros and add nothing
    gy[some] = torch.randn(len(some), N, generator=g, device="cuda").bfloat16()
    y = sk.sinkhorn_expert_product(x, w, offsets)
    gx, gw = torch.autograd.grad(y, (x, w), gy)
    of = torch.searchsorted(offsets[1:], some, right=True)
    assert (of[1:] >= of[:-1]).all()
    few = torch.cat([of.new_zeros(1), torch.bincount(of, minlength=E).cumsum(0)])
    want = ref.products(x[some].detach().cpu(), w.detach().cpu(), few.cpu(), None, gy[some].cpu())
    # sums in 32 bits of n products in any order, twice n E32 of their absolute values; one rounding
    for got, name, n in ((y[some], "y", K), (gx[some], "gx", N), (gw, "gw", len(some))):
        bound = rounding(want[name], torch.bfloat16) + 2 * (n + 8) * E32 * want["abs_" + name]
        assert ((got.double().cpu() - want[name]).abs() <= bound).all(), name
    assert (y[rows - 100:] == 0).all() and (gx[rows - 100:] == 0).all() and y.shape == (rows, N)


def test_what_cannot_be_split_is_refused():
    rows = (1 << 24) + 43  # a prime
    with pytest.raises(sk.SinkhornError):
        sk.sinkhorn_experts_forward(torch.empty(rows, 8, device="cuda", dtype=torch.bfloat16),
                                    torch.empty(1, 8, 8, device="cuda", dtype=torch.bfloat16),
                                    torch.zeros(2, device="cuda", dtype=torch.int32))
