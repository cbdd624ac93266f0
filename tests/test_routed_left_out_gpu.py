"""Pairs that a program leaves out after routing, as a limit on an expert's rows does: their slots are -1, their rows
stay among the experts' rows, and no slot names them."""
import pytest
import torch

import paper_1907_01729_amd as sk

pytestmark = pytest.mark.gpu

SIZES = [(1, 8, 1), (4, 5, 2), (40, 2048, 4), (777, 33, 2), (300, 64, 16), (3, 1001, 5), (20000, 8, 3)]


def limited(T, E, k, most, seed):
    """A routing of which each expert keeps its first `most` rows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    mask = torch.rand(T, generator=g, device="cuda") < 0.9
    r = sk.sinkhorn_route(torch.randn(T, E, generator=g, device="cuda") + 2 * torch.arange(E, device="cuda"), k,
                          mask=mask)
    rank = r.slots - r.offsets[r.experts.clamp(min=0).long()]
    return r, torch.where((r.slots >= 0) & (rank < most), r.slots, -1)


@pytest.mark.parametrize("T,D,k", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_rows_that_no_slot_names_have_no_gradient(T, D, k, dtype, p):
    r, slots = limited(T, max(k, 3), k, most=max(1, T // 2), seed=T)
    g = torch.Generator(device="cuda").manual_seed(D)
    z = torch.randn(T * k, D, generator=g, device="cuda").to(dtype)
    gy = torch.randn(T, D, generator=g, device="cuda").to(dtype)
    named = torch.zeros(T * k, dtype=torch.bool, device="cuda")
    named[slots[slots >= 0].long()] = True
    assert T < 40 or (~named[:int(r.offsets[-1])]).any()
    z[~named] = float("nan")  # takes no part
    # memory that the result may get, with something in it
    for _ in range(4):
        torch.full_like(z, 7.0)
        torch.full((T, k), float(3), device="cuda")
    torch.cuda.synchronize()
    leaves = z.clone().requires_grad_(), r.weights.clone().requires_grad_()
    y = sk.sinkhorn_expert_combine(*leaves, slots, r.offsets, p=p, seed=3)
    torch.full_like(z, 7.0), torch.full((T, k), float(3), device="cuda")
    gz, gw = torch.autograd.grad(y, leaves, gy)
    assert (gz[~named] == 0).all()
    assert (gw[slots < 0] == 0).all() and torch.isfinite(gw).all()
    # the rows that are named: as with the whole routing, which the pairs left out do not touch
    clean = torch.nan_to_num(z)
    whole, _ = sk.sinkhorn_combine_backward(clean, r.weights, r.slots, r.offsets, gy, p, 3)
    assert torch.equal(gz[named], whole[named])
    # every row, where no slot is left
    none = torch.full_like(slots, -1)
    gz, gw = sk.sinkhorn_combine_backward(clean, r.weights, none, r.offsets, gy, p, 3)
    assert not gz.any() and not gw.any()


def test_a_layer_with_a_limit():
    """The products' gradients with pairs left out, against the same layer with their rows' weights at zero."""
    T, k, E, D = 500, 2, 6, 32
    r, slots = limited(T, E, k, most=60, seed=5)
    g = torch.Generator(device="cuda").manual_seed(6)
    x, w = (torch.randn(*s, generator=g, device="cuda").bfloat16() for s in ((T, D), (E, D, D)))
    gy = torch.randn(T, D, generator=g, device="cuda").bfloat16()

    def layer(slots, weights):
        leaves = x.clone().requires_grad_(), w.clone().requires_grad_()
        h = sk.sinkhorn_expert_product(*leaves, r.offsets, r.tokens, slots)
        y = sk.sinkhorn_expert_combine(h, weights, slots, r.offsets, p=0.1, seed=2)
        return y, *torch.autograd.grad(y, leaves, gy)

    zeroed = torch.where(slots >= 0, r.weights, 0.0)
    assert (zeroed != r.weights).any()
    for a, b in zip(layer(slots, r.weights), layer(r.slots, zeroed)):
        assert torch.equal(a, b)
