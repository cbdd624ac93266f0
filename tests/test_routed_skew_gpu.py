"""Experts' products where the experts' shares of the rows are far apart: the weight gradient is summed in parts of each
expert's rows, and some experts have fewer rows than there are parts, or none."""
import math

import pytest
import torch

import paper_1907_01729_amd as sk
import routed_util as ref
from paper_1907_01729_amd.routed import _experts
from routed_util import rounding

pytestmark = pytest.mark.gpu

E32 = 2.0 ** -24  # unit roundoff of 32 bits


def skewed(counts, left_out, seed):
    """One expert a token, counts[e] tokens of expert e and some of none, in no order."""
    of = torch.cat([torch.full((n,), e) for e, n in enumerate(counts)] + [torch.full((left_out,), -1)]).int()
    return ref.order_of(of[torch.randperm(len(of), generator=torch.Generator().manual_seed(seed))][:, None],
                        len(counts))


@pytest.mark.parametrize("counts,left_out", [
    ((0, 9000, 0), 0), ((65, 8000, 1), 100), ((1, 64, 20000, 0), 0), ((63, 9000, 129, 0, 7), 3), ((12000, 1), 5),
    ((0, 0, 0, 12000), 0), ((0, 0), 5000)])
@pytest.mark.parametrize("K,N", [(128, 128), (64, 200)])
@pytest.mark.parametrize("gathered", [True, False])
def test_shares_far_apart(counts, left_out, K, N, gathered):
    offsets, tokens, slots = skewed(counts, left_out, seed=len(counts))
    g = torch.Generator().manual_seed(K)
    T, E, used = tokens.numel(), len(counts), int(offsets[-1])
    dtype = torch.bfloat16
    x, gy = torch.randn(T, K, generator=g).to(dtype), torch.randn(T, N, generator=g).to(dtype)
    w = (torch.randn(E, N, K, generator=g) / math.sqrt(K)).to(dtype)
    need = _experts(T, 1, E, K, N, 1)[2]
    assert need > E * N * K * 4  # in parts
    where = tokens if gathered else None
    want = ref.products(x, w, offsets, where, gy)
    dgy, dx = gy.cuda(), x.cuda()
    dgy[used:] = math.nan  # rows of no expert take no part
    (dx if not gathered else torch.empty(0))[used:] = math.nan
    dev = (offsets.cuda(), None if where is None else where.cuda())
    workspace = torch.full((need,), 0xFF, device="cuda", dtype=torch.uint8)  # NaN wherever no sum is written
    gw = sk.sinkhorn_experts_backward_weight(dgy, dx, *dev, workspace=workspace)
    # sums in 32 bits of n products in any order, twice n E32 of their absolute values; one rounding
    assert ((gw.double().cpu() - want["gw"]).abs() <=
            rounding(want["gw"], dtype) + 2 * (max(counts) + 8) * E32 * want["abs_gw"]).all()
    y = sk.sinkhorn_experts_forward(dx, w.cuda(), *dev)
    assert ((y.double().cpu() - want["y"]).abs() <=
            rounding(want["y"], dtype) + 2 * (K + 8) * E32 * want["abs_y"]).all()
    gx = sk.sinkhorn_experts_backward_input(dgy, w.cuda(), dev[0], slots.cuda() if gathered else None)
    assert ((gx.double().cpu() - want["gx"]).abs() <=
            rounding(want["gx"], dtype) + 2 * (N + 9) * E32 * want["abs_gx"]).all()
