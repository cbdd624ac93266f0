"""The weight gradient in parts where rows are no whole 16 bytes, or pointers are not aligned to them."""
import math

import pytest
import torch

import paper_1907_01729_amd as sk
import routed_util as ref
from paper_1907_01729_amd.routed import _experts
from routed_util import rounding

pytestmark = pytest.mark.gpu

E32 = 2.0 ** -24  # unit roundoff of 32 bits
TYPES = {torch.bfloat16: 1, torch.float16: 2}


def shifted(t):
    """The same contiguous values where no vector load can begin."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    flat[1:] = t.reshape(-1).cuda()
    return flat[1:].view(t.shape)


@pytest.mark.parametrize("counts,left_out", [((4000, 5000), 7), ((65, 8000, 1), 100), ((0, 9000, 0), 0), ((6001,), 0)])
@pytest.mark.parametrize("K,N", [(127, 128), (128, 127), (33, 17), (1, 1), (65, 200), (128, 136)])
@pytest.mark.parametrize("gathered", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
def test_parts(counts, left_out, K, N, gathered, dtype):
    of = torch.cat([torch.full((n,), e) for e, n in enumerate(counts)] + [torch.full((left_out,), -1)]).int()
    of = of[torch.randperm(len(of), generator=torch.Generator().manual_seed(K))]
    T, E = len(of), len(counts)
    offsets, tokens, _ = ref.order_of(of[:, None], E)
    g = torch.Generator().manual_seed(N)
    x, gy = torch.randn(T, K, generator=g).to(dtype), torch.randn(T, N, generator=g).to(dtype)
    want = ref.products(x, torch.zeros(E, N, K), offsets, tokens if gathered else None, gy)
    gy[int(offsets[-1]):] = math.nan  # rows of no expert take no part
    need = _experts(T, 1, E, K, N, TYPES[dtype])[2]
    assert need >= 2 * E * N * K * 4
    args = offsets.cuda(), tokens.cuda() if gathered else None
    # sums in 32 bits of n products in any order, twice n E32 of their absolute values; one rounding
    bound = rounding(want["gw"], dtype) + 2 * (max(counts) + 8) * E32 * want["abs_gw"]
    for put in (lambda t: t.cuda(), shifted):
        memory = torch.full((need + 64,), 0xFF, device="cuda", dtype=torch.uint8)  # NaN where no sum is written
        gw = sk.sinkhorn_experts_backward_weight(put(gy), put(x), *args, workspace=memory[:need])
        assert ((gw.double().cpu() - want["gw"]).abs() <= bound).all()
        assert (memory[need:] == 0xFF).all()
        assert torch.equal(gw, sk.sinkhorn_experts_backward_weight(put(gy), put(x), *args))
