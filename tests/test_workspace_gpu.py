"""The calls with the caller's workspace: the results of the calls without one, and refusals before a launch."""
import pytest
import torch

import paper_1907_01729_amd as sk
from paper_1907_01729_amd import _binding
from paper_1907_01729_amd.routed import _experts, _router

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def route_call():
    logits = torch.randn(3000, 40, generator=gen(1), device="cuda")
    need = _router(3000, 40, 4, 0, 1)[1]
    return need, lambda ws: sk.sinkhorn_route_forward(logits, 4, workspace=ws)[0]


def experts(T, k, E, K, N):
    g = gen(2)
    half = dict(device="cuda", dtype=torch.bfloat16, generator=g)
    r = sk.sinkhorn_route(torch.randn(T, E, generator=g, device="cuda"), k)
    return (r, torch.randn(T, K, **half), torch.randn(E, N, K, **half), torch.randn(T * k, N, **half),
            _experts(T, k, E, K, N, 1))


def input_call():
    r, _, w, gy, (_, need, _) = experts(300, 2, 4, 64, 48)
    return need, lambda ws: (sk.sinkhorn_experts_backward_input(gy, w, r.offsets, r.slots, workspace=ws),)


def weight_call():
    r, x, _, gy, (_, _, need) = experts(16384, 2, 2, 64, 128)
    return need, lambda ws: (sk.sinkhorn_experts_backward_weight(gy, x, r.offsets, r.tokens, workspace=ws),)


def forward_call(tol):
    g = gen(3)
    mu, nu = (torch.softmax(torch.randn(3, n, generator=g, device="cuda"), 1) for n in (700, 900))
    C = torch.rand(700, 900, generator=g, device="cuda")
    need = _binding.sinkhorn_workspace_bytes(3, 700, 900, 0, 0.1, 20, tol)
    return need, lambda ws: tuple(sk.sinkhorn_forward(mu, nu, C, 0.1, 20, tol, workspace=ws).values())


CALLS = {"route": route_call, "experts_input": input_call, "experts_weight": weight_call,
         "forward": lambda: forward_call(0.0), "forward_early_stop": lambda: forward_call(1e-3)}


@pytest.mark.parametrize("name", CALLS)
def test_with_the_callers_workspace(name):
    need, call = CALLS[name]()
    assert need > 0
    want = call(None)
    guard = 64
    for extra in (0, 4096):
        memory = torch.full((need + extra + guard,), 0xA5, device="cuda", dtype=torch.uint8)
        got = call(memory[:need + extra])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert (memory[need + extra:] == 0xA5).all()  # nothing past what was given
        assert (memory[:need] != 0xA5).any()  # it is what the kernels used
    floats = torch.empty((need + 3) // 4, device="cuda")
    for ws in (floats, torch.empty(need - 1, device="cuda", dtype=torch.uint8),
               torch.empty(need + 8, device="cuda", dtype=torch.uint8)[8:]):  # by bytes; too small; askew
        assert all(torch.equal(a, b) for a, b in zip(call(ws), want))
    for bad, error in ((torch.empty(need, dtype=torch.uint8), TypeError), (need, TypeError),
                       (torch.empty(1, device="cuda", dtype=torch.uint8).expand(need), ValueError),
                       (torch.empty(2 * need, device="cuda", dtype=torch.uint8)[::2], ValueError)):
        with pytest.raises(error):
            call(bad)
