"""A routed layer under torch.jit.trace, with and without gradients: the trace holds its calls, not their allocations."""
import pytest
import torch

import paper_1907_01729_amd as sk

pytestmark = pytest.mark.gpu


def make(*shape, seed, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def calls():
    T, E, k, K, N = 60, 4, 2, 72, 40
    r = sk.sinkhorn_route(make(T, E, seed=1), k)
    w, residual = make(E, N, K, seed=3, dtype=torch.bfloat16), make(T, N, seed=4, dtype=torch.bfloat16)
    return {"route": ((T, E), torch.float32, lambda x: tuple(sk.sinkhorn_route(x, k))),
            "product": ((T, K), torch.bfloat16, lambda x: sk.sinkhorn_expert_product(x, w, r.offsets, r.tokens, r.slots)),
            "dropout": ((T, K), torch.bfloat16, lambda x: sk.sinkhorn_dropout(x, 0.3, 5)),
            "combine": ((T * k, N), torch.bfloat16,
                        lambda x: sk.sinkhorn_expert_combine(x, r.weights, r.slots, r.offsets, residual=residual))}


@pytest.mark.parametrize("name", ["route", "product", "dropout", "combine"])
@pytest.mark.parametrize("grad", [False, True])
def test_a_trace_replays_the_call(name, grad):
    shape, dtype, call = calls()[name]
    with torch.set_grad_enabled(grad):
        traced = torch.jit.trace(call, make(*shape, seed=10, dtype=dtype).requires_grad_(grad), check_trace=False)
        for seed in (11, 12):
            x = make(*shape, seed=seed, dtype=dtype).requires_grad_(grad)
            got, want = traced(x), call(x)
            for u, v in zip(*((got, want) if isinstance(want, tuple) else ((got,), (want,)))):
                assert torch.equal(u, v)
            if grad:
                u, v = (y[0] if isinstance(y, tuple) else y for y in (got, want))
                g = make(*u.shape, seed=20, dtype=u.dtype)
                assert torch.equal(torch.autograd.grad(u, x, g)[0], torch.autograd.grad(v, x, g)[0])
