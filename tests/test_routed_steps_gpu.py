"""Whole training steps of a routed layer: captured with their backward pass, and with many slots to a token."""
import pytest
import torch

import paper_1907_01729_amd as sk
from test_routed_gpu import BF16, F16, F32, check_combine, layer, layer_inputs

pytestmark = pytest.mark.gpu


def step(args, gy, seed):
    """The layer's result, its losses, and the gradients of its inputs."""
    y, r = layer(*args, seed)
    one = torch.ones((), device="cuda")
    return [y, *r, *torch.autograd.grad((y, r.balance, r.z_loss), args[:4], (gy, one, one))]


@pytest.mark.parametrize("T", [4, 600])
def test_forward_and_backward_in_a_graph(T):
    """Captured once, replayed on new inputs with the program's own work between, against the eager step."""
    args = layer_inputs(T, 3)
    for t in args[:4]:
        t.requires_grad_()
    gy = torch.randn(T, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step(args, gy, 9)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(args, gy, 9)
    for seed in range(5):
        with torch.no_grad():
            for t, new in zip(args, layer_inputs(T, 40 + seed)):
                t.copy_(new)
            gy.copy_(gy.flip(0))
        graph.replay()
        torch.cuda.synchronize()
        want = step(args, gy, 9)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("T,D,k,dtype", [(2048, 1024, 8, BF16), (1500, 516, 6, F32), (1024, 257, 16, F16)])
def test_combination_of_many_slots(T, D, k, dtype):
    check_combine(T, D, k, dtype, 0.1)
