"""Host-side checks of the routed-layer operators: what the C ABI and the wrappers refuse (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_1907_01729_amd as sk
from paper_1907_01729_amd import _binding as b

P = ctypes.c_void_p(0x1000)  # never dereferenced on the paths tested


def route(r, ws=0, ptr=P, wsp=P):
    return sk.load_library().sinkhorn_route_forward(ctypes.byref(r), ptr, None, None, *[ptr] * 9, wsp,
                                                    ctypes.c_size_t(ws), None)


def route_back(r, ptr=P):
    return sk.load_library().sinkhorn_route_backward(ctypes.byref(r), *[ptr] * 5, None, None, None, ptr, None)


@pytest.mark.parametrize("args,code", [
    ((-1, 8, 2, 0, 1), -2), ((1 << 25, 8, 2, 0, 1), -2), ((4, 0, 1, 0, 1), -2), ((4, 1025, 1, 0, 1), -2),
    ((4, 8, 0, 0, 1), -2), ((4, 8, 9, 0, 1), -2), ((4, 64, 17, 0, 1), -2), ((4, 8, 2, 3, 1), -7),
    ((4, 8, 2, -1, 1), -7), ((4, 8, 2, 0, 2), -7),
])
def test_router_refusals(args, code):
    r = b.SkRouter(*args)
    assert route(r) == code and route_back(r) == code
    assert sk.load_library().sinkhorn_route_workspace_bytes(ctypes.byref(r)) == 0


def test_router_workspace_and_pointers():
    lib = sk.load_library()
    r = b.SkRouter(10000, 64, 2, 1, 1)
    need = lib.sinkhorn_route_workspace_bytes(ctypes.byref(r))
    assert need > 0
    assert route(r, ws=need - 1) == -5
    assert route(r, ws=need, ptr=None) == -1
    assert route(r, ws=need, wsp=None) == -1
    assert route_back(r, ptr=None) == -1
    assert route_back(b.SkRouter(0, 64, 2, 1, 1), ptr=None) == 0
    assert lib.sinkhorn_route_forward(None, *[P] * 13, ctypes.c_size_t(0), None) == -1
    assert lib.sinkhorn_route_workspace_bytes(ctypes.byref(b.SkRouter(1, 64, 2, 1, 1))) == 0


@pytest.mark.parametrize("args,code", [
    # T, k, E, K, N, dtype
    ((-1, 1, 4, 8, 8, 1), -2), ((4, 0, 4, 8, 8, 1), -2), ((4, 17, 4, 8, 8, 1), -2), ((4, 1, 0, 8, 8, 1), -2),
    ((4, 1, 1025, 8, 8, 1), -2), ((4, 1, 4, 0, 8, 1), -2), ((4, 1, 4, 8, 0, 1), -2), ((4, 1, 4, 65537, 8, 1), -2),
    ((1 << 24, 16, 4, 4096, 8, 1), -2), ((4, 1, 1024, 8192, 8192, 1), -2), ((4, 1, 4, 8, 8, 0), -7),
    ((4, 1, 4, 8, 8, 3), -7),
])
def test_experts_refusals(args, code):
    lib = sk.load_library()
    p = b.SkExperts(*args)
    assert lib.sinkhorn_experts_forward(ctypes.byref(p), P, P, P, P, P, None) == code
    assert lib.sinkhorn_experts_backward_input(ctypes.byref(p), P, P, P, P, P, P, ctypes.c_size_t(0), None) == code
    assert lib.sinkhorn_experts_backward_weight(ctypes.byref(p), P, P, P, P, P, P, ctypes.c_size_t(0), None) == code
    assert lib.sinkhorn_experts_workspace_bytes(ctypes.byref(p)) == 0
    assert lib.sinkhorn_experts_weight_workspace_bytes(ctypes.byref(p)) == 0


def test_experts_workspace_and_pointers():
    lib = sk.load_library()
    p = b.SkExperts(100, 2, 4, 64, 32, 1)
    need = lib.sinkhorn_experts_workspace_bytes(ctypes.byref(p))
    assert need > 0
    back = lib.sinkhorn_experts_backward_input
    assert back(ctypes.byref(p), P, P, P, P, P, P, ctypes.c_size_t(need - 1), None) == -5
    assert back(ctypes.byref(p), P, P, P, P, P, None, ctypes.c_size_t(need), None) == -1
    assert back(ctypes.byref(p), P, P, P, P, None, P, ctypes.c_size_t(need), None) == -1
    assert lib.sinkhorn_experts_forward(ctypes.byref(p), None, P, P, P, P, None) == -1
    assert lib.sinkhorn_experts_forward(None, P, P, P, P, P, None) == -1
    weight = lib.sinkhorn_experts_backward_weight
    assert weight(ctypes.byref(p), P, None, P, P, P, P, ctypes.c_size_t(1 << 30), None) == -1
    many = b.SkExperts(16384, 2, 2, 128, 128, 1)  # two small matrices over many rows: summed in parts
    need = lib.sinkhorn_experts_weight_workspace_bytes(ctypes.byref(many))
    assert need >= 2 * 2 * 128 * 128 * 4 and need % (2 * 128 * 128 * 4) == 0
    assert weight(ctypes.byref(many), P, P, P, P, P, P, ctypes.c_size_t(need - 1), None) == -5
    assert weight(ctypes.byref(many), P, P, P, P, P, None, ctypes.c_size_t(need), None) == -1
    assert lib.sinkhorn_experts_weight_workspace_bytes(ctypes.byref(b.SkExperts(64, 2, 8, 2048, 2048, 1))) == 0
    assert lib.sinkhorn_experts_forward(ctypes.byref(b.SkExperts(0, 2, 4, 64, 32, 1)), None, None, None, None, None,
                                        None) == 0


def dropout(n=8, dtype=0, p=0.5, ptr=P):
    return sk.load_library().sinkhorn_dropout(n, dtype, ptr, None, ptr, p, 1, 2, None)


def test_dropout_refusals():
    assert dropout(n=-1) == -2 and dropout(n=(1 << 34) + 1) == -2
    assert dropout(dtype=3) == -7 and dropout(dtype=-1) == -7
    for p in (-1e-9, 1.0, 2.0, float("nan"), float("inf")):
        assert dropout(p=p) == -7
    assert dropout(ptr=None) == -1
    assert dropout(n=0, ptr=None) == 0


@pytest.mark.parametrize("args,code", [
    # T, D, k, dtype
    ((-1, 8, 1, 0), -2), ((4, 0, 1, 0), -2), ((4, 8, 0, 0), -2), ((4, 8, 17, 0), -2), ((1 << 24, 1024, 2, 0), -2),
    ((4, 8, 1, 5), -7),
])
def test_combine_refusals(args, code):
    lib = sk.load_library()
    c = b.SkCombine(*args)
    assert lib.sinkhorn_combine_forward(ctypes.byref(c), P, P, P, None, P, 0.1, 1, 2, None) == code
    assert lib.sinkhorn_combine_backward(ctypes.byref(c), P, P, P, P, P, P, P, 0.1, 1, 2, None) == code


def test_combine_pointers_and_rate():
    lib = sk.load_library()
    c = b.SkCombine(4, 8, 2, 1)
    assert lib.sinkhorn_combine_forward(ctypes.byref(c), P, P, P, None, P, 1.0, 1, 2, None) == -7
    assert lib.sinkhorn_combine_forward(ctypes.byref(c), None, P, P, None, P, 0.1, 1, 2, None) == -1
    assert lib.sinkhorn_combine_backward(ctypes.byref(c), P, P, P, None, P, P, P, 0.1, 1, 2, None) == -1
    assert lib.sinkhorn_combine_forward(None, P, P, P, None, P, 0.1, 1, 2, None) == -1
    assert lib.sinkhorn_combine_forward(ctypes.byref(b.SkCombine(0, 8, 2, 1)), None, None, None, None, None, 0.1, 1,
                                        2, None) == 0


def test_wrappers_refuse_cpu_tensors():
    with pytest.raises(TypeError):
        sk.sinkhorn_route(torch.zeros(4, 8), 2)
    with pytest.raises(TypeError):
        sk.sinkhorn_dropout(torch.zeros(4), 0.1, 1)
    with pytest.raises(TypeError):
        sk.sinkhorn_expert_product(torch.zeros(4, 8), torch.zeros(2, 8, 8), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError):
        sk.sinkhorn_expert_combine(torch.zeros(8, 8), torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.int32),
                                   torch.zeros(3, dtype=torch.int32))
