"""What the C entries with gradients in 32 bits refuse (no GPU needed)."""
import ctypes

import pytest

import paper_1907_01729_amd as sk
from paper_1907_01729_amd import _binding as b

P = ctypes.c_void_p(0x1000)  # never dereferenced on the paths tested


@pytest.mark.parametrize("args,code", [
    # T, k, E, K, N, dtype
    ((-1, 1, 4, 8, 8, 1), -2), ((4, 17, 4, 8, 8, 1), -2), ((4, 1, 1025, 8, 8, 1), -2), ((4, 1, 4, 65537, 8, 1), -2),
    ((4, 1, 4, 8, 8, 0), -7), ((4, 1, 4, 8, 8, 3), -7)])
def test_input_gradients_refused(args, code):
    call = sk.load_library().sinkhorn_experts_backward_input32
    assert call(ctypes.byref(b.SkExperts(*args)), *[P] * 6, 1 << 40, None) == code


def test_input_gradient_pointers():
    lib, p = sk.load_library(), ctypes.byref(b.SkExperts(4, 2, 4, 64, 32, 1))
    call, need = lib.sinkhorn_experts_backward_input32, lib.sinkhorn_experts_workspace_bytes(p)
    assert need == 4 * 2 * 64 * 4
    assert call(None, *[P] * 6, need, None) == -1
    for i in (0, 1, 2, 4):  # not slots
        assert call(p, *[None if i == j else P for j in range(6)], need, None) == -1
    assert call(p, *[P] * 6, need - 1, None) == -5 and call(p, *[P] * 5, None, need, None) == -1
    assert call(ctypes.byref(b.SkExperts(0, 2, 4, 64, 32, 1)), *[None] * 6, 0, None) == 0


def test_activation_gradients_refused():
    call = sk.load_library().sinkhorn_activation_backward32
    good = ctypes.byref(b.SkPacking(4, 8, 128, 1))
    for args, code in (((-1, 8, 128, 1), -2), ((4, 0, 128, 1), -2), ((4, 8, 0, 1), -7), ((4, 8, 128, 3), -7)):
        assert call(ctypes.byref(b.SkPacking(*args)), 2, 0, *[P] * 6) == code
    assert call(ctypes.byref(b.SkPacking(4, 7, 128, 1)), 2, 1, *[P] * 6) == -2
    assert call(good, 4, 0, *[P] * 6) == -7 and call(good, 2, 2, *[P] * 6) == -7
    assert call(good, 2, 0, ctypes.c_void_p(0x1008), *[P] * 5) == -7
    assert call(None, 2, 0, *[P] * 6) == -1 and call(good, 2, 0, None, *[P] * 5) == -1
    assert call(good, 2, 0, P, P, None, P, P, None) == -1 and call(good, 2, 0, P, P, P, P, None, None) == -1
    assert call(good, 2, 0, P, P, None, None, None, None) == 0
