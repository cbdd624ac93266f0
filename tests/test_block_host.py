"""Host-side checks of the norms, the rows in 8 bits and their products: what the C ABI and the wrappers refuse (no GPU
needed)."""
import ctypes

import pytest
import torch

import paper_1907_01729_amd as sk
from paper_1907_01729_amd import _binding as b
from paper_1907_01729_amd import norm

P = ctypes.c_void_p(0x1000)  # never dereferenced on the paths tested
ODD = ctypes.c_void_p(0x1008)
INF, NAN = float("inf"), float("nan")

GOOD = dict(T=300, N=64, dtype=1, wdtype=1, gate=0, gdtype=0, after=1, before=1, scale=1.0, eps_after=0.0, eps_before=0.0)


def norms(**changes):
    return b.SkNorms(*{**GOOD, **changes}.values())


def norm_calls(p, ws=1 << 40):
    lib, ref = sk.load_library(), ctypes.byref(p)
    return {"forward": lib.sinkhorn_norm_forward(ref, *[P] * 6),
            "backward": lib.sinkhorn_norm_backward(ref, *[P] * 8, ctypes.c_size_t(ws), None)}


def residual_calls(p, ws=1 << 40):
    lib, ref = sk.load_library(), ctypes.byref(p)
    return {"forward": lib.sinkhorn_residual_norm_forward(ref, *[P] * 11),
            "backward": lib.sinkhorn_residual_norm_backward(ref, *[P] * 17, ctypes.c_size_t(ws), None)}


@pytest.mark.parametrize("changes,code", [
    (dict(T=-1), -2), (dict(T=(1 << 24) + 1), -2), (dict(N=0), -2), (dict(N=(1 << 16) + 1), -2),
    (dict(T=1 << 24, N=1025), -2), (dict(dtype=3), -7), (dict(dtype=-1), -7), (dict(wdtype=2), -7), (dict(wdtype=3), -7),
    (dict(before=3), -7), (dict(before=-1), -7), (dict(eps_before=-1e-9), -7), (dict(eps_before=INF), -7),
    (dict(eps_before=NAN), -7)])
def test_norms_refused(changes, code):
    p = norms(**changes)
    assert set(norm_calls(p).values()) == {code}
    assert set(residual_calls(p).values()) == {code}
    assert sk.load_library().sinkhorn_norm_workspace_bytes(ctypes.byref(p)) == 0


@pytest.mark.parametrize("changes,code", [
    (dict(gate=4), -7), (dict(gate=-1), -7), (dict(gate=1, gdtype=2), -7), (dict(after=3), -7), (dict(eps_after=NAN), -7),
    (dict(scale=INF), -7), (dict(scale=NAN), -7)])
def test_block_ends_refused(changes, code):
    p = norms(**changes)
    assert set(residual_calls(p).values()) == {code}
    assert sk.load_library().sinkhorn_norm_workspace_bytes(ctypes.byref(p)) == 0


def test_norm_pointers_and_workspace():
    lib, p = sk.load_library(), norms()
    ref, need = ctypes.byref(p), lib.sinkhorn_norm_workspace_bytes(ctypes.byref(norms()))
    assert need > 0
    z = ctypes.c_size_t
    assert lib.sinkhorn_norm_forward(ref, None, *[P] * 5) == -1
    assert lib.sinkhorn_norm_forward(ctypes.byref(norms(before=0)), *[P] * 6) == -7
    assert lib.sinkhorn_norm_backward(ref, *[P] * 8, z(need - 1), None) == -5
    assert lib.sinkhorn_norm_backward(ref, *[P] * 7, None, z(need), None) == -1
    assert lib.sinkhorn_norm_backward(ref, P, P, None, *[P] * 5, z(need), None) == -1
    back = lib.sinkhorn_residual_norm_backward
    full = ctypes.byref(norms(gate=2))
    assert back(full, *[P] * 17, z(need - 1), None) == -5
    assert back(full, None, *[P] * 16, z(need), None) == -1
    assert back(full, P, None, *[P] * 15, z(need), None) == -1
    assert back(full, P, P, None, *[P] * 14, z(need), None) == -1
    assert back(ref, *[P] * 17, z(need), None) == -7  # a gradient of a gate that there is not
    assert back(ctypes.byref(norms(gate=2, after=0)), *[P] * 17, z(need), None) == -7
    assert back(ctypes.byref(norms(gate=2, before=0)), *[P] * 17, z(need), None) == -7
    forward = lib.sinkhorn_residual_norm_forward
    assert forward(full, P, P, None, *[P] * 8) == -1
    assert forward(full, *[P] * 8, None, P, P) == -1
    for fn, n in ((lib.sinkhorn_norm_forward, 6), (forward, 11)):
        assert fn(None, *[P] * n) == -1
        assert fn(ctypes.byref(norms(T=0)), *[None] * n) == 0


@pytest.mark.parametrize("args,code", [
    # rows, columns, block, dtype
    ((-1, 8, 0, 1), -2), (((1 << 26) + 1, 8, 0, 1), -2), ((4, 0, 0, 1), -2), ((4, (1 << 17) + 1, 0, 1), -2),
    ((1 << 26, 512, 0, 1), -2), ((4, 8, 64, 1), -7), ((4, 8, -1, 1), -7), ((4, 8, 0, 3), -7)])
def test_packings_refused(args, code):
    lib, ref = sk.load_library(), ctypes.byref(b.SkPacking(*args))
    assert lib.sinkhorn_pack(ref, *[P] * 4) == code
    assert lib.sinkhorn_unpack(ref, *[P] * 4) == code
    assert lib.sinkhorn_activation_forward(ref, 2, 0, *[P] * 5) == code
    assert lib.sinkhorn_activation_backward(ref, 2, 0, *[P] * 6) == code


def test_packing_pointers():
    lib = sk.load_library()
    ref = ctypes.byref(b.SkPacking(4, 8, 128, 1))
    row = ctypes.byref(b.SkPacking(4, 8, 0, 1))
    assert lib.sinkhorn_pack(None, *[P] * 4) == -1 and lib.sinkhorn_pack(ref, None, P, P, None) == -1
    assert lib.sinkhorn_pack(ref, P, ODD, P, None) == -7 and lib.sinkhorn_unpack(ref, ODD, P, P, None) == -7
    assert lib.sinkhorn_pack(ctypes.byref(b.SkPacking(0, 8, 0, 1)), None, None, None, None) == 0
    forward, back = lib.sinkhorn_activation_forward, lib.sinkhorn_activation_backward
    for kind, gated in ((-1, 0), (4, 0), (2, 2)):
        assert forward(ref, kind, gated, *[P] * 5) == -7 and back(ref, kind, gated, *[P] * 6) == -7
    assert forward(ctypes.byref(b.SkPacking(4, 7, 128, 1)), 2, 1, *[P] * 5) == -2
    assert forward(ref, 2, 0, P, P, P, None, None) == -1 and forward(ref, 2, 0, P, P, None, P, None) == -1
    assert forward(row, 2, 0, *[P] * 5) == -7  # kept rows have a scale for 128 columns
    assert back(row, 2, 0, *[P] * 6) == -7
    assert back(ref, 2, 0, P, P, None, P, P, None) == -1 and back(ref, 2, 0, None, P, P, P, P, None) == -1
    assert back(ref, 2, 0, P, P, None, None, None, None) == 0


@pytest.mark.parametrize("args,code", [
    # T, k, E, K, N, dtype
    ((-1, 1, 4, 8, 8, 1), -2), ((4, 17, 4, 8, 8, 1), -2), ((4, 1, 1025, 8, 8, 1), -2), ((4, 1, 4, 65537, 8, 1), -2),
    ((1 << 24, 16, 4, 4096, 8, 1), -2), ((4, 1, 4, 8, 8, 3), -7)])
def test_packed_products_refused(args, code):
    assert sk.load_library().sinkhorn_experts_forward_packed(ctypes.byref(b.SkExperts(*args)), *[P] * 8) == code


def test_packed_product_pointers():
    call = sk.load_library().sinkhorn_experts_forward_packed
    p = ctypes.byref(b.SkExperts(4, 2, 4, 64, 32, 0))
    assert call(None, *[P] * 8) == -1
    for i in (0, 1, 2, 3, 4, 6):  # not tokens; offsets only with one expert
        assert call(p, *[None if i == j else P for j in range(7)], None) == -1
    assert call(p, ODD, *[P] * 7) == -7 and call(p, P, P, ODD, *[P] * 5) == -7
    assert call(ctypes.byref(b.SkExperts(0, 2, 4, 64, 32, 0)), *[None] * 8) == 0


def test_sizes_are_not_cut_off():
    for n in (1 << 31, (1 << 32) + 4, -(1 << 32) + 4):
        for i in range(2):
            with pytest.raises(sk.SinkhornError):
                norm._norms(*[n if i == j else 4 for j in range(2)], 1, 1, 0, 0, 0, 1, 1.0, 0.0, 0.0)


def test_wrappers_refuse_cpu_tensors():
    x = torch.zeros(4, 8)
    eight = sk.Packed(torch.zeros(2, 8, 16, dtype=torch.int8), torch.zeros(2, 8), 8)
    for call in (lambda: sk.sinkhorn_norm(x), lambda: sk.sinkhorn_residual_norm(x, x), lambda: sk.sinkhorn_pack(x),
                 lambda: sk.sinkhorn_unpack(eight), lambda: sk.sinkhorn_activation(x, "silu"),
                 lambda: sk.sinkhorn_expert_product_packed(x, eight, torch.zeros(3, dtype=torch.int32)),
                 lambda: sk.sinkhorn_expert_product_kept(x.bfloat16(), torch.zeros(2, 8, 8).bfloat16(),
                                                         torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(TypeError):
            call()
