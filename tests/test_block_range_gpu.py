"""Kept products in float16 whose gradient between product and activation 16 bits do not hold, though the result's are."""
import ctypes
import math

import pytest
import torch

import packed_util as ref
import paper_1907_01729_amd as sk
from paper_1907_01729_amd._binding import SkExperts, SkPacking
from routed_util import order_of, products, rounding

pytestmark = pytest.mark.gpu
F16 = torch.float16
U = 2.0 ** -24


def gen(seed):
    return torch.Generator().manual_seed(seed)


def case(kind, gated, gathered, large):
    """Gradients of the activated rows that 16 bits do not hold (large: about 6e5; else 2e-7, a few of the smallest steps),
    and rows whose other half, or whose derivative, brings them back: gated rows of 1e-6 or of 150 and 1e3; without a gate a silu
    far below zero, whose derivative is 2e-6, or a relu's inactive rows."""
    T, E, k, K, N = 60, 3, 2, 72, 40
    offsets, tokens, slots = (t.cuda() for t in order_of(torch.rand(T, E, generator=gen(1)).topk(k, 1).indices.int(), E))
    if not gathered:
        T, k, tokens, slots = T * k, 1, None, None

    def around(*shape, seed):  # of size 1 to 2, either sign
        u = 2 * torch.rand(*shape, generator=gen(seed)) - 1
        return u + u.sign()
    x = around(T, K * (1 + gated), seed=2)
    if gated:
        x = x * (1e-6 if large else torch.tensor([150.0, 1e3]).repeat_interleave(K))
    elif kind == "relu":
        x = -x.abs()
    else:
        x = -15.8 + 0.2 * x
    by = math.sqrt(1e5) if large else 2.0 ** -13
    w, gy = around(E, N, K, seed=3) * by, around(T * k, N, seed=4) * by
    leaf = lambda t: t.to(F16).cuda().requires_grad_()  # noqa: E731
    return leaf(x), leaf(w), gy.to(F16).cuda(), offsets, tokens, slots


@pytest.mark.parametrize("kind,gated,large", [("none", True, True), ("silu", True, True), ("gelu", True, True),
                                              ("silu", False, True), ("relu", False, True), ("none", True, False),
                                              ("silu", True, False)])
@pytest.mark.parametrize("gathered", [True, False])
def test_gradients_between_product_and_activation(kind, gated, large, gathered):
    x, w, gy, offsets, tokens, slots = case(kind, gated, gathered, large)
    y = sk.sinkhorn_expert_product_kept(x, w, offsets, tokens, slots, kind, gated)
    gx, = torch.autograd.grad(y, x, gy)
    W, G, o = w.detach().cpu().double(), gy.cpu().double(), offsets.cpu()
    t = None if tokens is None else tokens.cpu()
    kept = ref.unpack(*ref.pack(x, 128), 128).requires_grad_()
    a = ref.activate(kept, kind, gated)
    p = products(a.detach(), W, o, t, G)
    ga, K = p["gx"], w.shape[2]
    size = float(ga.abs().median())
    assert size > 2 * 65504 if large else size < 2.0 ** -20
    want, = torch.autograd.grad(a, kept, ga, retain_graph=True)
    assert float(want.abs().max()) < 65504
    # In units of 32 bits: the sums of N and of the slots' terms; the activation's value and derivative within
    # 12 (1 + |v|)^2 of terms of at most 1 + |v| times their size; and one rounding to 16 bits.
    v, u = kept.detach()[:, :K], kept.detach()[:, K:] if gated else torch.ones(1, dtype=torch.float64)
    sums, own = (w.shape[1] + 4) * U, 12 * U * (1 + v.abs()) ** 2
    slope, = torch.autograd.grad(a, kept, p["abs_gx"])
    off = sums * slope.abs()
    if kind != "relu":  # whose derivative is exact
        off[:, :K] += own * p["abs_gx"] * (u.abs() if gated else slope.abs() / p["abs_gx"])
    if gated:
        off[:, K:] += own * p["abs_gx"] * v.abs()
    assert bool(((gx.cpu().double() - want).abs() <= off + rounding(want, F16)).all())


# ---- the C entries with gradients in 32 bits ----

def _stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("dtype,code", [(torch.bfloat16, 1), (F16, 2)])
@pytest.mark.parametrize("T,E,k,K,N", [(1, 1, 1, 1, 1), (60, 3, 2, 72, 40), (90, 3, 1, 33, 17), (700, 2, 2, 264, 520)])
@pytest.mark.parametrize("gathered", [True, False])
def test_input_gradient_in_32_bits(T, E, k, K, N, dtype, code, gathered):
    """Rounded, it is the one in 16 bits."""
    offsets, tokens, slots = (t.cuda() for t in order_of(torch.rand(T, E, generator=gen(1)).topk(k, 1).indices.int(), E))
    rows = T if gathered else T * k
    w = torch.randn(E, N, K, generator=gen(2)).to(dtype).cuda()
    gy = torch.randn(T * k, N, generator=gen(3)).to(dtype).cuda()
    p = SkExperts(*((T, k) if gathered else (T * k, 1)), E, K, N, code)
    lib, ref_p = sk.load_library(), ctypes.byref(p)
    need = lib.sinkhorn_experts_workspace_bytes(ref_p)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    got = torch.full((rows + 1, K), 7.0, device="cuda")
    assert lib.sinkhorn_experts_backward_input32(ref_p, gy.data_ptr(), w.data_ptr(), offsets.data_ptr(),
                                                 slots.data_ptr() if gathered else None, got.data_ptr(), ws.data_ptr(),
                                                 need, _stream()) == 0
    want = sk.sinkhorn_experts_backward_input(gy, w, offsets, slots if gathered else None)
    assert torch.equal(got[:rows].to(dtype), want) and bool((got[rows] == 7).all())


@pytest.mark.parametrize("dtype,code", [(torch.float32, 0), (torch.bfloat16, 1), (F16, 2)])
@pytest.mark.parametrize("kind", range(4))
@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("T,K", [(1, 1), (37, 60), (5, 256)])
def test_activation_gradient_from_32_bits(T, K, kind, gated, dtype, code):
    """Of numbers that both types hold: the same bits."""
    x = torch.randn(T, K * (1 + gated), generator=gen(1)).to(dtype).cuda()
    gy = torch.randn(T, K, generator=gen(2)).to(dtype).cuda()
    packed = sk.sinkhorn_pack(x, 128)
    p, lib = ctypes.byref(SkPacking(T, K * (1 + gated), 128, code)), sk.load_library()
    got, want = [], []
    for out, call, g in ((got, lib.sinkhorn_activation_backward32, gy.float()), (want, lib.sinkhorn_activation_backward, gy)):
        out += [torch.full((T + 1, K), 7.0, dtype=dtype, device="cuda"), torch.full_like(torch.cat((x, x[:1])), 7.0)]
        assert call(p, kind, gated, packed.values.data_ptr(), packed.scales.data_ptr(), g.data_ptr(), out[0].data_ptr(),
                    out[1].data_ptr(), _stream()) == 0
    for u, v in zip(got, want):
        assert torch.equal(u, v) and bool((u[-1] == 7).all())
